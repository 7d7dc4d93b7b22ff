// Keys and values of the accepted path into the pages of the cache, for all layers in one launch.
//
// A warp takes one appended position of one sequence in a few layers: where it goes (the path's node, the
// page, the place in it) is looked up once, a chain of three loads that costs more than the copy of one row, and the rows of the
// layers are then copied by vectors of 16 bytes, the loads of several rows in flight together.
//
// Bound by the copy for whole prompts, by the look-up's latency for a handful of accepted tokens.
#include "launch.h"
#include "quads.cuh"
#include "tree.cuh"
#include "tree_ops.h"

namespace dssd {

namespace {

constexpr int kLayers = 4;  // layers of a warp
constexpr int kAtOnce = 4;  // pieces of K and of V that a lane has in flight

// the page of appended position i, or -1 with the reason in *flags
__device__ __forceinline__ int page_of(const AppendParams &P, long long b, int ctx, int i, int &place, unsigned &flags)
{
    const long long pos = (long long)ctx + i;
    const long long at = pos / P.page_size;
    place = (int)(pos - at * P.page_size);
    if (ctx < 0 || at >= P.max_pages) {
        flags |= DSSD_CACHE_FLAG_BAD_LENGTH;
        return -1;
    }
    const int page = ld_after(P.block_table + b * P.table_stride + at);
    if (page < 0 || page >= P.num_pages) {
        flags |= DSSD_CACHE_FLAG_BAD_PAGE;
        return -1;
    }
    return page;
}

__device__ __forceinline__ int node_of(const AppendParams &P, long long b, int i, unsigned &flags)
{
    const int node = P.path ? ld_after(P.path + b * P.N + i) : i;
    if (node < 0 || node >= P.N) {
        flags |= DSSD_CACHE_FLAG_BAD_NODE;
        return -1;
    }
    return node;
}

template <class Word>
__device__ __forceinline__ Word piece(const void *p);
template <>
__device__ __forceinline__ uint4 piece<uint4>(const void *p) { return ld_row16(p); }
template <>
__device__ __forceinline__ unsigned short piece<unsigned short>(const void *p) { return (unsigned short)ld_row_u16(p); }

// Word: a piece of the copy
template <class Word>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendParams P)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned chunks = (unsigned)((P.N + kWarps - 1) / kWarps);
    const unsigned groups = (unsigned)((P.layers + kLayers - 1) / kLayers);
    const unsigned chunk = blockIdx.x % chunks, rest = blockIdx.x / chunks;
    const int l0 = (int)(rest % groups) * kLayers;
    const long long b = rest / groups;
    const int i = (int)chunk * kWarps + warp;
    pdl_wait();
    pdl_trigger();
    const int last = ld_after(P.accept_len + b), ctx = ld_after(P.ctx_len + b);
    const int count = max(min(last, P.N - 1), -1) + 1;
    if (l0 == 0 && chunk == 0) {  // one CTA reports for the sequence
        unsigned flags = last >= P.N ? DSSD_CACHE_FLAG_BAD_NODE : 0u;
        for (int k = threadIdx.x; k < count; k += kThreads) {
            int place;
            node_of(P, b, k, flags);
            page_of(P, b, ctx, k, place, flags);
        }
        flags = __reduce_or_sync(0xffffffffu, flags);
        __shared__ unsigned all;
        if (threadIdx.x == 0) all = 0;
        __syncthreads();
        if (lane == 0 && flags) atomicOr(&all, flags);
        __syncthreads();
        if (threadIdx.x == 0) {
            if (P.flags) P.flags[b] = all;
            if (P.new_len) P.new_len[b] = ctx + count;
        }
    }
    if (i >= count) return;
    unsigned flags = 0;
    int place;
    const int node = node_of(P, b, i, flags);
    const int page = page_of(P, b, ctx, i, place, flags);
    if (node < 0 || page < 0) return;
    constexpr int kPer = sizeof(Word) / 2;  // elements of a piece
    const int per_head = P.D / kPer, pieces = P.Hkv * per_head;
    const int64_t from0 = b * P.new_b + node * P.new_n, to0 = page * P.cache_p + place * P.cache_t;
    const int items = min(kLayers, P.layers - l0) * pieces;
    for (int x0 = lane; x0 < items; x0 += 32 * kAtOnce) {
        Word k[kAtOnce], v[kAtOnce];
        int64_t to[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int x = x0 + 32 * u;
            if (x >= items) continue;
            const int l = x / pieces, e = x - l * pieces, h = e / per_head, d = (e - h * per_head) * kPer;
            const int64_t from = from0 + h * P.new_h + d + (l0 + l) * P.new_l;
            to[u] = to0 + h * P.cache_h + d + (l0 + l) * P.cache_l;
            k[u] = piece<Word>(static_cast<const unsigned short *>(P.k_new) + from);
            v[u] = piece<Word>(static_cast<const unsigned short *>(P.v_new) + from);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (x0 + 32 * u >= items) continue;
            *reinterpret_cast<Word *>(static_cast<unsigned short *>(P.k_cache) + to[u]) = k[u];
            *reinterpret_cast<Word *>(static_cast<unsigned short *>(P.v_cache) + to[u]) = v[u];
        }
    }
}

}  // namespace

cudaError_t append_launch(AppendParams &P, cudaStream_t stream)
{
    const long long grid = (long long)P.B * ((P.N + kWarps - 1) / kWarps) * ((P.layers + kLayers - 1) / kLayers);
    const int64_t strides = P.new_l | P.new_b | P.new_n | P.new_h | P.cache_l | P.cache_p | P.cache_t | P.cache_h;
    const uintptr_t bases = reinterpret_cast<uintptr_t>(P.k_new) | reinterpret_cast<uintptr_t>(P.v_new) |
                            reinterpret_cast<uintptr_t>(P.k_cache) | reinterpret_cast<uintptr_t>(P.v_cache);
    if (strides % 8 == 0 && P.D % 8 == 0 && bases % 16 == 0) return launch_pdl(append_kernel<uint4>, (unsigned)grid, kThreads, stream, P);
    return launch_pdl(append_kernel<unsigned short>, (unsigned)grid, kThreads, stream, P);
}

}  // namespace dssd
