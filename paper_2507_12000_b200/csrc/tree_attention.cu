// Attention of a drafted tree's nodes over a paged cache.
//
// The plain kernel: a CTA per (sequence, node, query head), a warp per key in turn, lanes along D, a running maximum and sum per
// warp, joined at the end.
#include "launch.h"
#include "quads.cuh"
#include "tree.cuh"
#include "tree_ops.h"

#include <cuda_bf16.h>

namespace dssd {

namespace {

template <int DT>
__device__ __forceinline__ float value(const void *p, int64_t i)
{
    const uint32_t h = ld_row_u16(static_cast<const char *>(p) + 2 * i);
    return DT == DSSD_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
template <int DT>
__device__ __forceinline__ unsigned short bits(float x)
{
    return DT == DSSD_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}

constexpr int kAT = 128;

template <int DT>
__global__ void __launch_bounds__(kAT) plain_attention_kernel(const __grid_constant__ TreeAttentionParams P)
{
    __shared__ short parent[kMaxNodes];
    __shared__ int bad;
    __shared__ float acc[4][128], top[4], sum[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int hq = blockIdx.x % (unsigned)P.Hq;
    const int j = (blockIdx.x / (unsigned)P.Hq) % (unsigned)P.N;
    const long long b = blockIdx.x / (unsigned)P.Hq / (unsigned)P.N;
    const int h = hq / (P.Hq / P.Hkv);
    pdl_wait();
    pdl_trigger();
    load_tree(P.parents, b, P.N, parent, &bad);
    unsigned flags = bad ? DSSD_CACHE_FLAG_BAD_NODE : 0u;
    const long long most = (long long)P.max_pages * P.page_size;
    int ctx = ld_after(P.ctx_len + b);
    if (ctx < 0 || ctx > most) {
        ctx = ctx < 0 ? 0 : (int)most;
        flags |= DSSD_CACHE_FLAG_BAD_LENGTH;
    }
    if (parent[j] >= 0) {
        float q[4], o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < 4; ++k) q[k] = lane + 32 * k < P.D ? value<DT>(P.q, b * P.q_b + j * P.q_n + hq * P.q_h + lane + 32 * k) * P.scale : 0.f;
        float m = DSSD_NEG_INF, l = 0.f;
        for (long long t = warp; t < (long long)ctx + P.N; t += 4) {
            const void *kp = P.k_cache, *vp = P.v_cache;
            int64_t at;
            if (t < ctx) {
                const int page = ld_after(P.block_table + b * P.table_stride + t / P.page_size);
                if (page < 0 || page >= P.num_pages) flags |= DSSD_CACHE_FLAG_BAD_PAGE;
                at = page < 0 || page >= P.num_pages ? -1 : page * P.cache_p + (t % P.page_size) * P.cache_t + h * P.cache_h;
            } else {
                const int i = (int)(t - ctx);
                int up = j;
                while (up > i) up = parent[up];
                if (up != i) continue;
                kp = P.k_new, vp = P.v_new;
                at = b * P.new_b + i * P.new_n + h * P.new_h;
            }
            float s = 0.f;
            for (int k = 0; k < 4; ++k)
                if (lane + 32 * k < P.D && at >= 0) s += q[k] * value<DT>(kp, at + lane + 32 * k);
            s = warp_sum(s);
            const float mn = fmaxf(m, s), w = expf(s - mn), f = expf(m - mn);
            m = mn;
            l = l * f + w;
            for (int k = 0; k < 4; ++k) o[k] = o[k] * f + (lane + 32 * k < P.D && at >= 0 ? w * value<DT>(vp, at + lane + 32 * k) : 0.f);
        }
        for (int k = 0; k < 4; ++k) acc[warp][lane + 32 * k] = o[k];
        if (lane == 0) top[warp] = m, sum[warp] = l;
        __syncthreads();
        float mt = DSSD_NEG_INF, lt = 0.f, ot = 0.f;
        for (int w = 0; w < 4; ++w) mt = fmaxf(mt, top[w]);
        for (int w = 0; w < 4; ++w) {
            const float f = top[w] == DSSD_NEG_INF ? 0.f : expf(top[w] - mt);
            lt += f * sum[w];
            ot += f * acc[w][threadIdx.x];
        }
        if (threadIdx.x < (unsigned)P.D)
            static_cast<unsigned short *>(P.o)[b * P.o_b + j * P.o_n + hq * P.o_h + threadIdx.x] = bits<DT>(ot / lt);
        if (threadIdx.x == 0 && P.lse) P.lse[(b * P.N + j) * P.Hq + hq] = mt + logf(lt);
    }
    if (flags && P.flags && lane == 0) atomicOr(P.flags + b, flags);
}

}  // namespace

size_t tree_attention_workspace(int B, int N, int Hq, int Hkv, int D)
{
    (void)B, (void)N, (void)Hq, (void)Hkv, (void)D;
    return 256;
}

cudaError_t tree_attention_launch(TreeAttentionParams &P, int dtype, void *workspace, cudaStream_t stream)
{
    (void)workspace;
    const unsigned grid = (unsigned)P.B * (unsigned)P.N * (unsigned)P.Hq;
    return dtype == DSSD_BF16 ? launch_pdl(plain_attention_kernel<DSSD_BF16>, grid, kAT, stream, P)
                              : launch_pdl(plain_attention_kernel<DSSD_F16>, grid, kAT, stream, P);
}

}  // namespace dssd
