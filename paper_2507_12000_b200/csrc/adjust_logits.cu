// Penalties for repeated tokens, biases and masks on the rows of logits of a drafted tree: two kernels.
//
// The copy (out of place, or where there are masks) passes the rows by vectors of 16 bytes; what a mask bans becomes -inf. It knows nothing
// of tokens, and is bound by memory.
//
// The patch then writes the entries that a penalty or a bias concerns, a few hundred of a row's 10^5.  Which they are, and how often each
// occurred, is counted in shared memory in a hash table of the sequence's own tokens: whole numbers, so that the order of the atomics
// changes nothing.  A table over the vocabulary would be 4 V bytes per sequence to clear, fill and read; counting by slices of the
// vocabulary in each CTA took 406 us for B=256 N=5 V=151936 in place (9728 CTAs that each read the history), and taking the touched vectors apart
// on the way made the copy of B=32 N=24 V=128256 issue-bound (141 us).  Where a sequence has more tokens than the table holds, the vocabulary is
// taken in ranges of the table's size and the table is indexed directly: it cannot overflow either way.
// The tokens drafted on a row's own way from the root are few and differ from row to row: an entry that is drafted anywhere walks up from its
// node.
#include "launch.h"
#include "quads.cuh"
#include "tree.cuh"
#include "tree_ops.h"

namespace dssd {

namespace {

template <int DT>
struct Vec;
template <>
struct Vec<DSSD_F32> {
    typedef uint32_t Word;
    static constexpr int kN = 4;
    static constexpr uint32_t kNegInf = 0xff800000u;
    __device__ static float value(Word w) { return __uint_as_float(w); }
    __device__ static Word bits(float x) { return __float_as_uint(x); }
    __device__ static Word load(const void *p) { return ld_row_u32(p); }
    // the entries of v whose bit of `allow` is clear become -inf
    __device__ static uint4 ban(const uint4 &v, uint32_t allow)
    {
        return make_uint4(allow & 1u ? v.x : kNegInf, allow & 2u ? v.y : kNegInf, allow & 4u ? v.z : kNegInf, allow & 8u ? v.w : kNegInf);
    }
};
template <>
struct Vec<DSSD_BF16> {
    typedef unsigned short Word;
    static constexpr int kN = 8;
    static constexpr uint32_t kNegInf = 0xff80u;
    __device__ static float value(Word w) { return __uint_as_float((uint32_t)w << 16); }
    __device__ static Word bits(float x)  // to nearest, ties to even; NaN stays NaN
    {
        unsigned short h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
        return h;
    }
    __device__ static Word load(const void *p) { return (Word)ld_row_u16(p); }
    __device__ static uint32_t ban2(uint32_t w, uint32_t allow)
    {
        return (allow & 1u ? w & 0xffffu : kNegInf) | (allow & 2u ? w & 0xffff0000u : kNegInf << 16);
    }
    __device__ static uint4 ban(const uint4 &v, uint32_t allow)
    {
        return make_uint4(ban2(v.x, allow), ban2(v.y, allow >> 2), ban2(v.z, allow >> 4), ban2(v.w, allow >> 6));
    }
};

// the mask of a row, or none
__device__ __forceinline__ const uint32_t *mask_of(const AdjustParams &P, long long row)
{
    if (!P.mask) return nullptr;
    const int m = P.mask_row ? ld_after(P.mask_row + row) : (int)row;
    return m >= 0 && m < P.mask_rows ? P.mask + (long long)m * ((P.V + 31) / 32) : nullptr;
}

// ---- the copy --------------------------------------------------------------------------------

constexpr int kCopyVecs = 8;  // of a thread

// kInPlace: only what a mask bans is written.  kVector: a row's entries lie alike to 16 bytes in both arrays.
template <int DT, bool kInPlace, bool kVector>
__global__ void __launch_bounds__(kThreads) adjust_copy_kernel(const __grid_constant__ AdjustParams P)
{
    typedef Vec<DT> E;
    typedef typename E::Word Word;
    constexpr uint32_t kAll = (1u << E::kN) - 1u;
    __shared__ short parent[kMaxNodes];
    __shared__ int there;
    const int t = threadIdx.x;
    const long long row = blockIdx.x / (unsigned)P.turns;
    const int turn = blockIdx.x % (unsigned)P.turns;
    const long long b = row / P.N;
    const int node = (int)(row - b * P.N);
    pdl_wait();
    pdl_trigger();
    const char *in = static_cast<const char *>(P.logits) + row * P.row_stride * (long long)sizeof(Word);
    char *out = static_cast<char *>(P.out) + row * P.out_stride * (long long)sizeof(Word);
    const uint32_t *mask = mask_of(P, row);
    if (kInPlace && !mask) return;
    const int words = (P.V + 31) / 32;
    // vectors begin on 16-byte boundaries of memory: the first at most kN - 1 entries before the row
    const int mis = kVector ? (int)((reinterpret_cast<uintptr_t>(in) / sizeof(Word)) % E::kN) : 0;
    bool known = !P.parents;
    auto allowed = [&](int v) {
        uint32_t a = kAll;
        if (mask && v + E::kN > 0 && v < P.V) {
            const int vv = max(v, 0), w = vv >> 5;
            const uint32_t lo = ld_after_u32(mask + w);
            const uint32_t hi = (vv & 31) > 32 - E::kN && w + 1 < words ? ld_after_u32(mask + w + 1) : 0u;
            a = (__funnelshift_r(lo, hi, vv & 31) << (vv - v)) & kAll;
        }
        return a;
    };
    for (int piece = turn; piece < P.pieces; piece += P.turns) {
        const int v0 = piece * (kThreads * kCopyVecs * E::kN) - mis + t * E::kN;
        uint4 x[kCopyVecs];
        uint32_t a[kCopyVecs];
#pragma unroll
        for (int k = 0; k < kCopyVecs; ++k) a[k] = allowed(v0 + k * kThreads * E::kN);
#pragma unroll
        for (int k = 0; k < kCopyVecs; ++k) {
            const int v = v0 + k * kThreads * E::kN;
            x[k] = make_uint4(0, 0, 0, 0);
            // (a vector that is banned altogether is not read, nor in place one that is not banned at all)
            if (kVector && v >= 0 && v + E::kN <= P.V && a[k] && !(kInPlace && a[k] == kAll)) x[k] = ld_row16(in + (long long)v * sizeof(Word));
        }
        if (!known) {  // is there a node?  (looked up while the row is on its way)
            for (int j = t; j < P.N; j += kThreads) {
                const int p = j ? ld_after(P.parents + b * (P.N - 1) + j - 1) : 0;
                parent[j] = (short)(p >= j && j ? -1 : max(p, -1));
            }
            __syncthreads();
            if (t == 0) {
                int up = node;
                while (up > 0) up = parent[up];
                there = up == 0;
            }
            __syncthreads();
            if (!there) return;
            known = true;
        }
#pragma unroll
        for (int k = 0; k < kCopyVecs; ++k) {
            const int v = v0 + k * kThreads * E::kN;
            if (kVector && v >= 0 && v + E::kN <= P.V) {
                if (!(kInPlace && a[k] == kAll)) *reinterpret_cast<uint4 *>(out + (long long)v * sizeof(Word)) = a[k] == kAll ? x[k] : E::ban(x[k], a[k]);
                continue;
            }
            for (int i = 0; i < E::kN; ++i) {
                if (v + i < 0 || v + i >= P.V) continue;
                Word *to = reinterpret_cast<Word *>(out) + v + i;
                if (!((a[k] >> i) & 1u)) *to = (Word)E::kNegInf;
                else if (!kInPlace) *to = E::load(in + (long long)(v + i) * sizeof(Word));
            }
        }
    }
}

// ---- the patch -------------------------------------------------------------------------------

constexpr int kPatch = 512;  // threads
constexpr uint32_t kInPrompt = 1u << 30, kDrafted = 1u << 31, kCount = kInPrompt - 1;

// shared memory: key, count and the last bias (its place in the list + 1) of every slot, then the list of slots in use
struct Table {
    int *key;
    uint32_t *count;
    unsigned short *bias, *used;
    int slots, first, direct;  // direct: slot = token - first, for tokens first .. first + slots - 1
    __device__ __forceinline__ int find(int v) const
    {
        if (direct) {
            const int s = v - first;
            if (s < 0 || s >= slots) return -1;
            key[s] = v;  // (every writer stores the same)
            return s;
        }
        unsigned s = ((unsigned)v * 2654435761u) >> 7 & (unsigned)(slots - 1);
        while (true) {  // there are more slots than tokens: an empty one comes
            int old = *(volatile int *)&key[s];  // (frequent tokens are there already)
            if (old == -1) old = atomicCAS(&key[s], -1, v);
            if (old == -1 || old == v) return (int)s;
            s = (s + 1) & (unsigned)(slots - 1);
        }
    }
};

template <int DT>
__global__ void __launch_bounds__(kPatch) adjust_patch_kernel(const __grid_constant__ AdjustParams P)
{
    typedef Vec<DT> E;
    typedef typename E::Word Word;
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ int token[kMaxNodes];
    __shared__ short parent[kMaxNodes];
    __shared__ const uint32_t *masks[kMaxNodes];
    __shared__ int bad, n_used;
    __shared__ unsigned all_flags;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const long long b = blockIdx.x / (unsigned)P.shares;
    const int share = blockIdx.x % (unsigned)P.shares;
    Table T;
    T.key = reinterpret_cast<int *>(raw);
    T.count = reinterpret_cast<uint32_t *>(T.key + P.slots);
    T.bias = reinterpret_cast<unsigned short *>(T.count + P.slots);
    T.used = T.bias + P.slots;
    T.slots = P.slots;
    if (t == 0) all_flags = 0;
    // After the copy only the logits are waited for: the copy let this kernel in when what came before it had ended, so that all other
    // arrays are as they should be.
    bool waited = !P.after_copy;
    if (waited) {
        pdl_wait();
        pdl_trigger();
    }
    load_tree(P.parents, b, P.N, parent, &bad);  // (with barriers)

    unsigned flags = bad ? DSSD_ADJUST_FLAG_BAD_PARENT : 0u;
    float repetition = 1.f, presence = 0.f, frequency = 0.f;
    if (P.repetition) repetition = ld_after(P.repetition + b);
    if (P.presence) presence = ld_after(P.presence + b);
    if (P.frequency) frequency = ld_after(P.frequency + b);
    if (!(repetition > 0.f && repetition < __int_as_float(0x7f800000))) {
        repetition = 1.f;
        flags |= DSSD_ADJUST_FLAG_BAD_VALUE;
    }
    int hl = P.L ? ld_after(P.history_len + b) : 0;
    const int pl = P.L ? ld_after(P.prompt_len + b) : 0;
    if (hl < 0 || hl > P.L) {
        hl = hl < 0 ? 0 : P.L;
        flags |= DSSD_ADJUST_FLAG_BAD_LENGTH;
    }
    if (t < P.N) {
        masks[t] = mask_of(P, b * P.N + t);
        if (t > 0) {
            token[t] = ld_after(P.draft_tokens + b * (P.N - 1) + t - 1);
            if (parent[t] >= 0 && (token[t] < 0 || token[t] >= P.V)) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
        }
        if (P.mask && P.mask_row && parent[t] >= 0 && ld_after(P.mask_row + b * P.N + t) >= P.mask_rows) flags |= DSSD_ADJUST_FLAG_BAD_MASK;
    }
    // With fewer tokens than three quarters of the slots the table is a hash table of all of them; else the vocabulary is taken in ranges.
    T.direct = (long long)hl + P.N + P.K > (long long)T.slots * 3 / 4;
    const int32_t *hist = P.history + b * P.history_stride;
    const int ranges = T.direct ? (P.V + T.slots - 1) / T.slots : 1;
    // the ranges are shared out first, what is in a range (or the one table) by the rows
    const int r_step = T.direct ? P.shares : 1, p_from = T.direct ? 0 : share, p_step = T.direct ? 1 : P.shares;
    for (int range = T.direct ? share : 0; range < ranges; range += r_step) {
        T.first = range * T.slots;
        __syncthreads();
        for (int i = t; i < T.slots; i += kPatch) T.key[i] = -1, T.count[i] = 0, T.bias[i] = 0;
        if (t == 0) n_used = 0;
        __syncthreads();
        // in eights: the tokens come from L2, and a request at a time would wait for each
        for (int i0 = t; i0 < hl; i0 += 8 * kPatch) {
            int tok[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) tok[u] = i0 + u * kPatch < hl ? ld_after(hist + i0 + u * kPatch) : 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * kPatch;
                if (i >= hl) break;
                if (tok[u] < 0 || tok[u] >= P.V) {
                    flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
                    continue;
                }
                const int s = T.find(tok[u]);
                if (s < 0) continue;
                if (i < pl) atomicOr(&T.count[s], kInPrompt);
                else atomicAdd(&T.count[s], 1u);
            }
        }
        if (t > 0 && t < P.N && parent[t] >= 0 && token[t] >= 0 && token[t] < P.V) {
            const int s = T.find(token[t]);
            if (s >= 0) atomicOr(&T.count[s], kDrafted);
        }
        // of a token's biases the last one holds: whoever stores first does not matter, the largest index stays
        for (int k0 = 0; k0 < P.K; k0 += kPatch) {
            const int k = k0 + t;
            const int v = k < P.K ? ld_after(P.bias_tokens + b * P.K + k) : -1;
            if (v >= P.V) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
            const int s = v >= 0 && v < P.V ? T.find(v) : -1;
            bool waiting = s >= 0;
            while (__syncthreads_or(waiting)) {
                if (waiting) T.bias[s] = (unsigned short)(k + 1);
                __syncthreads();
                if (waiting) waiting = T.bias[s] < (unsigned short)(k + 1);
            }
        }
        __syncthreads();
        for (int i = t; i < T.slots; i += kPatch) {  // (slots are a multiple of the threads)
            const bool in_use = T.key[i] >= 0;
            const unsigned who = __ballot_sync(0xffffffffu, in_use);
            int at = 0;
            if (lane == 0 && who) at = atomicAdd(&n_used, __popc(who));
            at = __shfl_sync(0xffffffffu, at, 0);
            if (in_use) T.used[at + __popc(who & ((1u << lane) - 1u))] = (unsigned short)i;
        }
        __syncthreads();
        if (!waited) {
            pdl_wait();
            pdl_trigger();
            waited = true;
        }
        // (entry, row) pairs: a warp takes 256 entries of a row at a time, eight requests in flight to a lane
        const int n = n_used, blocks = (n + 255) / 256;
        const int rows = (P.N - p_from + p_step - 1) / p_step;
        for (int unit = warp; unit < rows * blocks; unit += kPatch / 32) {
            const int r = unit / blocks, node = p_from + r * p_step;
            if (parent[node] < 0) continue;
            const long long row = b * P.N + node;
            const char *in = static_cast<const char *>(P.logits) + row * P.row_stride * (long long)sizeof(Word);
            Word *out = static_cast<Word *>(P.out) + row * P.out_stride;
            const uint32_t *mask = masks[node];
            constexpr int kAtOnce = 8;
            const int e0 = (unit - r * blocks) * 256 + lane;
            int slot[kAtOnce], v[kAtOnce];
            Word w[kAtOnce];
            uint32_t allow[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int e = e0 + u * 32;
                slot[u] = e < n ? T.used[e] : -1;
                v[u] = slot[u] >= 0 ? T.key[slot[u]] : 0;
                w[u] = slot[u] >= 0 ? E::load(in + (long long)v[u] * sizeof(Word)) : 0;
                allow[u] = mask && slot[u] >= 0 ? ld_after_u32(mask + (v[u] >> 5)) >> (v[u] & 31) : 1u;
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (slot[u] < 0 || !(allow[u] & 1u)) continue;
                const uint32_t c = T.count[slot[u]];
                const unsigned k = T.bias[slot[u]];
                uint32_t n_out = c & kCount;
                if (c & kDrafted)
                    for (int j = node; j > 0; j = parent[j]) n_out += token[j] == v[u];
                if (!(n_out | (c & kInPrompt) | k)) continue;  // drafted on other ways only
                float x = E::value(w[u]);
                if (n_out || (c & kInPrompt)) x = x > 0.f ? __fdiv_rn(x, repetition) : __fmul_rn(x, repetition);
                if (n_out) x = __fsub_rn(__fsub_rn(x, __fmul_rn(frequency, (float)n_out)), presence);
                if (k) x = __fadd_rn(x, ld_after(P.bias_values + b * P.K + k - 1));
                out[v[u]] = E::bits(x);
            }
        }
    }
    if (!waited) {  // (a share without a range)
        pdl_wait();
        pdl_trigger();
    }
    if (share == 0 && P.flags) {
        // (in ranges, a range sees all tokens; every CTA of the sequence sees the same flags)
        flags = __reduce_or_sync(0xffffffffu, flags);
        if ((t & 31) == 0 && flags) atomicOr(&all_flags, flags);
        __syncthreads();
        if (t == 0) P.flags[b] = all_flags;
    }
}

constexpr int kMaxSlots = 16384;

template <int DT>
cudaError_t patch(const AdjustParams &P, cudaStream_t stream)
{
    const size_t smem = (size_t)P.slots * 12;
    if (smem > 40 * 1024) {  // (with what is declared in the kernel, beyond the 48 KB that need no leave)
        static PerContext allowed;
        if (!allowed.get([] { return (int)(cudaFuncSetAttribute(adjust_patch_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlots * 12) == cudaSuccess); })) {
            const cudaError_t e = cudaGetLastError();
            return e == cudaSuccess ? cudaErrorInvalidConfiguration : e;
        }
    }
    return launch_pdl(adjust_patch_kernel<DT>, (unsigned)P.B * (unsigned)P.shares, kPatch, stream, P, smem);
}

template <int DT, bool kInPlace>
cudaError_t copy(const AdjustParams &P, bool vector, cudaStream_t stream)
{
    const unsigned grid = (unsigned)((long long)P.B * P.N * P.turns);
    return vector ? launch_pdl(adjust_copy_kernel<DT, kInPlace, true>, grid, kThreads, stream, P)
                  : launch_pdl(adjust_copy_kernel<DT, kInPlace, false>, grid, kThreads, stream, P);
}

}  // namespace

int adjust_copy_entries(int dtype) { return kThreads * kCopyVecs * (dtype == DSSD_BF16 ? 8 : 4); }

cudaError_t adjust_launch(AdjustParams &P, int dtype, cudaStream_t stream)
{
    const int esz = dtype == DSSD_BF16 ? 2 : 4;
    const bool in_place = P.out == P.logits, bf = dtype == DSSD_BF16;
    // a vector store needs the two rows at the same place of a 16-byte line, for every row
    const uintptr_t a = reinterpret_cast<uintptr_t>(P.logits), c = reinterpret_cast<uintptr_t>(P.out);
    const bool vector = (a - c) % 16 == 0 && ((P.row_stride - P.out_stride) * esz) % 16 == 0;
    P.after_copy = !in_place || P.mask;
    if (P.after_copy) {
        const int per = adjust_copy_entries(dtype);
        const int most = P.V + (vector && (a % 16 || (P.row_stride * esz) % 16) ? 16 / esz - 1 : 0);  // with the entries before a row's start
        P.pieces = (most + per - 1) / per;
        // In place most rows have no mask as a rule, and a CTA that finds none has nothing to do: no more of them than fill the GPU.
        P.turns = P.pieces;
        while (in_place && P.turns > 1 && (long long)P.B * P.N * P.turns > 148 * 32) P.turns = (P.turns + 1) / 2;
        const cudaError_t e = bf ? (in_place ? copy<DSSD_BF16, true>(P, vector, stream) : copy<DSSD_BF16, false>(P, vector, stream))
                                 : (in_place ? copy<DSSD_F32, true>(P, vector, stream) : copy<DSSD_F32, false>(P, vector, stream));
        if (e != cudaSuccess) return e;
    }
    // a slot and a third for each token that there may be
    P.slots = 512;
    while (P.slots < kMaxSlots && (long long)P.slots * 3 / 4 < (long long)P.L + P.N + P.K) P.slots *= 2;
    // sequences alone on the GPU have their rows (or the ranges of a large table) shared out
    P.shares = 1;
    while (P.shares < 32 && (long long)P.B * P.shares < 2 * 148 && P.shares < P.N) P.shares *= 2;
    return bf ? patch<DSSD_BF16>(P, stream) : patch<DSSD_F32>(P, stream);
}

}  // namespace dssd
