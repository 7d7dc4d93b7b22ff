// Penalties for repeated tokens, biases and masks on the rows of logits of a drafted tree.
//
// What a token's logit needs is how often the token occurred.  A CTA takes a slice of one sequence's
// vocabulary and counts, in shared memory and in whole numbers (so that the order of the atomics changes nothing), the
// history's tokens that fall into it; the history is a few KB that every CTA of the sequence reads from L2, where a table
// of counts over the vocabulary would be 4 V bytes to clear, fill and read per sequence.  A bitmap says which entries anything
// concerns at all.  The rows of all nodes are then passed through the slice by vectors of 16 bytes: a vector that nothing
// concerns is copied (or, in place, not even read); the others are taken apart.  The tokens drafted on a row's own way from the root are
// few and differ from row to row: an entry that is drafted anywhere walks up from its node.
//
// Bound by the copy of the rows, or in place by the rows' masked and touched entries.
#include "launch.h"
#include "tree.cuh"
#include "tree_ops.h"

namespace dssd {

namespace {

constexpr int kSliceMax = 4096;
constexpr uint32_t kInPrompt = 1u << 30, kDrafted = 1u << 31, kCount = kInPrompt - 1;
constexpr unsigned kNoBias = 0xffffu;

struct AdjustSmem {
    uint32_t count[kSliceMax];
    unsigned short bias[kSliceMax];       // the last entry of the list for the token, kNoBias: none
    uint32_t touched[kSliceMax / 32 + 1];
    int token[kMaxNodes];
    short parent[kMaxNodes];
    int bad;
    unsigned flags;
};

template <int DT>
struct Vec;
template <>
struct Vec<DSSD_F32> {
    static constexpr int kN = 4;
    __device__ static float get(const uint4 &v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
    __device__ static uint32_t bits(float x) { return __float_as_uint(x); }
    __device__ static void set(uint4 &v, int i, uint32_t w) { (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = w; }
    static constexpr uint32_t kNegInf = 0xff800000u;
    typedef uint32_t Word;
};
template <>
struct Vec<DSSD_BF16> {
    static constexpr int kN = 8;
    __device__ static float get(const uint4 &v, int i)
    {
        const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return (i & 1) ? bf16_hi(w) : bf16_lo(w);
    }
    // to nearest, ties to even; NaN stays NaN
    __device__ static uint32_t bits(float x)
    {
        unsigned short h;
        asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
        return h;
    }
    __device__ static void set(uint4 &v, int i, uint32_t h)
    {
        uint32_t &w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        w = (i & 1) ? (w & 0xffffu) | (h << 16) : (w & 0xffff0000u) | h;
    }
    static constexpr uint32_t kNegInf = 0xff80u;
    typedef unsigned short Word;
};

__device__ __forceinline__ uint4 ld16(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

struct Penalty {
    float repetition, presence, frequency;
};

// the new value of the entry at `off` of the slice in node `node`'s row
__device__ float adjusted(const AdjustSmem &S, const AdjustParams &P, const Penalty &pen, long long b, int node, int v, int off, float x)
{
    const uint32_t c = S.count[off];
    uint32_t n_out = c & kCount;
    if (c & kDrafted)
        for (int j = node; j > 0; j = S.parent[j]) n_out += S.token[j] == v;
    if (n_out || (c & kInPrompt)) x = x > 0.f ? __fdiv_rn(x, pen.repetition) : x * pen.repetition;
    x = __fsub_rn(x, __fmul_rn(pen.frequency, (float)n_out));
    if (n_out) x = __fsub_rn(x, pen.presence);
    const unsigned k = S.bias[off];
    if (k != kNoBias) x = __fadd_rn(x, ld_after(P.bias_values + b * P.K + k));
    return x;
}

template <int DT, bool kInPlace, bool kVector>
__global__ void __launch_bounds__(kThreads) adjust_kernel(const __grid_constant__ AdjustParams P)
{
    extern __shared__ __align__(16) unsigned char raw[];
    AdjustSmem &S = *reinterpret_cast<AdjustSmem *>(raw);
    typedef Vec<DT> E;
    typedef typename E::Word Word;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const long long b = blockIdx.x / (unsigned)P.slices;
    const int sl = blockIdx.x % (unsigned)P.slices;
    const int v0 = sl * P.slice, v1 = min(P.V, v0 + P.slice);
    pdl_wait();
    pdl_trigger();

    for (int i = t; i < P.slice; i += kThreads) S.count[i] = 0, S.bias[i] = (unsigned short)kNoBias;
    for (int i = t; i <= P.slice / 32; i += kThreads) S.touched[i] = 0;
    if (t == 0) S.flags = 0;
    load_tree(P.parents, b, P.N, S.parent, &S.bad);  // (with barriers)

    unsigned flags = 0;
    if (S.bad) flags |= DSSD_ADJUST_FLAG_BAD_PARENT;
    Penalty pen = {1.f, 0.f, 0.f};
    if (P.repetition) pen.repetition = ld_after(P.repetition + b);
    if (P.presence) pen.presence = ld_after(P.presence + b);
    if (P.frequency) pen.frequency = ld_after(P.frequency + b);
    if (!(pen.repetition > 0.f && pen.repetition < __int_as_float(0x7f800000))) {
        pen.repetition = 1.f;
        flags |= DSSD_ADJUST_FLAG_BAD_VALUE;
    }
    int hl = P.L ? ld_after(P.history_len + b) : 0, pl = P.L ? ld_after(P.prompt_len + b) : 0;
    if (hl < 0 || hl > P.L) {
        hl = hl < 0 ? 0 : P.L;
        flags |= DSSD_ADJUST_FLAG_BAD_LENGTH;
    }
    // in eights: the tokens come from L2, and a request at a time would wait for each
    const int32_t *hist = P.history + b * P.history_stride;
    for (int i0 = t; i0 < hl; i0 += 8 * kThreads) {
        int tok[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) tok[u] = i0 + u * kThreads < hl ? ld_after(hist + i0 + u * kThreads) : v0 - 1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int v = tok[u], i = i0 + u * kThreads;
            if (i < hl && (v < 0 || v >= P.V)) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
            if (i < hl && v >= v0 && v < v1) {
                if (i < pl) atomicOr(&S.count[v - v0], kInPrompt);
                else atomicAdd(&S.count[v - v0], 1u);
                atomicOr(&S.touched[(v - v0) >> 5], 1u << ((v - v0) & 31));
            }
        }
    }
    if (t > 0 && t < P.N) {
        const int v = ld_after(P.draft_tokens + b * (P.N - 1) + t - 1);
        const bool there = S.parent[t] >= 0;
        S.token[t] = v;
        if (there && (v < 0 || v >= P.V)) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
        if (there && v >= v0 && v < v1) {
            atomicOr(&S.count[v - v0], kDrafted);
            atomicOr(&S.touched[(v - v0) >> 5], 1u << ((v - v0) & 31));
        }
    }
    __syncthreads();
    // The last entry for a token holds: whoever stores first does not matter, the largest index stays.
    for (int k0 = 0; k0 < P.K; k0 += kThreads) {
        const int k = k0 + t;
        const int v = k < P.K ? ld_after(P.bias_tokens + b * P.K + k) : -1;
        if (v >= P.V) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
        const bool mine = v >= v0 && v < v1;
        if (mine) atomicOr(&S.touched[(v - v0) >> 5], 1u << ((v - v0) & 31));
        // entries of later turns overwrite those of earlier ones; within a turn the largest k wins after at most as many steps
        // as a token has entries in it
        bool waiting = mine;
        __syncthreads();
        while (__syncthreads_or(waiting)) {
            if (waiting) S.bias[v - v0] = (unsigned short)k;
            __syncthreads();
            if (waiting) waiting = S.bias[v - v0] < (unsigned short)k;
        }
    }
    if (sl == 0 && P.flags) {
        if (P.mask_row && t < P.N && S.parent[t] >= 0 && ld_after(P.mask_row + b * P.N + t) >= P.mask_rows) flags |= DSSD_ADJUST_FLAG_BAD_MASK;
        if (flags) atomicOr(&S.flags, flags);
    }
    __syncthreads();
    if (sl == 0 && t == 0 && P.flags) P.flags[b] = S.flags;

    const int words = (P.V + 31) / 32;
    const int units = P.N * P.segments;
    for (int u = warp; u < units; u += kWarps) {
        const int node = u / P.segments, seg = u - node * P.segments;
        if (S.parent[node] < 0) continue;
        const long long row = b * P.N + node;
        const char *in = static_cast<const char *>(P.logits) + row * P.row_stride * (long long)sizeof(Word);
        char *out = static_cast<char *>(P.out) + row * P.out_stride * (long long)sizeof(Word);
        const uint32_t *mask = nullptr;
        if (P.mask) {
            const int m = P.mask_row ? ld_after(P.mask_row + row) : (int)row;
            if (m >= 0 && m < P.mask_rows) mask = P.mask + (long long)m * words;
        }
        // vectors begin on 16-byte boundaries of memory: entry `base` of the row, at most kN - 1 before the slice
        const int mis = kVector ? (int)((reinterpret_cast<uintptr_t>(in) / sizeof(Word) + v0) % E::kN) : 0;
        const int base = v0 - mis + seg * 1024;
        constexpr int kVecs = 1024 / E::kN / 32;  // of a lane
#pragma unroll
        for (int h = 0; h < kVecs; h += 4) {
            uint32_t hit[4], allow[4];
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int v = base + ((h + k) * 32 + lane) * E::kN;
                const int lo = max(v0 - v, 0), n = min(v1 - v, E::kN);  // entries lo .. n-1 of the vector are in the slice
                const uint32_t in_slice = n > lo ? ((1u << n) - 1u) & ~((1u << lo) - 1u) : 0u;
                hit[k] = 0;
                allow[k] = (1u << E::kN) - 1u;
                if (in_slice) {
                    const int off = v - v0;
                    // (bits before the slice are not looked at: shifted in as zeros)
                    const int o = max(off, 0), w = o >> 5;
                    const uint32_t two = __funnelshift_r(S.touched[w], w < P.slice / 32 ? S.touched[w + 1] : 0u, o & 31);
                    hit[k] = (two << (o - off)) & in_slice;
                    if (mask) {
                        const int vv = max(v, 0), mw = vv >> 5;
                        const uint32_t a = ld_after_u32(mask + mw);
                        const uint32_t c = (vv & 31) > 32 - E::kN && mw + 1 < words ? ld_after_u32(mask + mw + 1) : 0u;
                        allow[k] = ((__funnelshift_r(a, c, vv & 31) << (vv - v)) & in_slice) | (~in_slice & allow[k]);
                    }
                }
                x[k] = make_uint4(0, 0, 0, 0);
                const uint32_t live = kInPlace ? hit[k] & allow[k] : allow[k] & in_slice;  // entries whose old value matters
                const bool partly = in_slice != (1u << E::kN) - 1u || !kVector;
                const bool store_all = !kInPlace || hit[k] || (~allow[k] & in_slice);
                // a vector that is written at all is written whole: what stays as it is has to be read
                const bool need = !partly && store_all && (kInPlace ? (allow[k] != 0) : live != 0);
                if (need) x[k] = ld16(in + (long long)v * sizeof(Word));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int v = base + ((h + k) * 32 + lane) * E::kN;
                const int lo = max(v0 - v, 0), n = min(v1 - v, E::kN);
                if (n <= lo) continue;
                const bool whole = lo == 0 && n == E::kN && kVector;
                const uint32_t all = (1u << E::kN) - 1u;
                if (whole) {
                    if (kInPlace && hit[k] == 0 && allow[k] == all) continue;
                    if (hit[k] | (~allow[k] & all)) {
#pragma unroll
                        for (int i = 0; i < E::kN; ++i) {
                            if (!((allow[k] >> i) & 1u)) E::set(x[k], i, E::kNegInf);
                            else if ((hit[k] >> i) & 1u) E::set(x[k], i, E::bits(adjusted(S, P, pen, b, node, v + i, v + i - v0, E::get(x[k], i))));
                        }
                    }
                    *reinterpret_cast<uint4 *>(out + (long long)v * sizeof(Word)) = x[k];
                } else {
                    for (int i = lo; i < n; ++i) {
                        Word *to = reinterpret_cast<Word *>(out) + v + i;
                        if (!((allow[k] >> i) & 1u)) {
                            *to = (Word)E::kNegInf;
                            continue;
                        }
                        const bool touch = (hit[k] >> i) & 1u;
                        if (kInPlace && !touch) continue;
                        Word w = *(reinterpret_cast<const volatile Word *>(in) + v + i);
                        if (touch) {
                            const float f = sizeof(Word) == 4 ? __uint_as_float((uint32_t)w) : __uint_as_float((uint32_t)w << 16);
                            w = (Word)E::bits(adjusted(S, P, pen, b, node, v + i, v + i - v0, f));
                        }
                        *to = w;
                    }
                }
            }
        }
    }
}

template <int DT, bool kInPlace>
cudaError_t launch_as(const AdjustParams &P, bool vector, cudaStream_t stream)
{
    const unsigned grid = (unsigned)((long long)P.B * P.slices);
    return vector ? launch_pdl(adjust_kernel<DT, kInPlace, true>, grid, kThreads, stream, P, sizeof(AdjustSmem))
                  : launch_pdl(adjust_kernel<DT, kInPlace, false>, grid, kThreads, stream, P, sizeof(AdjustSmem));
}

}  // namespace

cudaError_t adjust_launch(AdjustParams &P, int dtype, cudaStream_t stream)
{
    const int esz = dtype == DSSD_BF16 ? 2 : 4;
    const bool in_place = P.out == P.logits;
    // a vector store needs the two rows at the same place of a 16-byte line, for every row
    const uintptr_t a = reinterpret_cast<uintptr_t>(P.logits), c = reinterpret_cast<uintptr_t>(P.out);
    const bool vector = (a - c) % 16 == 0 && ((P.row_stride - P.out_stride) * esz) % 16 == 0;
    P.slice = kSliceMax;
    while (P.slice > 1024 && (long long)P.B * ((P.V + P.slice - 1) / P.slice) < 4 * 148) P.slice /= 2;
    P.slices = (P.V + P.slice - 1) / P.slice;
    P.segments = P.slice / 1024 + (vector ? 1 : 0);
    if (vector && a % 16 == 0 && (P.row_stride * esz) % 16 == 0) P.segments = P.slice / 1024;
    if (dtype == DSSD_BF16)
        return in_place ? launch_as<DSSD_BF16, true>(P, vector, stream) : launch_as<DSSD_BF16, false>(P, vector, stream);
    return in_place ? launch_as<DSSD_F32, true>(P, vector, stream) : launch_as<DSSD_F32, false>(P, vector, stream);
}

}  // namespace dssd
