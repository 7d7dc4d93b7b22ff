// Penalties for repeated tokens, biases and masks on the rows of logits of a drafted tree: two kernels.
//
// Which entries a penalty or a bias concerns, a few hundred of a row's 10^5, is the same for all rows of a sequence but for the tokens drafted on the
// row's own way.  The first kernel, a CTA per sequence, counts the sequence's own tokens in a hash table in shared memory (in whole numbers, so that the
// order of the atomics changes nothing) and leaves a list of them, by buckets of 16384 entries of the vocabulary.  Where a sequence has more tokens
// than the table holds, the vocabulary is taken in ranges of the table's size, shared out over CTAs, and the table is indexed directly: it cannot overflow either
// way.  A table over the vocabulary would be 4 V bytes per sequence to clear, fill and read.
//
// The second kernel passes the rows by vectors of 16 bytes (in place: only rows with a mask, and there what the mask bans) and then patches the listed entries
// of the part that it just wrote, which are in L2 still.  It waits for the list only then: copying and counting run at the same time.
//
// In place the patch is a kernel of its own, a CTA to a row.
//
// Bound by the copy of the rows, or in place by the entries that change.  Counting by slices of the vocabulary in every CTA of the copy took 141 us for
// B=32 N=24 V=128256 and 406 for B=256 N=5 V=151936 in place; a patch after the copy that counted for itself 90 and 78.
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
constexpr int kBucketLog = 14;
constexpr uint32_t kInPrompt = 1u << 30, kDrafted = 1u << 31, kCount = kInPrompt - 1;

// An entry of the list: token, occurrences with their flags, place of its bias in the request's list + 1 (0: none), the bias
__device__ __forceinline__ uint4 list_entry(int v, uint32_t count, unsigned bias, float value) { return make_uint4((uint32_t)v, count, bias, __float_as_uint(value)); }

// What the penalties of a request do to the listed entries of a row
struct Request {
    float repetition, presence, frequency;
    __device__ __forceinline__ Request(const AdjustParams &P, long long b) : repetition(1.f), presence(0.f), frequency(0.f)
    {
        if (P.repetition) repetition = ld_after(P.repetition + b);
        if (P.presence) presence = ld_after(P.presence + b);
        if (P.frequency) frequency = ld_after(P.frequency + b);
        if (!(repetition > 0.f && repetition < __int_as_float(0x7f800000))) repetition = 1.f;
    }
};
// The entry that x stands for, in the row of `node`, if that counts it and no mask bans it: `old` is what it held in the given logits
template <int DT>
__device__ __forceinline__ void patch(const Request &r, const uint4 &x, typename Vec<DT>::Word old, bool banned, char *out, int node, const short *parent, const int *token)
{
    typedef Vec<DT> E;
    if (banned) return;
    const int v = (int)x.x;
    uint32_t n_out = x.y & kCount;
    if (x.y & kDrafted)
        for (int j = node; j > 0; j = parent[j]) n_out += token[j] == v;
    if (!(n_out | (x.y & kInPrompt) | x.z)) return;  // drafted on other ways only
    float f = E::value(old);
    if (n_out || (x.y & kInPrompt)) f = f > 0.f ? __fdiv_rn(f, r.repetition) : __fmul_rn(f, r.repetition);
    if (n_out) f = __fsub_rn(__fsub_rn(f, __fmul_rn(r.frequency, (float)n_out)), r.presence);
    if (x.z) f = __fadd_rn(f, __uint_as_float(x.w));
    reinterpret_cast<typename E::Word *>(out)[v] = E::bits(f);
}
__device__ __forceinline__ bool banned_by(const uint32_t *mask, int v) { return mask && !((ld_after_u32(mask + (v >> 5)) >> (v & 31)) & 1u); }

// The nodes' parents and tokens in shared memory; whether there is a node `node`.  All threads of the CTA.
__device__ __forceinline__ bool load_way(const AdjustParams &P, long long b, int node, short *parent, int *token)
{
    for (int j = threadIdx.x; j < P.N; j += blockDim.x) {
        int p = j ? j - 1 : 0;
        if (P.parents && j) p = ld_after(P.parents + b * (P.N - 1) + j - 1);
        parent[j] = (short)(p >= j && j ? -1 : max(p, -1));
        if (j) token[j] = ld_after(P.draft_tokens + b * (P.N - 1) + j - 1);
    }
    __syncthreads();
    int up = node;
    while (up > 0) up = parent[up];
    return up == 0;
}

// kInPlace: only what a mask bans is written.  kVector: a row's entries lie alike to 16 bytes in both arrays.
template <int DT, bool kInPlace, bool kVector>
__global__ void __launch_bounds__(kThreads) adjust_copy_kernel(const __grid_constant__ AdjustParams P)
{
    typedef Vec<DT> E;
    typedef typename E::Word Word;
    constexpr uint32_t kAll = (1u << E::kN) - 1u;
    __shared__ short parent[kMaxNodes];
    __shared__ int token[kMaxNodes];
    const int t = threadIdx.x;
    const long long row = blockIdx.x / (unsigned)P.turns;
    const int turn = blockIdx.x % (unsigned)P.turns;
    const long long b = row / P.N;
    const int node = (int)(row - b * P.N);
    // The kernel before this one, which makes the list, let this one in when what came before it had ended: all arrays but the list are as they
    // should be, and the list is waited for below.
    const char *in = static_cast<const char *>(P.logits) + row * P.row_stride * (long long)sizeof(Word);
    char *out = static_cast<char *>(P.out) + row * P.out_stride * (long long)sizeof(Word);
    const uint32_t *mask = mask_of(P, row);
    const uint4 *list = P.list + b * P.list_size;
    const int2 *buckets = P.buckets + b * P.n_buckets;
    const int words = (P.V + 31) / 32;
    // vectors begin on 16-byte boundaries of memory: the first at most kN - 1 entries before the row
    const int mis = kVector ? (int)((reinterpret_cast<uintptr_t>(in) / sizeof(Word)) % E::kN) : 0;
    if (kInPlace) {
        // The list is not for this kernel, and CTAs that wait for it would stand in the way of those with a mask: one waits, so that this
        // kernel ends after the one before it.
        if (blockIdx.x == 0) pdl_wait();
        if (!mask) return;
    }
    if (!load_way(P, b, node, parent, token)) {
        if (!kInPlace) pdl_wait();
        return;
    }
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
    constexpr int kPiece = kThreads * kCopyVecs * E::kN;
    for (int piece = turn; piece < P.pieces; piece += P.turns) {
        const int v0 = piece * kPiece - mis + t * E::kN;
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
        // Out of place the listed entries of this part are looked up while the row is on its way (the list is ready but for the first CTAs).
        const int from = max(piece * kPiece - mis, 0), to = min((piece + 1) * kPiece - mis, P.V);
        int bucket = from >> kBucketLog, at = 0, end = 0;
        uint4 x0 = make_uint4(0, 0, 0, 0);
        if (!kInPlace) {
            if (piece == turn) {
                pdl_wait();
                pdl_trigger();
            }
            if (bucket < P.n_buckets) {
                const unsigned long long span = ld_after(reinterpret_cast<const unsigned long long *>(buckets + bucket));
                at = (int)(uint32_t)span + t, end = (int)(span >> 32);
                if (at < end) x0 = ld_row16(list + at);
            }
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
        if (!kInPlace) {
            __syncthreads();  // (an entry is patched by another thread than the one that copied it)
            const Request r(P, b);
            for (; bucket <= (to - 1) >> kBucketLog; ++bucket) {
                if (bucket > from >> kBucketLog) {
                    const unsigned long long span = ld_after(reinterpret_cast<const unsigned long long *>(buckets + bucket));
                    at = (int)(uint32_t)span + t, end = (int)(span >> 32);
                    if (at < end) x0 = ld_row16(list + at);
                }
                while (at < end) {
                    const int v = (int)x0.x;
                    if (v >= from && v < to) patch<DT>(r, x0, E::load(in + (long long)v * sizeof(Word)), banned_by(mask, v), out, node, parent, token);
                    at += kThreads;
                    if (at < end) x0 = ld_row16(list + at);
                }
            }
        }
    }
}

// In place: a CTA patches the listed entries of a row, four requests in flight to a thread.
template <int DT>
__global__ void __launch_bounds__(kThreads) adjust_patch_kernel(const __grid_constant__ AdjustParams P)
{
    typedef Vec<DT> E;
    typedef typename E::Word Word;
    __shared__ short parent[kMaxNodes];
    __shared__ int token[kMaxNodes];
    const int t = threadIdx.x;
    const long long row = blockIdx.x, b = row / P.N;
    const int node = (int)(row - b * P.N);
    pdl_wait();
    pdl_trigger();
    char *out = static_cast<char *>(P.out) + row * P.out_stride * (long long)sizeof(Word);
    const uint32_t *mask = mask_of(P, row);
    const uint4 *list = P.list + b * P.list_size;
    const unsigned long long *buckets = reinterpret_cast<const unsigned long long *>(P.buckets + b * P.n_buckets);
    // a hash table's buckets follow one another; those of ranges have gaps between them
    const int step = P.gaps ? 1 : P.n_buckets;
    unsigned long long first = ld_after(buckets), last = ld_after(buckets + step - 1);
    const Request r(P, b);
    if (!load_way(P, b, node, parent, token)) return;
    for (int k = 0; k < P.n_buckets; k += step) {
        if (k) first = last = ld_after(buckets + k);
        const int end = (int)(last >> 32);
        for (int e0 = (int)(uint32_t)first + t; e0 < end; e0 += 4 * kThreads) {
            uint4 x[4];
            Word old[4];
            bool banned[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = e0 + u * kThreads < end ? ld_row16(list + e0 + u * kThreads) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                banned[u] = e0 + u * kThreads >= end;
                old[u] = banned[u] ? 0 : E::load(out + (long long)(int)x[u].x * sizeof(Word));
                if (!banned[u]) banned[u] = banned_by(mask, (int)x[u].x);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) patch<DT>(r, x[u], old[u], banned[u], out, node, parent, token);
        }
    }
}

// ---- the list --------------------------------------------------------------------------------

constexpr int kList = 512;  // threads
constexpr int kMaxBuckets = 1024;

// shared memory: key, count and the last bias (its place in the request's list + 1) of every slot
struct Table {
    int *key;
    uint32_t *count;
    unsigned short *bias;
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

__global__ void __launch_bounds__(kList) adjust_list_kernel(const __grid_constant__ AdjustParams P)
{
    extern __shared__ __align__(16) unsigned char raw[];
    __shared__ short parent[kMaxNodes];
    __shared__ int bad, start[kMaxBuckets], below;
    __shared__ unsigned all_flags;
    __shared__ float first_values[kList];
    const int t = threadIdx.x, lane = t & 31;
    const long long b = blockIdx.x / (unsigned)P.shares;
    const int share = blockIdx.x % (unsigned)P.shares;
    Table T;
    T.key = reinterpret_cast<int *>(raw);
    T.count = reinterpret_cast<uint32_t *>(T.key + P.slots);
    T.bias = reinterpret_cast<unsigned short *>(T.count + P.slots);
    T.slots = P.slots;
    if (t == 0) all_flags = 0;
    // In this order, and with nothing in between: the copy reads and writes the logits without a wait of its own, so it may not be let in before all that came
    // before this kernel has ended.
    pdl_wait();
    pdl_trigger();
    // what is needed first is asked for at once, the history as far as it may go
    const int32_t *hist = P.history + b * P.history_stride;
    int tok0[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) tok0[u] = t + u * kList < P.L ? ld_after(hist + t + u * kList) : 0;
    const int bias0 = t < P.K ? ld_after(P.bias_tokens + b * P.K + t) : -1;
    const float value0 = t < P.K ? ld_after(P.bias_values + b * P.K + t) : 0.f;
    int hl = P.L ? ld_after(P.history_len + b) : 0;
    const int pl = P.L ? ld_after(P.prompt_len + b) : 0;
    const float r = P.repetition ? ld_after(P.repetition + b) : 1.f;
    int drafted = t > 0 && t < P.N ? ld_after(P.draft_tokens + b * (P.N - 1) + t - 1) : -1;
    load_tree(P.parents, b, P.N, parent, &bad);  // (with barriers)
    first_values[t] = value0;

    unsigned flags = bad ? DSSD_ADJUST_FLAG_BAD_PARENT : 0u;
    {
        if (!(r > 0.f && r < __int_as_float(0x7f800000))) flags |= DSSD_ADJUST_FLAG_BAD_VALUE;
    }
    if (hl < 0 || hl > P.L) {
        hl = hl < 0 ? 0 : P.L;
        flags |= DSSD_ADJUST_FLAG_BAD_LENGTH;
    }
    if (t >= P.N || parent[t] < 0) drafted = -1;
    else {
        if (t > 0 && (drafted < 0 || drafted >= P.V)) {
            drafted = -1;
            flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
        }
        if (P.mask && P.mask_row && ld_after(P.mask_row + b * P.N + t) >= P.mask_rows) flags |= DSSD_ADJUST_FLAG_BAD_MASK;
    }
    // With fewer tokens than three quarters of the slots the table is a hash table of all of them; else the vocabulary is taken in ranges of
    // the largest table, which are buckets.
    T.direct = (long long)hl + P.N + P.K > (long long)T.slots * 3 / 4;
    uint4 *list = P.list + b * P.list_size;
    int2 *buckets = P.buckets + b * P.n_buckets;
    for (int range = T.direct ? share : 0; range < (T.direct ? P.n_buckets : share == 0 ? 1 : 0); range += P.shares) {
        T.first = range << kBucketLog;
        __syncthreads();
        for (int i = t; i < T.slots; i += kList) T.key[i] = -1, T.count[i] = 0, T.bias[i] = 0;
        for (int i = t; i < P.n_buckets && !T.direct; i += kList) start[i] = 0;
        if (t == 0) below = 0;
        __syncthreads();
        int under = 0;  // tokens before the range: no more than these have entries before its own
        // in eights: the tokens come from L2, and a request at a time would wait for each
        for (int i0 = t; i0 < hl; i0 += 8 * kList) {
            int tok[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) tok[u] = i0 == t ? tok0[u] : i0 + u * kList < hl ? ld_after(hist + i0 + u * kList) : 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * kList;
                if (i >= hl) break;
                if (tok[u] < 0 || tok[u] >= P.V) {
                    flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
                    continue;
                }
                under += tok[u] < T.first;
                const int s = T.find(tok[u]);
                if (s < 0) continue;
                if (i < pl) atomicOr(&T.count[s], kInPrompt);
                else atomicAdd(&T.count[s], 1u);
            }
        }
        if (drafted >= 0) {
            under += drafted < T.first;
            const int s = T.find(drafted);
            if (s >= 0) atomicOr(&T.count[s], kDrafted);
        }
        // of a token's biases the last one holds: whoever stores first does not matter, the largest index stays
        for (int k0 = 0; k0 < P.K; k0 += kList) {
            const int k = k0 + t;
            const int v = k0 == 0 ? bias0 : k < P.K ? ld_after(P.bias_tokens + b * P.K + k) : -1;
            if (v >= P.V) flags |= DSSD_ADJUST_FLAG_BAD_TOKEN;
            const int s = v >= 0 && v < P.V ? T.find(v) : -1;
            under += v >= 0 && v < T.first;
            bool waiting = s >= 0;
            while (__syncthreads_or(waiting)) {
                if (waiting) T.bias[s] = (unsigned short)(k + 1);
                __syncthreads();
                if (waiting) waiting = T.bias[s] < (unsigned short)(k + 1);
            }
        }
        if (T.direct) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) under += __shfl_xor_sync(0xffffffffu, under, o);
            if (lane == 0 && under) atomicAdd(&below, under);
            if (t == 0) start[range] = 0;
        }
        __syncthreads();
        // entries to their buckets: how many, where each begins, then the entries (their order within a bucket changes nothing)
        for (int i = t; i < T.slots; i += kList)
            if (T.key[i] >= 0) atomicAdd(&start[T.key[i] >> kBucketLog], 1);
        __syncthreads();
        if (T.direct) {
            if (t == 0) {
                const int n = start[range];
                start[range] = below;
                buckets[range] = make_int2(below, below + n);
            }
        } else if (t < 32) {
            int base = 0;
            for (int k0 = 0; k0 < P.n_buckets; k0 += 32) {
                const int k = k0 + lane, n = k < P.n_buckets ? start[k] : 0;
                int end = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, end, o);
                    if (lane >= o) end += up;
                }
                if (k < P.n_buckets) {
                    start[k] = base + end - n;
                    buckets[k] = make_int2(base + end - n, base + end);
                }
                base += __shfl_sync(0xffffffffu, end, 31);
            }
        }
        __syncthreads();
        for (int i = t; i < T.slots; i += kList) {
            const int v = T.key[i];
            if (v < 0) continue;
            const unsigned k = T.bias[i];
            list[atomicAdd(&start[v >> kBucketLog], 1)] = list_entry(v, T.count[i], k, !k ? 0.f : k <= kList ? first_values[k - 1] : ld_after(P.bias_values + b * P.K + k - 1));
        }
    }
    if (share == 0 && P.flags) {
        // (every CTA of the sequence sees all tokens, share 0 at least once)
        flags = __reduce_or_sync(0xffffffffu, flags);
        __syncthreads();
        if (lane == 0 && flags) atomicOr(&all_flags, flags);
        __syncthreads();
        if (t == 0) P.flags[b] = all_flags;
    }
}

constexpr int kMaxSlots = 1 << kBucketLog;

cudaError_t make_list(const AdjustParams &P, cudaStream_t stream)
{
    const size_t smem = (size_t)P.slots * 10;
    if (smem > 40 * 1024) {  // (with what is declared in the kernel, beyond the 48 KB that need no leave)
        static PerContext allowed;
        if (!allowed.get([] { return (int)(cudaFuncSetAttribute(adjust_list_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlots * 10) == cudaSuccess); })) {
            const cudaError_t e = cudaGetLastError();
            return e == cudaSuccess ? cudaErrorInvalidConfiguration : e;
        }
    }
    return launch_pdl(adjust_list_kernel, (unsigned)P.B * (unsigned)P.shares, kList, stream, P, smem);
}

template <int DT, bool kInPlace>
cudaError_t copy(const AdjustParams &P, bool vector, cudaStream_t stream)
{
    const unsigned grid = (unsigned)((long long)P.B * P.N * P.turns);
    return vector ? launch_pdl(adjust_copy_kernel<DT, kInPlace, true>, grid, kThreads, stream, P)
                  : launch_pdl(adjust_copy_kernel<DT, kInPlace, false>, grid, kThreads, stream, P);
}

// a slot and a third for each token that there may be
int slots_of(long long tokens)
{
    int n = 512;
    while (n < kMaxSlots && (long long)n * 3 / 4 < tokens) n *= 2;
    return n;
}
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
int buckets_of(int V) { return (V + (1 << kBucketLog) - 1) >> kBucketLog; }

}  // namespace

static_assert(DSSD_ADJUST_MAX_V <= kMaxBuckets << kBucketLog, "a counter per bucket");

int adjust_copy_entries(int dtype) { return kThreads * kCopyVecs * (dtype == DSSD_BF16 ? 8 : 4); }

size_t adjust_workspace(int B, int N, int V, int L, int K)
{
    return round256((size_t)B * ((size_t)L + N + K) * sizeof(uint4)) + round256((size_t)B * buckets_of(V) * sizeof(int2));
}

cudaError_t adjust_launch(AdjustParams &P, int dtype, void *workspace, cudaStream_t stream)
{
    const int esz = dtype == DSSD_BF16 ? 2 : 4;
    const bool in_place = P.out == P.logits, bf = dtype == DSSD_BF16;
    const long long tokens = (long long)P.L + P.N + P.K;
    P.list = static_cast<uint4 *>(workspace);
    P.list_size = tokens;
    P.buckets = reinterpret_cast<int2 *>(static_cast<char *>(workspace) + round256((size_t)P.B * (size_t)tokens * sizeof(uint4)));
    P.n_buckets = buckets_of(P.V);
    P.slots = slots_of(tokens);
    // tables that may have to be taken in ranges: a few CTAs for these
    P.shares = 1;
    if ((long long)P.slots * 3 / 4 < tokens)
        while (P.shares < P.n_buckets && P.shares < 16 && (long long)P.B * P.shares < 2 * 148) P.shares *= 2;
    cudaError_t e = make_list(P, stream);
    if (e != cudaSuccess) return e;
    // a vector store needs the two rows at the same place of a 16-byte line, for every row
    const uintptr_t a = reinterpret_cast<uintptr_t>(P.logits), c = reinterpret_cast<uintptr_t>(P.out);
    const bool vector = (a - c) % 16 == 0 && ((P.row_stride - P.out_stride) * esz) % 16 == 0;
    const int per = adjust_copy_entries(dtype);
    const int most = P.V + (vector && (a % 16 || (P.row_stride * esz) % 16) ? 16 / esz - 1 : 0);  // with the entries before a row's start
    P.pieces = (most + per - 1) / per;
    P.turns = P.pieces;
    if (in_place) {
        if (P.mask) {
            // most rows have no mask as a rule, and a CTA that finds none has nothing to do: no more of them than fill the GPU a few times over
            while (P.turns > 1 && (long long)P.B * P.N * P.turns > 148 * 64) P.turns = (P.turns + 1) / 2;
            e = bf ? copy<DSSD_BF16, true>(P, vector, stream) : copy<DSSD_F32, true>(P, vector, stream);
            if (e != cudaSuccess) return e;
        }
        P.gaps = (long long)P.slots * 3 / 4 < tokens;
        const unsigned rows = (unsigned)((long long)P.B * P.N);
        return bf ? launch_pdl(adjust_patch_kernel<DSSD_BF16>, rows, kThreads, stream, P) : launch_pdl(adjust_patch_kernel<DSSD_F32>, rows, kThreads, stream, P);
    }
    return bf ? copy<DSSD_BF16, false>(P, vector, stream) : copy<DSSD_F32, false>(P, vector, stream);
}

}  // namespace dssd
