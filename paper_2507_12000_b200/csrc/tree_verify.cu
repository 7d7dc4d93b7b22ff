// The verdict on a drafted tree: one thread-block cluster per sequence walks from the root to the last accepted node.
//
// After r rejections at a node the residual distribution is max(0, p - a q) / m with two numbers a and m:
//   max(0, max(0, p - a q) / m - c q) = max(0, p - (a + m c) q) / m,
// (inside the outer maximum nothing changes where p - a q < 0, since q >= 0), so a rejection is one sum over the two rows
// as they lie in memory and no row is ever written.  Drawing siblings without replacement only scales q by c between them, one divided by the sum of what
// is left of q: a rejected token x has p(x) - a q(x) <= 0 from then on, so that its removal from q is not seen.  That sum is taken over the tokens that are
// left, in the pass that reads q anyway, whenever another sibling follows: one minus the rejected ones has no digits left after a sibling that the draft was sure of.
//
// Every CTA of the cluster holds a slice of the vocabulary and the same scalars; sums meet through
// distributed shared memory and are added in rank order by everybody, so that all CTAs take the same way.  A node costs one pass over its logits
// and one exchange, a rejection one pass over both rows and one exchange; the last of these passes leaves the sums of chunks that the draw
// picks from.  A warp takes a chunk of 512 entries at a time.
//
// The tests and the draw are decisions: what is wanted is the answer that exact arithmetic gives.  A pass in float32 (3 to 5 instructions an entry)
// gives p, its sums and m with known bounds on their errors, and a comparison further apart than those is certain.
// One that is not takes the node again in float64 (25 to 35 instructions an entry: 2^x by a table of 16 entries, each in banks of its own, and a polynomial).
// That is mostly a draw whose uniform falls too near a step of the distribution, sum over v of min(p_v, 4 sum_error) of all draws: for Gaussian logits over
// a Zipf bias 2 % at V=32000 T=0.8, 6 to 10 % at V=50272 T=1, 17 to 29 % at V=151936 T=1.2, the larger after a rejection.  With everything in float64 the verdicts of B=128 N=12 V=151936 took 232 us.
//
// Bound by the latency of a chain of dependent reductions for few sequences, by the visited rows for many.
#include <math.h>

#include "launch.h"
#include "quads.cuh"
#include "tree.cuh"
#include "tree_ops.h"

namespace dssd {

namespace {

constexpr int kMaxCluster = 16;
constexpr int kMaxChunks = 1024;  // of a CTA's slice
constexpr int kBlock = 512;       // entries that a warp loads at once

struct VerifySmem {
    double table[16];
    double part[2][kMaxCluster], part2[2][kMaxCluster];  // what the CTAs of the cluster exchange, in turns
    double warp[2][kWarps], warp2[2][kWarps];
    double chunk[kMaxChunks];
    int token[kMaxNodes];
    short parent[kMaxNodes], child[kMaxNodes], sibling[kMaxNodes];
    int bad;
    unsigned long long again[1];  // the draw was not certain
};

// Bounds of the errors of a float32 pass, relative to the whole distribution, of a sum of p over any entries.  In numerator and row's sum alike, per term: ex2,
// 2^-22; the rounding of x = l c1 - r, ln(2) 2^-24 |x|, where sum p |x| is at most the logarithm of the number of entries; the rounding of c1, half of that at the
// most between entries; six levels of float32 additions of 2^-24.
__host__ inline double sum_error(int V) { return 2.0 * (2.4e-7 + 4.2e-8 * (1.5 * log2((double)V + 1.0)) + 6.0 * 6.0e-8); }
// Of one p far down, relative, more for each power of two: the rounding of c1, ln(2) 2^-24 |log2 p|.
constexpr double kBitError = 4.2e-8;
constexpr double kProductError = 2.5e-7;  // of a q in the residual, for each unit of a
constexpr double kRestError = 4e-7;       // of what is left of q, relative: six levels of float32 additions

__device__ __forceinline__ double as_double(int hi, int lo) { return __hiloint2double(hi, lo); }

// A float32 as float64 by its bits, 2^896 times too small (a conversion instruction has a quarter of the throughput of a product): exact for zeros and
// subnormal numbers too.  Infinities and NaN become numbers of that size times 2^128 and more.
__device__ __forceinline__ double shrunk(uint32_t w)
{
    return as_double((int)((w & 0x7fffffffu) >> 3 | (w & 0x80000000u)), (int)(w << 29));
}
constexpr double kGrow = 0x1p896, kGrowA = 0x1p803, kGrowS = 0x1p93;  // (of which the product is the first)

// p - a q in units of the row's sum: a and s come with their part of the factor.  a q comes first, so that a large a meets what is small; a is below 2^156
// and the sum below 2^931, so that neither part overflows.
__device__ __forceinline__ double residual(double p, uint32_t q, double a, double s) { return __fma_rn(-s, shrunk(q) * a, p); }

// 2^x = 2^(k / 16) 2^r, |r| <= 1/32; the polynomial is the exponential series to the fourth power (relative error below 5e-11).
// 0 below 2^-1000, infinity above 2^1000.
// x = (l - top) c for a logit l given by its bits, top and c by shrunk() and its inverse: the difference comes first, since a product beyond 2^53 would leave
// nothing of x.  Minus infinity is 0 whatever top is.
__device__ __forceinline__ double weight(uint32_t l, double top, double c, const double *table)
{
    const double x = (shrunk(l) - top) * c;
    const uint32_t hi = (uint32_t)__double2hiint(x);
    const double big = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number, held in the low bits
    const double t = __fma_rn(x, 16.0, big);
    const int k = __double2loint(t);
    const double r = __fma_rn(t - big, -1.0 / 16.0, x);
    double p = __fma_rn(r, 9.6181291076284772e-3, 5.5504108664821580e-2);  // ln(2)^n / n!
    p = __fma_rn(p, r, 2.4022650695910071e-1);
    p = __fma_rn(p, r, 6.9314718055994531e-1);
    p = __fma_rn(p, r, 1.0);
    const double y = p * table[k & 15];
    const bool far = (hi & 0x7fffffffu) > 0x408f4000u || l == 0xff800000u;  // |x| > 1000
    const int yh = far ? ((int)hi < 0 ? 0 : 0x7ff00000) : __double2hiint(y) + ((k >> 4) << 20);
    return as_double(yh, far ? 0 : __double2loint(y));
}

// x of all threads, and y where it is wanted: warps in order and CTAs in rank order; the same in every thread
template <bool kBoth>
__device__ __forceinline__ double cluster_sum(VerifySmem &S, double x, double &y, unsigned ctas, int &turn)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    x = warp_sum(x);
    if (kBoth) y = warp_sum(y);
    if (lane == 0) {
        S.warp[turn][warp] = x;
        if (kBoth) S.warp2[turn][warp] = y;
    }
    __syncthreads();
    double s = 0.0, s2 = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        s += S.warp[turn][w];
        if (kBoth) s2 += S.warp2[turn][w];
    }
    if (ctas > 1) {
        if (threadIdx.x < ctas) {
            cluster_store(&S.part[turn][cluster_rank()], threadIdx.x, s);
            if (kBoth) cluster_store(&S.part2[turn][cluster_rank()], threadIdx.x, s2);
        }
        cluster_arrive();
        cluster_wait();
        s = s2 = 0.0;
        for (unsigned c = 0; c < ctas; ++c) {
            s += S.part[turn][c];
            if (kBoth) s2 += S.part2[turn][c];
        }
    }
    if (kBoth) y = s2;
    turn ^= 1;  // (a thread that is here again has seen every other thread's arrival at the exchange between)
    return s;
}

template <int DT>
struct Logits;
template <>
struct Logits<DSSD_BF16> {
    typedef Quads16 Q;
    static constexpr uint32_t kFill = 0xff80u;
    __device__ static uint32_t bits(const uint2 &v, int i) { return i == 0 ? v.x << 16 : i == 1 ? v.x & 0xffff0000u : i == 2 ? v.y << 16 : v.y & 0xffff0000u; }
    __device__ static uint32_t one(const char *row, int v) { return ld_row_u16(row + 2ll * v) << 16; }
    __device__ static float max16(const uint2 (&w)[4])
    {
        uint32_t m = max_bf16x2(max_bf16x2(w[0].x, w[0].y), max_bf16x2(w[1].x, w[1].y));
        m = max_bf16x2(m, max_bf16x2(max_bf16x2(w[2].x, w[2].y), max_bf16x2(w[3].x, w[3].y)));
        return fmaxf(bf16_lo(m), bf16_hi(m));
    }
};
template <>
struct Logits<DSSD_F32> {
    typedef Quads32 Q;
    static constexpr uint32_t kFill = 0xff800000u;
    __device__ static uint32_t bits(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ static uint32_t one(const char *row, int v) { return ld_row_u32(row + 4ll * v); }
    __device__ static float max16(const uint4 (&w)[4])
    {
        float m = DSSD_NEG_INF;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[u].x), __uint_as_float(w[u].y)), fmaxf(__uint_as_float(w[u].z), __uint_as_float(w[u].w))));
        return m;
    }
};
__device__ __forceinline__ bool is_nan(uint32_t w) { return (w & 0x7fffffffu) > 0x7f800000u; }

// A CTA's slice of a row, by chunks of whole blocks
struct Slice {
    int V, v0, v1, chunk, chunks;
};

// A warp's blocks: those of its chunks, one after the other
struct Walk {
    const Slice &P;
    int k, at;
    __device__ __forceinline__ Walk(const Slice &p, int warp) : P(p), k(warp), at(p.v0 + warp * p.chunk) {}
    __device__ __forceinline__ bool more() const { return k < P.chunks; }
    __device__ __forceinline__ bool next()  // whether the chunk ends with the block that is left
    {
        at += kBlock;
        if (at < min(P.v1, P.v0 + (k + 1) * P.chunk)) return false;
        k += kWarps;
        at = P.v0 + k * P.chunk;
        return true;
    }
};

// whole 16-byte pieces of `bytes` at p
__device__ __forceinline__ void prefetch_l2(const void *p, int bytes)
{
    const uintptr_t from = (reinterpret_cast<uintptr_t>(p) + 15) & ~(uintptr_t)15, to = (reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes) & ~(uintptr_t)15;
    if (to > from) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((uint32_t)(to - from)) : "memory");
}

__device__ __forceinline__ int exponent(double x) { return ((__double2hiint(x) >> 20) & 0x7ff) - 1023; }

// kShift: rows may begin off the boundaries of four entries.  kWithout: siblings were drawn without replacement.
template <int DT, bool kShift, bool kWithout>
__global__ void __launch_bounds__(kThreads, 2) tree_verify_kernel(const __grid_constant__ TreeVerifyParams P)
{
    typedef Logits<DT> E;
    __shared__ VerifySmem S;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    unsigned ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const unsigned me = ctas > 1 ? cluster_rank() : 0;
    const long long b = blockIdx.x / ctas;
    const int v0 = (int)min((long long)P.V, (long long)me * P.slice), v1 = (int)min((long long)P.V, (long long)v0 + P.slice);
    const int chunks = (v1 - v0 + P.chunk - 1) / P.chunk;
    const Slice slice = {P.V, v0, v1, P.chunk, chunks};
    if (t < 16) S.table[t] = exp2(t / 16.0);
    pdl_wait();
    pdl_trigger();
    load_tree(P.parents, b, P.N, S.parent, &S.bad);
    if (t < P.N) {
        if (t > 0) S.token[t] = ld_after(P.draft_tokens + b * (P.N - 1) + t - 1);
        int child = 0, sibling = 0;  // 0: none
        for (int j = P.N - 1; j > t; --j) {
            if (S.parent[j] == t) child = j;
            if (t > 0 && S.parent[j] == S.parent[t]) sibling = j;
        }
        S.child[t] = (short)child;
        S.sibling[t] = (short)sibling;
    }
    if (ctas > 1) {  // nobody writes into a CTA's shared memory before it runs
        cluster_arrive();
        cluster_wait();
    }
    __syncthreads();
    const double u_draw = (double)ld_after(P.uniforms_rs + b);
    int turn = 0;
    unsigned eflags = S.bad ? DSSD_EDGE_FLAG_BAD_PARENT : 0u, rflags = 0;

    int node = 0, length = 0;
    double a = 0.0, m = 1.0, c = 1.0, top = 0.0, sum = 1.0, inv = 1.0;
    double a_error = 0.0, m_error = 0.0, c_error = 0.0;
    int refused = 0, mine = -1;  // siblings so far; the one of this lane's number
    bool alive = true, fine = false;
    const float c1 = (float)P.c1;
    const double c1_grown = P.c1 * kGrow;
    const char *row;
    const float *qrow;
    // what a test needs, asked for before the pass that comes before it
    struct Asked {
        uint32_t l;
        float q, u;
        bool ok;
    };
    auto ask = [&](int j) {
        Asked r = {0u, 0.f, 1.f, false};
        const int x = S.token[j];
        if (j > 0 && x >= 0 && x < P.V) {
            r.ok = true;
            r.l = E::one(row, x);
            r.q = ld_after(qrow + x);
            r.u = ld_after(P.uniforms + b * (P.N - 1) + j - 1);
        }
        return r;
    };
    // the sum of a chunk, where the draw will want it
    auto close = [&](bool keep, bool ends, int k, double &part, double &total) {
        if (!keep || !ends) return;
        part = warp_sum(part);
        if (lane == 0) S.chunk[k] = part, total += part;
        part = 0.0;
    };
    if (me == 0 && t == 0) P.path[b * P.N] = 0;
    bool relative = false, plain = false;  // take the row relative to its maximum (in top); draw from p after all
    while (true) {
        row = static_cast<const char *>(P.logits) + (b * P.N + node) * P.row_stride * (long long)E::Q::kBytes;
        qrow = P.draft_q + (b * P.N + node) * (long long)P.V;
        int j = plain ? 0 : S.child[node];
        const bool has_child = S.child[node] > 0;
        bool kept = j == 0;  // the pass leaves the chunks' sums
        bool certain = true;
        Asked next = ask(j);
        if (!relative) top = 0.0;
        if (j > 0 && t == 0 && v1 > v0) {
            // What comes next is asked of memory now: this CTA's part of q, which a rejection reads, and of the first child's row.
            prefetch_l2(qrow + v0, (v1 - v0) * 4);
            prefetch_l2(static_cast<const char *>(P.logits) + ((b * P.N + j) * P.row_stride + v0) * (long long)E::Q::kBytes, (v1 - v0) * E::Q::kBytes);
        }
        {
            // the sum of 2^((l - top) c1); NaN where the row holds one, or +inf
            double part = 0.0, total = 0.0;
            Walk w(slice, warp);
            if (!fine) {
                WarpQuads<typename E::Q, 4, kShift> N;
                if (w.more()) N.load(row, P.V, w.at, E::kFill);
                while (w.more()) {
                    typename E::Q::Raw q[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) q[u] = N.at(u);
                    const int k = w.k;
                    const bool ends = w.next();
                    if (w.more()) N.load(row, P.V, w.at, E::kFill);  // on its way while this block is summed
                    // relative to a whole power of two near the lane's largest term, so that its sum's scaling is exact
                    float r = ceilf(E::max16(q) * c1);
                    r = r > -1000.f ? r : -1000.f;
                    f32x2 acc[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    const f32x2 c2 = pack2(c1, c1), r2 = pack2(-r, -r);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float x, y;
                            unpack2(fma2(pack2(__uint_as_float(E::bits(q[u], 2 * i)), __uint_as_float(E::bits(q[u], 2 * i + 1))), c2, r2), x, y);
                            acc[i] = add2(acc[i], pack2(ex2(x), ex2(y)));
                        }
                    float x, y;
                    unpack2(add2(acc[0], acc[1]), x, y);
                    // Beyond 2^1000 the sum is out of range, and has to be seen to be: there the rounding of l c1 may leave nothing of a lane's terms.
                    const float lane_sum = r > 1000.f ? x + y + __int_as_float(0x7f800000) : x + y;
                    part += (double)lane_sum * as_double((1023 + (int)fminf(r, 1000.f)) << 20, 0);
                    close(kept, ends, k, part, total);
                }
            } else {
                while (w.more()) {
#pragma unroll 1
                    for (int half = 0; half < kBlock; half += kBlock / 2) {
                        WarpQuads<typename E::Q, 2, kShift> L;
                        L.load(row, P.V, w.at + half, E::kFill);
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const typename E::Q::Raw q = L.at(u);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t x = E::bits(q, i);
                                part += weight(x, top, c1_grown, S.table);
                                if (is_nan(x)) part = __longlong_as_double(0x7ff8000000000000ll);
                            }
                        }
                    }
                    const int k = w.k;
                    close(kept, w.next(), k, part, total);
                }
            }
            double none = 0.0;
            sum = cluster_sum<false>(S, kept ? total : part, none, ctas, turn);
        }
        alive = sum == sum;
        if (alive && !(sum > 1e-280 && sum < 1e280)) {
            if (!fine) {
                fine = true;
                continue;
            }
            // out of range: relative to the row's maximum, which each CTA finds for itself
            alive = false;
            if (!relative) {
                float mx = DSSD_NEG_INF;
                for (int v = t; v < P.V; v += kThreads) mx = fmaxf(mx, __uint_as_float(E::one(row, v)));
                mx = warp_max(mx);
                __syncthreads();
                if (lane == 0) S.warp[0][warp] = (double)mx;
                __syncthreads();
                double most = S.warp[0][0];
                for (int w = 1; w < kWarps; ++w) most = fmax(most, S.warp[0][w]);
                __syncthreads();
                if (most > -1e300 && most < 1e300) {
                    top = shrunk(__float_as_uint((float)most));
                    relative = true;
                    continue;
                }
            }
        }
        if (!alive) eflags |= DSSD_EDGE_FLAG_NONFINITE;
        inv = 1.0 / sum;
        a = 0.0, m = 1.0, c = 1.0;
        a_error = m_error = c_error = 0.0;
        refused = 0, mine = -1;
        const double slack = fine ? 0.0 : P.sum_error, C = (fine ? P.c1 : (double)c1) * kGrow;
        bool taken = false;
        auto more_error = [&] { return kWithout ? c * (m_error + m * c_error) : m_error; };  // of c m
        while (j > 0) {
            if (!next.ok) eflags |= DSSD_EDGE_FLAG_BAD_TOKEN;
            if (next.ok && alive) {
                const double qx = (double)next.q, u = (double)next.u;
                const double px = weight(next.l, top, C, S.table) * inv;
                const double left = fmax(px - a * qx, 0.0), want = u * (c * m) * qx;
                taken = u < 1.0 && (qx <= 0.0 ? left > 0.0 : want < left);
                // (a NaN q rejects, whatever the errors)
                if (!fine && u < 1.0 && qx > 0.0 && !(fabs(px - a * qx - want) > px * (slack + kBitError * (double)(1 - exponent(px))) + qx * (a_error + u * more_error()))) {
                    certain = false;
                    break;
                }
                if (taken) break;
            }
            // rejected: what is left of p
            a += c * m;
            a_error += more_error();
            if (kWithout && next.ok && refused++ == lane) mine = S.token[j];
            if (!fine && alive && !(a < 1e6)) {
                certain = false;
                break;
            }
            j = S.sibling[j];
            next = ask(j);
            kept = j == 0;
            m = 0.0;
            if (!alive) continue;
            // the sum of max(0, p - a q): in float64 in units of the row's sum, in float32 in units of the power of two below it; and of q over the tokens
            // that were not refused
            double part = 0.0, total = 0.0, rest = 0.0;
            const bool follows = kWithout && j > 0;
            // which of this lane's entries, in blocks of 128 from `from` on, are refused tokens: bit 4 u + i for entry i of its quad of block u
            auto refused_in = [&](int from, int count) {
                uint32_t bits = 0;
                auto add = [&](int x) {
                    const int at = x - from;
                    if (at >= 0 && at < count && (at >> 2 & 31) == lane) bits |= 1u << (at >> 7) * 4 + (at & 3);
                };
                if (refused > 32)
                    for (int k = S.child[node]; k != j; k = S.sibling[k]) add(S.token[k]);
                else
                    for (unsigned some = __ballot_sync(0xffffffffu, mine >= from && mine < from + count); some; some &= some - 1)
                        add(__shfl_sync(0xffffffffu, mine, __ffs(some) - 1));
                return bits;
            };
            Walk w(slice, warp);
            if (!fine) {
                const int e = exponent(sum);
                const float aF = (float)(a * sum * as_double((1023 - e) << 20, 0));
                const f32x2 c2 = pack2(c1, c1), r2 = pack2(-(float)e, -(float)e), a2 = pack2(-aF, -aF);
                WarpQuads<typename E::Q, 4, kShift> N;
                WarpQuads<Quads32, 4, kShift> NQ;
                if (w.more()) {
                    N.load(row, P.V, w.at, E::kFill);
                    NQ.load(reinterpret_cast<const char *>(qrow), P.V, w.at, 0u);
                }
                while (w.more()) {
                    typename E::Q::Raw l[4];
                    uint4 q[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) l[u] = N.at(u), q[u] = NQ.at(u);
                    if (follows) {
                        const uint32_t gone = refused_in(w.at, kBlock);
                        f32x2 s2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                        if (__any_sync(0xffffffffu, gone)) {
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const uint32_t g = gone >> 4 * u;
                                s2[0] = add2(s2[0], pack2(g & 1u ? 0.f : __uint_as_float(q[u].x), g & 2u ? 0.f : __uint_as_float(q[u].y)));
                                s2[1] = add2(s2[1], pack2(g & 4u ? 0.f : __uint_as_float(q[u].z), g & 8u ? 0.f : __uint_as_float(q[u].w)));
                            }
                        } else {
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                s2[0] = add2(s2[0], pack2(__uint_as_float(q[u].x), __uint_as_float(q[u].y)));
                                s2[1] = add2(s2[1], pack2(__uint_as_float(q[u].z), __uint_as_float(q[u].w)));
                            }
                        }
                        float x, y;
                        unpack2(add2(s2[0], s2[1]), x, y);
                        rest += (double)(x + y);
                    }
                    const int k = w.k;
                    const bool ends = w.next();
                    if (w.more()) {
                        N.load(row, P.V, w.at, E::kFill);
                        NQ.load(reinterpret_cast<const char *>(qrow), P.V, w.at, 0u);
                    }
                    f32x2 acc[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    float x, y;
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            unpack2(fma2(pack2(__uint_as_float(E::bits(l[u], 2 * i)), __uint_as_float(E::bits(l[u], 2 * i + 1))), c2, r2), x, y);
                            const f32x2 q2 = i == 0 ? pack2(__uint_as_float(q[u].x), __uint_as_float(q[u].y)) : pack2(__uint_as_float(q[u].z), __uint_as_float(q[u].w));
                            unpack2(fma2(a2, q2, pack2(ex2(x), ex2(y))), x, y);
                            acc[i] = add2(acc[i], pack2(fmaxf(x, 0.f), fmaxf(y, 0.f)));
                        }
                    unpack2(add2(acc[0], acc[1]), x, y);
                    part += (double)(x + y);
                    close(kept, ends, k, part, total);
                }
                m = (kept ? total : part) * as_double((1023 + e) << 20, 0);
            } else {
                const double aG = a * kGrowA, sG = sum * kGrowS;
                while (w.more()) {
#pragma unroll 1
                    for (int half = 0; half < kBlock; half += kBlock / 2) {
                        WarpQuads<typename E::Q, 2, kShift> L;
                        WarpQuads<Quads32, 2, kShift> R;
                        L.load(row, P.V, w.at + half, E::kFill);
                        R.load(reinterpret_cast<const char *>(qrow), P.V, w.at + half, 0u);
                        const uint32_t gone = follows ? refused_in(w.at + half, kBlock / 2) : 0u;
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const typename E::Q::Raw l = L.at(u);
                            const uint4 q = R.at(u);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const double p = weight(E::bits(l, i), top, c1_grown, S.table);
                                const uint32_t qb = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
                                const double d = residual(p, qb, aG, sG);
                                part += d > 0.0 ? d : 0.0;
                                // (positive and finite)
                                if (follows && qb - 1u < 0x7f7fffffu && !(gone >> (4 * u + i) & 1u)) rest += shrunk(qb);
                            }
                        }
                    }
                    const int k = w.k;
                    close(kept, w.next(), k, part, total);
                }
                m = kept ? total : part;
                rest *= kGrow;
            }
            m = cluster_sum<kWithout>(S, m, rest, ctas, turn) * inv;
            if (follows) {
                c = rest > 0.0 ? 1.0 / rest : 0.0;  // (nothing left of q: nothing more is subtracted)
                c_error = fine ? 0.0 : kRestError;  // (relative)
                if (!fine && !(rest > 1e-20 && rest < 1e20)) {
                    certain = false;
                    break;
                }
            }
            m_error = slack + a_error + (1.0 + a) * (fine ? 0.0 : kProductError);
            if (!fine && !(m > 8.0 * m_error)) {  // what is left is no more than the errors
                certain = false;
                break;
            }
        }
        if (!certain) {
            fine = true;
            continue;
        }
        if (taken) {
            node = j;
            ++length;
            fine = relative = false;
            if (me == 0 && t == 0) P.path[b * P.N + length] = j;
            continue;
        }

        // the draw, from p or from max(0, p - a q)
        rflags = has_child ? (plain ? DSSD_RS_FLAG_FALLBACK : 0u) : DSSD_RS_FLAG_BONUS;
        if (a > 0.0 && !(m > 0.0)) {
            if (alive) {  // the row's own sums once more
                plain = true;
                continue;
            }
            rflags |= DSSD_RS_FLAG_FALLBACK;
        }
        // What the exchange after the last pass left: the CTAs' sums, in units of the row's.  The chunks' sums of a float32 pass over p - a q are
        // in units of a power of two below that.
        const double unit = !fine && a > 0.0 ? as_double((1023 + exponent(sum)) << 20, 0) : 1.0;
        const double aG = a * kGrowA, sG = sum * kGrowS, total = a > 0.0 ? m * sum : sum, target = u_draw * total;
        const double *const parts = S.part[turn ^ 1];
        int owner = -1, last = 0;  // last: the last CTA with mass
        double run = 0.0, before = 0.0;
        for (unsigned k = 0; k < ctas; ++k) {
            const double w = ctas > 1 ? parts[k] : total;
            if (w > 0.0) last = (int)k;
            if (owner < 0 && run + w > target) owner = (int)k, before = run;
            run += w;
        }
        __syncthreads();  // (the chunks' sums)
        const bool invalid = !alive || !(total > 0.0);
        const bool short_of = owner < 0;  // rounding left none: the last entry with mass
        if (short_of) owner = last;
        if (invalid) rflags |= DSSD_RS_FLAG_INVALID;
        if (invalid) owner = 0;
        // the uniform's place and the steps of the distribution have to be further apart than this
        const double margin = fine ? -1.0 : 2.0 * sum * (a > 0.0 ? m_error : P.sum_error);
        if (me == (unsigned)owner && warp == 0) {
            int token = -1;
            bool sure = true;
            if (!invalid) {
                // the chunk, 32 at a time
                double r = before;
                int pick = -1, lastk = 0;
                for (int k0 = 0; k0 < chunks && pick < 0; k0 += 32) {
                    const int k = k0 + lane;
                    const double w = k < chunks ? S.chunk[k] * unit : 0.0;
                    double cum = w;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double up = __shfl_up_sync(0xffffffffu, cum, o);
                        if (lane >= o) cum += up;
                    }
                    const unsigned some = __ballot_sync(0xffffffffu, w > 0.0);
                    if (some) lastk = k0 + 31 - __clz(some);
                    const unsigned over = __ballot_sync(0xffffffffu, !short_of && w > 0.0 && r + cum > target);
                    if (over) {
                        const int l = __ffs(over) - 1;
                        pick = k0 + l;
                        const double upto = __shfl_sync(0xffffffffu, cum, l), its = __shfl_sync(0xffffffffu, w, l);
                        r += upto - its;
                    } else
                        r += __shfl_sync(0xffffffffu, cum, 31);
                }
                const bool hit = pick >= 0;
                const int k = hit ? pick : lastk;
                int last_v = -1;
                sure = fine;
                const int e = min(v1, v0 + (k + 1) * P.chunk);
                for (int base = v0 + k * P.chunk; base < e && token < 0; base += kBlock) {
                    // sixteen neighbouring entries to a lane, all loads together
                    const int v = base + lane * 16;
                    uint32_t l16[16], q16[16];
                    double w[16], mine = 0.0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) l16[i] = v + i < e ? E::one(row, v + i) : 0xff800000u;
#pragma unroll
                    for (int i = 0; i < 16; ++i) q16[i] = a > 0.0 && v + i < e ? ld_row_u32(qrow + v + i) : 0u;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const double p = weight(l16[i], top, C, S.table);
                        const double d = a > 0.0 ? residual(p, q16[i], aG, sG) : p;
                        w[i] = d > 0.0 ? d : 0.0;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) mine += w[i];
                    double cum = mine;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double up = __shfl_up_sync(0xffffffffu, cum, o);
                        if (lane >= o) cum += up;
                    }
                    const unsigned some = __ballot_sync(0xffffffffu, mine > 0.0);
                    const unsigned over = __ballot_sync(0xffffffffu, hit && mine > 0.0 && r + cum > target);
                    // the lane that the target is in, or the last with mass
                    const int l = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : -1;
                    if (l >= 0) {
                        double run2 = r + cum - mine;
                        int found = -1, lastw = -1;
                        bool fits = false;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (w[i] > 0.0) lastw = v + i;
                            if (found < 0 && w[i] > 0.0 && run2 + w[i] > target) {
                                found = v + i;
                                fits = target - run2 > margin && run2 + w[i] - target > margin;
                            }
                            run2 += w[i];
                        }
                        const int f = __shfl_sync(0xffffffffu, found, l), lw = __shfl_sync(0xffffffffu, lastw, l);
                        const bool ft = __shfl_sync(0xffffffffu, (int)fits, l) != 0;
                        last_v = lw;
                        if (over) {
                            token = f >= 0 ? f : lw;  // (the lane's sum and its entries' differ by their rounding)
                            sure = sure || (f >= 0 && ft);
                        }
                    }
                    r += __shfl_sync(0xffffffffu, cum, 31);
                }
                if (token < 0) token = last_v;
            }
            if (lane == 0 && sure) P.token[b] = token;
            if (ctas > 1) {
                if (lane < (int)ctas) cluster_store(&S.again[0], lane, (unsigned long long)!sure);
            } else if (lane == 0)
                S.again[0] = !sure;
        }
        // (a CTA's shared memory outlives the others' stores into it)
        if (ctas > 1) {
            cluster_arrive();
            cluster_wait();
        } else
            __syncthreads();
        if (!S.again[0]) break;
        fine = true;
        __syncthreads();
    }
    if (me == 0) {
        for (int k = length + 1 + t; k < P.N; k += kThreads) P.path[b * P.N + k] = -1;
        if (t == 0) {
            P.accept_len[b] = length;
            if (P.edge_flags) P.edge_flags[b] = eflags;
            if (P.rs_flags) P.rs_flags[b] = rflags;
        }
    }
}

template <int DT, bool kShift, bool kWithout>
cudaError_t launch_as(const TreeVerifyParams &P, unsigned ctas, cudaStream_t stream)
{
    if (ctas > 8) {
        static PerContext allowed;
        if (!allowed.get([] { return (int)allow_cluster(tree_verify_kernel<DT, kShift, kWithout>, 16, kThreads); })) {
            cudaGetLastError();
            return cudaErrorNotSupported;
        }
    }
    return launch_pdl(tree_verify_kernel<DT, kShift, kWithout>, (unsigned)P.B * ctas, kThreads, stream, P, 0, ctas);
}

template <int DT, bool kShift>
cudaError_t launch_either(const TreeVerifyParams &P, unsigned ctas, cudaStream_t stream)
{
    return P.replacement ? launch_as<DT, kShift, false>(P, ctas, stream) : launch_as<DT, kShift, true>(P, ctas, stream);
}

}  // namespace

cudaError_t tree_verify_launch(TreeVerifyParams &P, int dtype, cudaStream_t stream)
{
    P.sum_error = sum_error(P.V);
    const int blocks = (P.V + kBlock - 1) / kBlock;
    // A cluster of more CTAs makes a sequence's passes shorter, and lets fewer sequences walk at a time.  Two CTAs of this kernel fit an SM: as many
    // to a sequence as leave room for all (us of 1 2 4 8 16 CTAs: B=8 V=32000 24.4 22.4 19.1 17.1 17.8; B=64 V=128256 150 94 64 69 102; B=160
    // V=32000 113 77 70 95 200), but no CTA with more than 72 KB of a row (B=128 V=151936: 512 286 198 168 227; float32, B=86 V=86704: 132 with four, 109 with eight) and no warp without a block
    // (B=160 V=8192: 48 40 51 83 176).  Sixteen where there are few sequences (B=2 V=50272: 33 27 21 17.5 16.6; B=16 V=128256: 94 56 37 28 31).
    const int esz = dtype == DSSD_BF16 ? 2 : 4;
    unsigned ctas = 1;
    while (ctas < 8 && blocks > kWarps * (int)ctas && ((long long)P.B * ctas * 2 <= 448 || (long long)P.V * esz > 72000ll * ctas)) ctas *= 2;
    if (ctas == 8 && P.B <= 4 && blocks > kWarps * 8) ctas = 16;
    cudaError_t e = cudaErrorNotSupported;
    const bool shift = (P.V | P.row_stride) % 4 != 0 || reinterpret_cast<uintptr_t>(P.logits) % 16 != 0 || reinterpret_cast<uintptr_t>(P.draft_q) % 16 != 0;
    for (; e == cudaErrorNotSupported; ctas /= 2) {  // (a device that takes no clusters of sixteen)
        const int per = (blocks + (int)ctas - 1) / (int)ctas;
        P.slice = per > (1 << 30) / kBlock ? 1 << 30 : per * kBlock;
        P.chunk = kBlock;
        while ((long long)P.chunk * kMaxChunks < P.slice) P.chunk *= 2;
        if (dtype == DSSD_BF16) e = shift ? launch_either<DSSD_BF16, true>(P, ctas, stream) : launch_either<DSSD_BF16, false>(P, ctas, stream);
        else e = shift ? launch_either<DSSD_F32, true>(P, ctas, stream) : launch_either<DSSD_F32, false>(P, ctas, stream);
        if (ctas <= 8) break;
    }
    return e;
}

}  // namespace dssd
