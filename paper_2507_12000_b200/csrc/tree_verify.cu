// The verdict on a drafted tree: one thread-block cluster per sequence walks from the root to the last accepted node.
//
// After r rejections at a node the residual distribution is max(0, p - a q) / m with two numbers a and m:
//   max(0, max(0, p - a q) / m - c q) = max(0, p - (a + m c) q) / m,
// (inside the outer maximum nothing changes where p - a q < 0, since q >= 0), so a rejection is one sum over the two rows
// as they lie in memory and no row is ever written.  Drawing siblings without replacement only scales q by c between them:
// a rejected token x has p(x) - a q(x) <= 0 from then on, so that its removal from q is not seen.
//
// Every CTA of the cluster holds a slice of the vocabulary and the same scalars; sums meet through
// distributed shared memory and are added in rank order by everybody, so that all CTAs take the same way.  A node costs one pass over its logits
// and one exchange, a rejection one pass over both rows and one exchange; the last of these passes leaves the sums of chunks that the draw
// picks from.  A warp takes a chunk of 512 entries at a time.
//
// The draw compares a uniform with sums over 10^5 terms: an error of 1e-7 in p, in the sum or in a would move a step of the distribution past the
// uniform once in a few hundred draws.  So p and the sums are float64: 2^x by a table of 16 entries (each in banks of its own: no conflicts) and a
// polynomial.  No maximum is needed, since float64 holds 2^(+-1000): a row whose sum leaves that range is taken again, relative to its maximum.
//
// Bound by the latency of a chain of dependent reductions for few sequences; by the float64 pipes (10 to 12 operations an entry) and the visited
// rows for many.
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
    double part[2][kMaxCluster][2];  // what the CTAs of the cluster exchange, in turns
    double warp[kWarps][2];
    double chunk[kMaxChunks];
    double own, picked;
    int token[kMaxNodes];
    short parent[kMaxNodes], child[kMaxNodes], sibling[kMaxNodes];
    int bad, found;
};

__device__ __forceinline__ double as_double(int hi, int lo) { return __hiloint2double(hi, lo); }

// A logit as float64 by its bits (a conversion instruction has a quarter of the throughput of a product).  Zeros become 2^-127; infinities and NaN
// become numbers of 2^128 and more.
template <int DT>
__device__ __forceinline__ double widen(uint32_t w)  // the bits of a float32
{
    const int hi = (int)(((w & 0x7fffffffu) >> 3) + 0x38000000u | (w & 0x80000000u));
    return as_double(hi, DT == DSSD_BF16 ? 0 : (int)(w << 29));
}

// 2^x = 2^(k / 16) 2^r, |r| <= 1/32; the polynomial is the exponential series to the fourth power (relative error below 5e-11).
// 0 below 2^-1000, infinity above 2^1000.
__device__ __forceinline__ double exp2_64(double x, const double *table)
{
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
    const bool far = (hi & 0x7fffffffu) > 0x408f4000u;  // |x| > 1000
    const int yh = far ? ((int)hi < 0 ? 0 : 0x7ff00000) : __double2hiint(y) + ((k >> 4) << 20);
    return as_double(yh, far ? 0 : __double2loint(y));
}

struct Two {
    double a, b;
};

// (a, b) of all threads, warps in order and CTAs in rank order; the same in every thread.  own: this CTA's a.
__device__ Two cluster_sum(VerifySmem &S, Two v, unsigned ctas, int &turn)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v.a = warp_sum(v.a);
    v.b = warp_sum(v.b);
    if (lane == 0) S.warp[warp][0] = v.a, S.warp[warp][1] = v.b;
    __syncthreads();
    Two s = {0.0, 0.0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s.a += S.warp[w][0], s.b += S.warp[w][1];
    if (ctas == 1) {
        __syncthreads();
        return s;
    }
    const unsigned me = cluster_rank();
    if (threadIdx.x < ctas) {
        cluster_store(&S.part[turn][me][0], threadIdx.x, s.a);
        cluster_store(&S.part[turn][me][1], threadIdx.x, s.b);
    }
    cluster_arrive();
    cluster_wait();
    Two all = {0.0, 0.0};
    for (unsigned c = 0; c < ctas; ++c) all.a += S.part[turn][c][0], all.b += S.part[turn][c][1];
    turn ^= 1;
    return all;
}

template <int DT>
struct Logits;
template <>
struct Logits<DSSD_BF16> {
    typedef Quads16 Q;
    static constexpr uint32_t kFill = 0xff80u;
    __device__ static uint32_t bits(const uint2 &v, int i) { return i == 0 ? v.x << 16 : i == 1 ? v.x & 0xffff0000u : i == 2 ? v.y << 16 : v.y & 0xffff0000u; }
    __device__ static uint32_t one(const char *row, int v) { return ld_row_u16(row + 2ll * v) << 16; }
};
template <>
struct Logits<DSSD_F32> {
    typedef Quads32 Q;
    static constexpr uint32_t kFill = 0xff800000u;
    __device__ static uint32_t bits(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ static uint32_t one(const char *row, int v) { return ld_row_u32(row + 4ll * v); }
};
__device__ __forceinline__ bool is_nan(uint32_t w) { return (w & 0x7fffffffu) > 0x7f800000u; }

// kShift: rows may begin off the boundaries of four entries
template <int DT, bool kShift>
__global__ void __launch_bounds__(kThreads, 3) tree_verify_kernel(const __grid_constant__ TreeVerifyParams P)
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
    int turn = 0;
    unsigned eflags = S.bad ? DSSD_EDGE_FLAG_BAD_PARENT : 0u, rflags = 0;

    int node = 0, length = 0;
    double a = 0.0, m = 1.0, c = 1.0, gone = 0.0, ref = 0.0, sum = 1.0, inv = 1.0;
    bool alive = true;
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
    auto lse_pass = [&](bool keep) {
        Two s = {0.0, 0.0};
        for (int k = warp; k < chunks; k += kWarps) {
            double part = 0.0;
            unsigned odd = 0;
            for (int at = v0 + k * P.chunk; at < min(v1, v0 + (k + 1) * P.chunk); at += kBlock) {
                WarpQuads<typename E::Q, 4, kShift> L;
                L.load(row, P.V, at, E::kFill);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const typename E::Q::Raw w = L.at(u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x = E::bits(w, i);
                        odd |= is_nan(x);
                        part += exp2_64(__fma_rn(widen<DT>(x), P.c1, -ref), S.table);
                    }
                }
            }
            s.b += odd ? 1.0 : 0.0;
            if (keep) {
                part = warp_sum(part);
                if (lane == 0) S.chunk[k] = part;
                s.a += lane == 0 ? part : 0.0;
            } else
                s.a += part;
        }
        return s;
    };
    auto rest_pass = [&](bool keep) {  // in units of the row's sum
        double total = 0.0;
        const double aS = a * sum;
        for (int k = warp; k < chunks; k += kWarps) {
            double part = 0.0;
            for (int at = v0 + k * P.chunk; at < min(v1, v0 + (k + 1) * P.chunk); at += kBlock) {
                WarpQuads<typename E::Q, 4, kShift> L;
                WarpQuads<Quads32, 4, kShift> R;
                L.load(row, P.V, at, E::kFill);
                R.load(reinterpret_cast<const char *>(qrow), P.V, at, 0u);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const typename E::Q::Raw w = L.at(u);
                    const uint4 q = R.at(u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const double e = exp2_64(__fma_rn(widen<DT>(E::bits(w, i)), P.c1, -ref), S.table);
                        const uint32_t qb = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
                        const double r = __fma_rn(-aS, widen<DSSD_F32>(qb), e);  // (a q of zero is 2^-127: below any p)
                        part += r > 0.0 ? r : 0.0;
                    }
                }
            }
            if (keep) {
                part = warp_sum(part);
                if (lane == 0) S.chunk[k] = part;
                total += lane == 0 ? part : 0.0;
            } else
                total += part;
        }
        return total;
    };
    if (me == 0 && t == 0) P.path[b * P.N] = 0;
    bool has_child, kept;
    while (true) {
        row = static_cast<const char *>(P.logits) + (b * P.N + node) * P.row_stride * (long long)E::Q::kBytes;
        qrow = P.draft_q + (b * P.N + node) * (long long)P.V;
        int j = S.child[node];
        has_child = j > 0;
        kept = !has_child;  // the pass leaves the chunks' sums
        Asked next = ask(j);
        ref = 0.0;
        Two all = cluster_sum(S, lse_pass(kept), ctas, turn);
        alive = all.b == 0.0;
        if (alive && !(all.a > 1e-280 && all.a < 1e280)) {
            // out of range: relative to the row's maximum, which the CTAs find by the same exchange, each for itself
            float mx = DSSD_NEG_INF;
            for (int v = t; v < P.V; v += kThreads) mx = fmaxf(mx, __uint_as_float(E::one(row, v)));
            mx = warp_max(mx);
            __syncthreads();
            if (lane == 0) S.warp[warp][0] = (double)mx;
            __syncthreads();
            double top = S.warp[0][0];
            for (int w = 1; w < kWarps; ++w) top = fmax(top, S.warp[w][0]);
            __syncthreads();
            alive = top > -1e300 && top < 1e300;
            if (alive) {
                ref = top * P.c1;
                all = cluster_sum(S, lse_pass(kept), ctas, turn);
            }
        }
        if (!alive) eflags |= DSSD_EDGE_FLAG_NONFINITE;
        sum = all.a;
        inv = 1.0 / sum;
        a = 0.0, m = 1.0, c = 1.0, gone = 0.0;
        bool taken = false;
        while (j > 0) {
            if (!next.ok) eflags |= DSSD_EDGE_FLAG_BAD_TOKEN;
            const double qx = (double)next.q, u = (double)next.u;
            const double px = exp2_64(__fma_rn(widen<DT>(next.l), P.c1, -ref), S.table) * inv;
            const double left = fmax(px - a * qx, 0.0);
            if (next.ok && alive && u < 1.0 && (qx <= 0.0 ? left > 0.0 : u * (c * m) * qx < left)) {
                taken = true;
                break;
            }
            // rejected: what is left of p
            a += c * m;
            if (!P.replacement) {
                if (next.ok && qx > 0.0) gone += qx;
                c = 1.0 / fmax(1.0 - gone, 1e-300);  // (nothing left of q: p where q has no mass)
            }
            j = S.sibling[j];
            next = ask(j);
            kept = j == 0;
            m = alive ? cluster_sum(S, {rest_pass(kept), 0.0}, ctas, turn).a * inv : 0.0;
        }
        if (!taken) break;
        node = j;
        ++length;
        if (me == 0 && t == 0) P.path[b * P.N + length] = j;
    }

    // the draw, from p or from max(0, p - a q), both in units of the row's sum
    if (!has_child) rflags |= DSSD_RS_FLAG_BONUS;
    if (a > 0.0 && !(m > 0.0)) {
        rflags |= DSSD_RS_FLAG_FALLBACK;
        a = 0.0;
        if (alive) cluster_sum(S, lse_pass(true), ctas, turn);
    }
    const double aS = a * sum;
    auto mass = [&](int v) {
        double r = exp2_64(__fma_rn(widen<DT>(E::one(row, v)), P.c1, -ref), S.table);
        if (a > 0.0) r = __fma_rn(-aS, widen<DSSD_F32>(ld_row_u32(qrow + v)), r);
        return r > 0.0 ? r : 0.0;
    };
    __syncthreads();
    // a CTA's sum is that of its chunks in order
    if (warp == 0) {
        double s = 0.0;
        for (int k = lane; k < chunks; k += 32) s += alive ? S.chunk[k] : 0.0;
        s = warp_sum(s);
        if (lane == 0) S.own = s;
    }
    __syncthreads();
    const double own = S.own;
    if (ctas > 1) {
        if (t < (int)ctas) cluster_store(&S.part[turn][me][0], t, own);
        cluster_arrive();
        cluster_wait();
    }
    double total = 0.0;
    for (unsigned k = 0; k < ctas; ++k) total += ctas > 1 ? S.part[turn][k][0] : own;
    const double target = (double)ld_after(P.uniforms_rs + b) * total;
    int owner = -1, last = 0;  // last: the last CTA with mass
    double run = 0.0, before = 0.0;
    for (unsigned k = 0; k < ctas; ++k) {
        const double w = ctas > 1 ? S.part[turn][k][0] : own;
        if (w > 0.0) last = (int)k;
        if (owner < 0 && run + w > target) owner = (int)k, before = run;
        run += w;
    }
    const bool invalid = !alive || !(total > 0.0);
    const bool short_of = owner < 0;  // rounding left none: the last entry with mass
    if (short_of) owner = last;
    if (invalid) rflags |= DSSD_RS_FLAG_INVALID;
    if (me == (unsigned)(invalid ? 0 : owner) && warp == 0) {
        int token = -1;
        if (!invalid) {
            // the chunk, 32 at a time
            double r = before;
            int pick = -1, lastk = 0;
            for (int k0 = 0; k0 < chunks && pick < 0; k0 += 32) {
                const int k = k0 + lane;
                const double w = k < chunks ? S.chunk[k] : 0.0;
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
            const int e = min(v1, v0 + (k + 1) * P.chunk);
            for (int base = v0 + k * P.chunk; base < e && token < 0; base += 128) {
                // four runs of 32 entries: their loads together
                double w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = base + 32 * i + lane < e ? mass(base + 32 * i + lane) : 0.0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    double cum = w[i];
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double up = __shfl_up_sync(0xffffffffu, cum, o);
                        if (lane >= o) cum += up;
                    }
                    const unsigned some = __ballot_sync(0xffffffffu, w[i] > 0.0);
                    if (some) last_v = base + 32 * i + 31 - __clz(some);
                    const unsigned over = __ballot_sync(0xffffffffu, w[i] > 0.0 && r + cum > target);
                    if (hit && over && token < 0) token = base + 32 * i + __ffs(over) - 1;
                    r += __shfl_sync(0xffffffffu, cum, 31);
                }
            }
            if (token < 0) token = last_v;
        }
        if (lane == 0) P.token[b] = token;
    }
    if (me == 0) {
        for (int k = length + 1 + t; k < P.N; k += kThreads) P.path[b * P.N + k] = -1;
        if (t == 0) {
            P.accept_len[b] = length;
            if (P.edge_flags) P.edge_flags[b] = eflags;
            if (P.rs_flags) P.rs_flags[b] = rflags;
        }
    }
    if (ctas > 1) {  // (a CTA's shared memory outlives the others' stores into it)
        cluster_arrive();
        cluster_wait();
    }
}

template <int DT, bool kShift>
cudaError_t launch_as(const TreeVerifyParams &P, unsigned ctas, cudaStream_t stream)
{
    if (ctas > 8) {
        static PerContext allowed;
        if (!allowed.get([] { return (int)allow_cluster(tree_verify_kernel<DT, kShift>, 16, kThreads); })) {
            cudaGetLastError();
            return cudaErrorNotSupported;
        }
    }
    return launch_pdl(tree_verify_kernel<DT, kShift>, (unsigned)P.B * ctas, kThreads, stream, P, 0, ctas);
}

}  // namespace

size_t tree_verify_workspace(int B, int N, int V)
{
    (void)V;
    return (((size_t)B * (size_t)N * 16) + 255) & ~(size_t)255;
}

cudaError_t tree_verify_launch(TreeVerifyParams &P, int dtype, void *workspace, cudaStream_t stream)
{
    (void)workspace;
    const int blocks = (P.V + kBlock - 1) / kBlock;
    // Clusters of eight as long as every warp has a block: a sequence's passes follow one another, and the GPU holds many more sequences than
    // eights of CTAs, so that long and short walks even out.  Sixteen where there are few sequences.
    unsigned ctas = 1;
    while (ctas < 8 && blocks > kWarps * (int)ctas) ctas *= 2;
    if (ctas == 8 && P.B <= 18 && blocks > kWarps * 8) ctas = 16;
    cudaError_t e = cudaErrorNotSupported;
    const bool shift = (P.V | P.row_stride) % 4 != 0 || reinterpret_cast<uintptr_t>(P.logits) % 16 != 0 || reinterpret_cast<uintptr_t>(P.draft_q) % 16 != 0;
    for (; e == cudaErrorNotSupported; ctas /= 2) {  // (a device that takes no clusters of sixteen)
        const int per = (blocks + (int)ctas - 1) / (int)ctas;
        P.slice = per > (1 << 30) / kBlock ? 1 << 30 : per * kBlock;
        P.chunk = kBlock;
        while ((long long)P.chunk * kMaxChunks < P.slice) P.chunk *= 2;
        if (dtype == DSSD_BF16) e = shift ? launch_as<DSSD_BF16, true>(P, ctas, stream) : launch_as<DSSD_BF16, false>(P, ctas, stream);
        else e = shift ? launch_as<DSSD_F32, true>(P, ctas, stream) : launch_as<DSSD_F32, false>(P, ctas, stream);
        if (ctas <= 8) break;
    }
    return e;
}

}  // namespace dssd
