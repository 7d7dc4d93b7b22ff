// The verdict on a drafted tree: one thread-block cluster per sequence walks from the root to the last accepted node.
//
// After r rejections at a node the residual distribution is max(0, p - a q) / m with two numbers a and m:
//   max(0, max(0, p - a q) / m - c q) = max(0, p - (a + m c) q) / m,
// (inside the outer maximum nothing changes where p - a q < 0, since q >= 0), so a rejection is one sum over the two rows
// as they lie in memory and no row is ever written.  Drawing siblings without replacement only scales q by c between them:
// a rejected token x has p(x) - a q(x) <= 0 from then on, so that its removal from q is not seen.
//
// Every CTA of the cluster holds a slice of the vocabulary and the same scalars; sums meet through
// distributed shared memory and are added in rank order by everybody, so that all CTAs take the same way.  Whole numbers come out
// of comparisons with sums over 10^5 terms: p and the sums are float64, 2^x by a table of 64 entries and a polynomial.
//
// Bound by the latency of a chain of dependent reductions for few sequences, by the visited rows for many.
#include "launch.h"
#include "quads.cuh"
#include "tree.cuh"
#include "tree_ops.h"

namespace dssd {

namespace {

constexpr int kVT = 512;  // threads
constexpr int kVWarps = kVT / 32;
constexpr int kMaxCluster = 16;
constexpr int kMaxChunks = 1024;  // of a CTA's slice, for the draw

struct VerifySmem {
    double table[64];
    double part[2][kMaxCluster][2];  // what the CTAs of the cluster exchange, in turns
    double warp[kVWarps][2];
    double chunk[kMaxChunks];
    double picked[2];
    int token[kMaxNodes];
    short parent[kMaxNodes];
    int bad;
    int found;
};

// 2^x for x <= 0 or so: 2^x = 2^(k / 64) 2^r, |r| <= 1/128; the polynomial is the exponential series to the fourth power
// (relative error below 4e-14).  Below 2^-1000: 0.
__device__ __forceinline__ double exp2_64(double x, const double *table)
{
    if (!(x > -1000.0)) return x != x ? x : 0.0;
    const double big = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to a whole number, held in the low bits
    const double t = __fma_rn(x, 64.0, big);
    const int k = __double2loint(t);
    const double r = __fma_rn(t - big, -1.0 / 64.0, x) * 0.69314718055994530942;
    double p = __fma_rn(r, 1.0 / 24.0, 1.0 / 6.0);
    p = __fma_rn(p, r, 0.5);
    p = __fma_rn(p, r, 1.0);
    p = __fma_rn(p, r, 1.0);
    const double y = p * table[k & 63];
    return __hiloint2double(__double2hiint(y) + ((k >> 6) << 20), __double2loint(y));
}

struct Two {
    double a, b;
};

// (a, b) of all CTAs, added in rank order; the same in every thread
__device__ Two cluster_sum(VerifySmem &S, Two v, unsigned ctas, int &turn)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v.a = warp_sum(v.a);
    v.b = warp_sum(v.b);
    __syncthreads();
    if (lane == 0) S.warp[warp][0] = v.a, S.warp[warp][1] = v.b;
    __syncthreads();
    Two s = {0.0, 0.0};
    for (int w = 0; w < kVWarps; ++w) s.a += S.warp[w][0], s.b += S.warp[w][1];
    if (ctas == 1) return s;
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

// the largest a over all CTAs
__device__ double cluster_max(VerifySmem &S, double v, unsigned ctas, int &turn)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if (lane == 0) S.warp[warp][0] = v;
    __syncthreads();
    for (int w = 0; w < kVWarps; ++w) v = fmax(v, S.warp[w][0]);
    if (ctas == 1) return v;
    const unsigned me = cluster_rank();
    if (threadIdx.x < ctas) cluster_store(&S.part[turn][me][0], threadIdx.x, v);
    cluster_arrive();
    cluster_wait();
    for (unsigned c = 0; c < ctas; ++c) v = fmax(v, S.part[turn][c][0]);
    turn ^= 1;
    return v;
}

template <int DT>
__device__ __forceinline__ float logit(const char *row, int v)
{
    return DT == DSSD_BF16 ? __uint_as_float(ld_row_u16(row + 2ll * v) << 16) : __uint_as_float(ld_row_u32(row + 4ll * v));
}

template <int DT>
__global__ void __launch_bounds__(kVT) tree_verify_kernel(const __grid_constant__ TreeVerifyParams P)
{
    __shared__ VerifySmem S;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    unsigned ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const unsigned me = ctas > 1 ? cluster_rank() : 0;
    const long long b = blockIdx.x / ctas;
    const int v0 = (int)min((long long)P.V, (long long)me * P.slice), v1 = (int)min((long long)P.V, (long long)v0 + P.slice);
    if (t < 64) S.table[t] = exp2(t / 64.0);
    pdl_wait();
    pdl_trigger();
    load_tree(P.parents, b, P.N, S.parent, &S.bad);
    if (t > 0 && t < P.N) S.token[t] = ld_after(P.draft_tokens + b * (P.N - 1) + t - 1);
    if (ctas > 1) {  // nobody writes into a CTA's shared memory before it runs
        cluster_arrive();
        cluster_wait();
    }
    __syncthreads();
    int turn = 0;
    unsigned eflags = S.bad ? DSSD_EDGE_FLAG_BAD_PARENT : 0u, rflags = 0;

    constexpr int esz = Elem<DT>::kBytes;
    int node = 0, length = 0;
    double a = 0.0, m = 1.0, c = 1.0, gone = 0.0, ref = 0.0, inv = 0.0;
    bool alive = true, fresh = true, has_child = false;
    const char *row = nullptr;
    const float *qrow = nullptr;
    if (me == 0 && t == 0) P.path[b * P.N] = 0;
    for (int j = 1; j <= P.N; ++j) {
        if (fresh) {  // the node's log-sum-exp
            row = static_cast<const char *>(P.logits) + (b * P.N + node) * P.row_stride * (long long)esz;
            qrow = P.draft_q + (b * P.N + node) * (long long)P.V;
            float mx = DSSD_NEG_INF;
            bool odd = false;
            for (int v = v0 + t; v < v1; v += kVT) {
                const float x = logit<DT>(row, v);
                odd |= !(x < __int_as_float(0x7f800000));
                mx = fmaxf(mx, x);
            }
            // one exchange tells both: +inf stands for a row that has no finite log-sum-exp
            const double top = cluster_max(S, odd ? (double)__int_as_float(0x7f800000) : (double)mx, ctas, turn);
            alive = top > -1e300 && top < 1e300;
            ref = top * P.c1;
            double s = 0.0;
            if (alive)
                for (int v = v0 + t; v < v1; v += kVT) s += exp2_64(__fma_rn((double)logit<DT>(row, v), P.c1, -ref), S.table);
            const Two all = cluster_sum(S, {s, 0.0}, ctas, turn);
            if (!alive) eflags |= DSSD_EDGE_FLAG_NONFINITE;
            inv = 1.0 / all.a;
            a = 0.0, m = 1.0, c = 1.0, gone = 0.0;
            fresh = false;
            has_child = false;
        }
        if (j == P.N) break;
        if (S.parent[j] != node) continue;
        has_child = true;
        const int x = S.token[j];
        double left = 0.0, qx = 0.0;
        bool ok = x >= 0 && x < P.V;
        if (!ok) eflags |= DSSD_EDGE_FLAG_BAD_TOKEN;
        if (ok) {
            const double px = exp2_64(__fma_rn((double)logit<DT>(row, x), P.c1, -ref), S.table) * inv;
            qx = (double)ld_after(qrow + x);
            left = px - a * qx;
            left = left > 0.0 ? left : 0.0;
            const double u = (double)ld_after(P.uniforms + b * (P.N - 1) + j - 1);
            ok = alive && (qx <= 0.0 ? left > 0.0 && u < 1.0 : u < 1.0 && u * (c * m) * qx < left);
        }
        if (ok) {
            node = j;
            ++length;
            if (me == 0 && t == 0) P.path[b * P.N + length] = j;
            fresh = true;
            continue;
        }
        // rejected: what is left of p
        a += c * m;
        if (!P.replacement) {
            if (qx > 0.0) gone += qx;
            c = 1.0 / fmax(1.0 - gone, 1e-300);  // (nothing left of q: p where q has no mass)
        }
        double s = 0.0;
        if (alive)
            for (int v = v0 + t; v < v1; v += kVT) {
                const double r = exp2_64(__fma_rn((double)logit<DT>(row, v), P.c1, -ref), S.table) * inv - a * (double)__uint_as_float(ld_row_u32(qrow + v));
                if (r > 0.0) s += r;
            }
        m = cluster_sum(S, {s, 0.0}, ctas, turn).a;
    }

    // the draw
    if (!has_child) rflags |= DSSD_RS_FLAG_BONUS;
    if (a > 0.0 && !(m > 0.0)) {
        rflags |= DSSD_RS_FLAG_FALLBACK;
        a = 0.0;
    }
    auto mass = [&](int v) {
        double r = exp2_64(__fma_rn((double)logit<DT>(row, v), P.c1, -ref), S.table) * inv;
        if (a > 0.0) r -= a * (double)__uint_as_float(ld_row_u32(qrow + v));
        return r > 0.0 ? r : 0.0;
    };
    const int width = v1 - v0;
    int size = 256;
    while ((long long)size * kMaxChunks < P.slice) size *= 2;
    const int chunks = (width + size - 1) / size;
    if (alive)
        for (int k = warp; k < chunks; k += kVWarps) {
            double s = 0.0;
            const int e = min(width, (k + 1) * size);
            for (int v = k * size + lane; v < e; v += 32) s += mass(v0 + v);
            s = warp_sum(s);
            if (lane == 0) S.chunk[k] = s;
        }
    __syncthreads();
    // a CTA's sum is that of its chunks in index order
    if (t == 0) {
        double s = 0.0;
        for (int k = 0; k < chunks; ++k) s += alive ? S.chunk[k] : 0.0;
        S.picked[0] = s;
    }
    __syncthreads();
    const double own = S.picked[0];
    double before = 0.0, total = own;
    int last = 0;  // the last CTA with mass
    if (ctas > 1) {
        if (t < (int)ctas) cluster_store(&S.part[turn][me][0], t, own);
        cluster_arrive();
        cluster_wait();
        total = 0.0;
        for (unsigned k = 0; k < ctas; ++k) total += S.part[turn][k][0];
    }
    const double u = (double)ld_after(P.uniforms_rs + b);
    const double target = u * total;
    int owner = -1;
    double run = 0.0;
    for (unsigned k = 0; k < ctas; ++k) {
        const double w = ctas > 1 ? S.part[turn][k][0] : own;
        if (w > 0.0) last = (int)k;
        if (owner < 0 && run + w > target) owner = (int)k, before = run;
        run += w;
    }
    const bool invalid = !alive || !(total > 0.0);
    const bool short_of = owner < 0;  // rounding left none
    if (short_of) owner = last;
    if (invalid) rflags |= DSSD_RS_FLAG_INVALID;
    if (me == (unsigned)(invalid ? 0 : owner)) {
        if (t == 0) {
            S.found = -1;
            int k = 0, lastk = 0;
            double r = before;
            bool hit = false;
            if (!invalid) {
                for (k = 0; k < chunks; ++k) {
                    if (S.chunk[k] > 0.0) lastk = k;
                    if (!short_of && r + S.chunk[k] > target) {
                        hit = true;
                        break;
                    }
                    r += S.chunk[k];
                }
            }
            S.picked[0] = r;
            S.found = hit ? k : -1 - lastk;
        }
        __syncthreads();
        if (warp == 0) {
            int token = -1;
            if (!invalid) {
                const bool hit = S.found >= 0;
                const int k = hit ? S.found : -1 - S.found;
                double r = S.picked[0];
                int last_v = -1;
                const int e = min(width, (k + 1) * size);
                for (int base = k * size; base < e && token < 0; base += 32) {
                    const int v = base + lane;
                    const double w = v < e ? mass(v0 + v) : 0.0;
                    double cum = w;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double up = __shfl_up_sync(0xffffffffu, cum, o);
                        if (lane >= o) cum += up;
                    }
                    const unsigned some = __ballot_sync(0xffffffffu, w > 0.0);
                    if (some) last_v = base + 31 - __clz(some);
                    const unsigned over = __ballot_sync(0xffffffffu, w > 0.0 && r + cum > target);
                    if (hit && over) token = v0 + base + __ffs(over) - 1;
                    r += __shfl_sync(0xffffffffu, cum, 31);
                }
                if (token < 0) token = v0 + last_v;
            }
            if (lane == 0) P.token[b] = token;
        }
    }
    if (me == 0) {
        for (int k = length + 1 + t; k < P.N; k += kVT) P.path[b * P.N + k] = -1;
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

}  // namespace

size_t tree_verify_workspace(int B, int N, int V)
{
    (void)V;
    return (((size_t)B * (size_t)N * 16) + 255) & ~(size_t)255;
}

cudaError_t tree_verify_launch(TreeVerifyParams &P, int dtype, void *workspace, cudaStream_t stream)
{
    (void)workspace;
    // as many CTAs to a sequence as there are SMs for them, but no fewer than two turns of the threads each
    unsigned ctas = 1;
    while (ctas < 8 && (long long)P.B * ctas * 2 <= 2 * 148 && P.V > 2 * kVT * (int)ctas) ctas *= 2;
    P.slice = (int)(((long long)P.V + ctas - 1) / ctas);
    const unsigned grid = (unsigned)P.B * ctas;
    return dtype == DSSD_BF16 ? launch_pdl(tree_verify_kernel<DSSD_BF16>, grid, kVT, stream, P, 0, ctas)
                              : launch_pdl(tree_verify_kernel<DSSD_F32>, grid, kVT, stream, P, 0, ctas);
}

}  // namespace dssd
