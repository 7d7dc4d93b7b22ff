// Attention of a drafted tree's nodes over a paged cache.
//
// The rows of a key head are the nodes times the query heads that share it, 128 to a tile of the tensor core: S = Q K^T for 128
// keys at a time into tensor memory, a thread per row for the softmax, P back into tensor memory as 16-bit values, O += P V.  A tile of
// keys serves all rows of its head, so the cache is read once (once per 256 rows).  The keys of a sequence are
// its nodes (tile 0, masked by ancestors) and then the cache, 128 positions to a tile, brought in by tiled copies, one per page or part of a
// page, into a ring of stages; the copies fill what lies outside a head's size with zeros, so any size works on 64 or 128 columns.
//
// Two groups of four warps do the softmax, each with an S and an O of its own (tensor memory holds two of each): while one is at its exponentials
// the tensor core works for the other.  With more than 128 rows each group has a tile of rows; with fewer both have the same rows and every
// other tile of keys, and the two results are joined at the end.  One group for all keys took 2700 cycles a tile, as long as the cache's bytes take to arrive.
//
// What bounds it: the cache's bytes as long as a tile's 64 KB take longer to arrive (2900 cycles of an SM's share of the measured
// bandwidth) than 128 rows of softmax (128 exponentials a thread, 1024 cycles of the special-function units) and
// two products (1024 cycles); for 256 rows the products and exponentials come to the same 2048 cycles.
//
// Split: all (sequence, key head, row tile) items, each with its tiles, lie on one line, and every CTA takes an equal piece of that line whatever the lengths are.
// An item that lies in several pieces leaves a partial result (O, maximum, sum) per piece in the workspace, at places that only its CTA writes, and a second
// kernel joins them in order: the same bits on every run, and nothing to clear.
//
// The maximum that weights refer to is only raised when a tile exceeds it by more than 2^8: raising it means to read, scale and write back O.
// The sum refers to the same maximum, so the quotient is not changed; P stays below 2^8.
#include "launch.h"
#include "quads.cuh"
#include "tcgen05.cuh"
#include "tree.cuh"
#include "tree_ops.h"

#include <cuda_bf16.h>

namespace dssd {

namespace {

constexpr int kTile = 128;      // keys of a tile, rows of a tile
constexpr int kMaxCtas = 148;   // pieces of the line
// tiles to a piece at least (us with 1, 2 and 4: B=1 N=1 ctx 2047 16.4 18.0 20.1; B=20 N=9 ctx 29 17.1 11.6 17.7; B=2 N=11 ctx 4760 18.8 16.6 18.1)
constexpr int kMinTiles = 2;
constexpr int kAttend = 384;     // threads: copies, products and an idle warp; the two groups of the softmax

struct Geometry {
    CUtensorMap q, k_new, v_new, k_cache, v_cache;
    const int32_t *block_table;
    int64_t table_stride;
    int max_pages, num_pages, page_size;
    int box_log;                // positions of a copy, the greatest common divisor of the page and 128: a power of two
    int tile_pages, tile_rest;  // 128 divided by the page: the quotient and the rest
    const int32_t *ctx_len, *parents;
    int B, N, Hkv, G, D;
    int nodes_per_tile, row_items;  // nodes in a tile of rows; items of kMT tiles to a key head
    float scale, c;                 // c = scale * log2(e)
    void *o;
    int64_t o_b, o_n, o_h;
    float *lse;
    uint32_t *flags;
    long long wait_cycles;  // the limit of every wait inside
    int withhold;           // the sequence whose nodes' keys are never copied (-1: none)
    float *part;      // [2 kMaxCtas][kMT * 128][kDP]
    float2 *part_ml;  // [2 kMaxCtas][kMT * 128] maximum in powers of two, sum
    int4 *joins;      // [kMaxCtas] the item that this piece is the second of: sequence, item, slot of its first piece, its last piece; sequence -1: none
};

__device__ __forceinline__ int length(const Geometry &P, long long b, bool *bad = nullptr)
{
    const int n = ld_after(P.ctx_len + b);
    const int most = P.max_pages * P.page_size;
    if (bad) *bad = n < 0 || n > most;
    return min(max(n, 0), most);
}
__device__ __forceinline__ int tiles_of(int ctx) { return 1 + (ctx + kTile - 1) / kTile; }

// all tiles of the line, by one warp (all lanes get it)
__device__ long long measure(const Geometry &P, bool report)
{
    long long all = 0;
    for (long long i = threadIdx.x & 31; i < P.B; i += 32) {
        bool bad;
        all += tiles_of(length(P, i, &bad));
        if (report && bad && P.flags) atomicOr(P.flags + i, DSSD_CACHE_FLAG_BAD_LENGTH);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    return all * P.Hkv * P.row_items;
}
__device__ __forceinline__ long long pieces(long long total, unsigned grid)
{
    const long long n = (total + kMinTiles - 1) / kMinTiles;
    return n < (long long)grid ? n : (long long)grid;
}

// a / b of numbers that are small as a rule
__device__ __forceinline__ long long quotient(long long a, long long b)
{
    return ((a | b) >> 32) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// where a piece of the line begins
struct Place {
    long long b;
    int item, tile, tiles;  // item of the sequence; tile of it; its tiles
    int ctx;
};
__device__ Place find(const Geometry &P, long long at)  // one warp, all lanes get it
{
    const int lane = threadIdx.x & 31;
    const long long items = (long long)P.Hkv * P.row_items;
    Place r = {0, 0, 0, 1, 0};
    long long base = 0;
    for (long long i0 = 0; i0 < P.B; i0 += 32) {
        const long long i = i0 + lane;
        const int ctx = i < P.B ? length(P, i) : 0;
        const int t = i < P.B ? tiles_of(ctx) : 0;
        long long end = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end += up;
        }
        const unsigned in = __ballot_sync(0xffffffffu, i < P.B && base + end * items > at);
        if (in) {
            const int l = __ffs(in) - 1;
            const long long start = base + (__shfl_sync(0xffffffffu, end, l) - __shfl_sync(0xffffffffu, t, l)) * items;
            r.b = i0 + l;
            r.tiles = __shfl_sync(0xffffffffu, t, l);
            r.ctx = __shfl_sync(0xffffffffu, ctx, l);
            r.item = (int)quotient(at - start, r.tiles);
            r.tile = (int)((at - start) - (long long)r.item * r.tiles);
            return r;
        }
        base += __shfl_sync(0xffffffffu, end, 31) * items;
    }
    return r;
}
// the next item
__device__ __forceinline__ void advance(const Geometry &P, Place &p)
{
    p.tile = 0;
    if (++p.item == P.Hkv * P.row_items) {
        p.item = 0;
        if (++p.b < P.B) {
            p.ctx = length(P, p.b);
            p.tiles = tiles_of(p.ctx);
        }
    }
}

template <int DT>
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if (DT == DSSD_BF16) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    return pack_half2(lo, hi);
}

template <int DP, int kMT>
struct Smem {
    static constexpr int kStages = DP == 64 ? 5 : kMT == 1 ? 3 : 2;
    static constexpr int kChunk = kTile * 128;             // 64 columns of a tile
    static constexpr int kOperand = kTile * DP * 2;
    static constexpr int kQ = 0, kKV = kMT * kOperand;     // then K and V of the stages in turn
    static constexpr int kRest = kKV + kStages * 2 * kOperand;
    struct Rest {
        uint64_t q_full, q_empty, k_full[kStages], v_full[kStages], k_empty[kStages], v_empty[kStages], s_full[2], p_ready[2], o_done[2], o_free[2], half, drained;
        signed char parent[kMT == 1 ? 4 : 8][128];  // of the nodes, for each warp of the softmax that meets tile 0
        float2 other[kMT == 1 ? 128 : 1];     // maximum and sum of the second group's half of the keys
        Place place;
        long long count;
        uint32_t tmem;
        int failed;
    };
    static constexpr size_t kBytes = kRest + sizeof(Rest) + 1024;  // (the base is aligned by hand)
    static_assert(kBytes <= 232448, "a CTA has 227 KB of shared memory");
};

// Whichever wait ran out, nothing of this CTA's piece is sure to be done: all of its sequences say so, and what the second kernel would join is no
// number.  (A call, so that it takes no registers from what comes before it.)
__device__ __noinline__ void give_up(const Geometry &P, Place p, long long count, int rows)
{
    if (threadIdx.x == 0 && P.flags)
        while (count > 0) {
            atomicOr(P.flags + p.b, DSSD_CACHE_FLAG_TIMEOUT);
            count -= p.tiles - p.tile;
            advance(P, p);
        }
    const float nan = __int_as_float(0x7fc00000);
    for (int i = threadIdx.x; i < 2 * rows; i += kAttend) P.part_ml[2ll * blockIdx.x * rows + i] = make_float2(nan, nan);
}

template <int DT, int DP, int kMT>
__global__ void __launch_bounds__(kAttend, 1) tree_attention_kernel(const __grid_constant__ Geometry P)
{
    typedef Smem<DP, kMT> M;
    extern __shared__ unsigned char raw[];
    unsigned char *base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    typename M::Rest &S = *reinterpret_cast<typename M::Rest *>(base + M::kRest);
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    constexpr int kChunks = DP / 64;

    if (t == 0) {
        bar_init(&S.q_full, 1);
        bar_init(&S.q_empty, 1);
        for (int i = 0; i < M::kStages; ++i) {
            bar_init(&S.k_full[i], 1);
            bar_init(&S.v_full[i], 1);
            bar_init(&S.k_empty[i], 1);
            bar_init(&S.v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&S.s_full[i], 1);
            bar_init(&S.p_ready[i], 128);
            bar_init(&S.o_done[i], 1);
            bar_init(&S.o_free[i], 128);
        }
        bar_init(&S.half, 128);
        bar_init(&S.drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        S.failed = 0;
    }
    if (warp == 1) tmem_alloc(&S.tmem, 512);
    if (warp == 0 && lane == 0) {
        prefetch_map(&P.q);
        prefetch_map(&P.k_new);
        prefetch_map(&P.v_new);
        prefetch_map(&P.k_cache);
        prefetch_map(&P.v_cache);
    }
    pdl_wait();
    pdl_trigger();
    if (warp == 3) {  // which piece of the line is this CTA's
        const long long total = measure(P, blockIdx.x == 0), c = blockIdx.x;
        const long long n = pieces(total, gridDim.x);
        long long from = 0, to = 0;
        if (c < n) from = quotient(c * total, n), to = quotient((c + 1) * total, n);
        Place p = {0, 0, 0, 1, 0};
        if (to > from) p = find(P, from);
        if (lane == 0) {
            S.place = p, S.count = to - from;
            // an item that begins in the piece before and goes on here is joined under this piece's number
            int4 join = make_int4(-1, 0, 0, 0);
            if (to > from && p.tile > 0) {
                const long long x0 = from - p.tile, before = quotient((c - 1) * total, n);
                if (before <= x0) join = make_int4((int)p.b, p.item, 2 * (int)(c - 1) + (before == x0 ? 0 : 1), (int)quotient((x0 + p.tiles) * n - 1, total));
            }
            P.joins[c] = join;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = S.tmem;
    const Waits failed = {&S.failed, P.wait_cycles};
    Place at = S.place;
    long long left = S.count;

    if (warp == 0 || warp == 2) {
        // ---- copies: Q and K by one warp, V by the other
        const bool keys = warp == 0;
        const CUtensorMap *const fresh = keys ? &P.k_new : &P.v_new, *const cache = keys ? &P.k_cache : &P.v_cache;
        uint64_t *const full_bar = keys ? S.k_full : S.v_full, *const empty_bar = keys ? S.k_empty : S.v_empty;
        unsigned char *const ring = base + M::kKV + (keys ? 0 : M::kOperand);
        int stage = 0;
        unsigned round = 0, items = 0;
        bool ok = true;
        while (left > 0 && ok) {
            const int h = at.item / P.row_items, rt = at.item - h * P.row_items;
            const int n = (int)(left < at.tiles - at.tile ? left : at.tiles - at.tile);
            if (keys) {
                if (items) ok = warp_wait(&S.q_empty, (items - 1) & 1, failed);
                if (!ok) break;
                if (elect()) {
                    bar_expect(&S.q_full, (uint32_t)(kMT * kChunks * P.nodes_per_tile * P.G * 128));
                    for (int m = 0; m < kMT; ++m)
                        for (int x = 0; x < kChunks; ++x)
                            copy_5d(base + M::kQ + m * M::kOperand + x * M::kChunk, &P.q, &S.q_full, x * 64, 0, h, (rt * kMT + m) * P.nodes_per_tile, (int)at.b);
                }
                __syncwarp();
            }
            ++items;
            // Lane y looks up the page of the tile's box y (of its first 32), and where it lies in it, which it carries along from tile to tile (a division
            // each time took longer than the copies).  One thread issues the copies.
            const int first = (at.tile > 0 ? (at.tile - 1) * kTile : 0) + (lane << P.box_log);
            int page_at = first / P.page_size, off = first - page_at * P.page_size;
            const int32_t *table = P.block_table + at.b * P.table_stride;
            auto number = [&](int p) {
                int pg = ld_after(table + p);
                if (pg < 0 || pg >= P.num_pages) {
                    if (P.flags) atomicOr(P.flags + at.b, DSSD_CACHE_FLAG_BAD_PAGE);
                    pg = max(P.num_pages, 1);  // outside the cache: zeros come
                }
                return pg;
            };
            for (int i = at.tile; ok && i < at.tile + n; ++i) {
                unsigned char *const to = ring + stage * 2 * M::kOperand;
                uint64_t *const bar = full_bar + stage;
                const int pos = (i - 1) * kTile;
                const int valid = i == 0 ? P.N : min(kTile, at.ctx - pos);
                const int boxes = (valid + (1 << P.box_log) - 1) >> P.box_log;  // of the cache's tiles
                int page = 0, place = off;
                if (i > 0 && lane < boxes) page = number(page_at);  // before the wait for the stage
                ok = warp_wait(empty_bar + stage, (round & 1) ^ 1, failed);
                if (!ok) break;
                const bool one = elect();
                const bool withheld = keys && i == 0 && at.b == P.withhold;
                if (one && !withheld) bar_expect(bar, (uint32_t)(kChunks * 128 * (i == 0 ? P.N : boxes << P.box_log)));
                if (i == 0) {
                    if (one && !withheld)
                        for (int x = 0; x < kChunks; ++x) copy_4d(to + x * M::kChunk, fresh, bar, x * 64, h, 0, (int)at.b);
                } else {
                    for (int y0 = 0; y0 < boxes; y0 += 32) {
                        if (y0 > 0 && y0 + lane < boxes) {  // (pages of less than four positions)
                            const int p = pos + ((y0 + lane) << P.box_log);
                            page = number(p / P.page_size), place = p % P.page_size;
                        }
#pragma unroll 4
                        for (int y = 0; y < 32; ++y) {
                            if (y0 + y >= boxes) break;
                            const int pg = __shfl_sync(0xffffffffu, page, y), of = __shfl_sync(0xffffffffu, place, y);
                            unsigned char *const at_box = to + ((y0 + y) << (P.box_log + 7));
                            if (one)
#pragma unroll
                                for (int x = 0; x < kChunks; ++x) copy_4d(at_box + x * M::kChunk, cache, bar, x * 64, h, of, pg);
                        }
                    }
                    // 128 positions on
                    page_at += P.tile_pages;
                    off += P.tile_rest;
                    if (off >= P.page_size) off -= P.page_size, ++page_at;
                }
                __syncwarp();
                if (++stage == M::kStages) stage = 0, ++round;
            }
            left -= n;
            advance(P, at);
        }
        // What this warp asked for arrives before the shared memory goes, whoever gave up (as a rule it is there): the last use of each stage, and of Q.
        for (int s = 0; s < M::kStages; ++s) {
            const unsigned uses = round + (s < stage);
            if (uses) bar_drain(full_bar + s, (uses - 1) & 1, failed);
        }
        if (keys && items) bar_drain(&S.q_full, (items - 1) & 1, failed);
    } else if (warp == 1) {
        // ---- products: the warp goes through the tiles together and one thread issues, so that operands stay in uniform registers
        int stage = 0, next = 0;  // of PV, of QK
        unsigned round = 0, next_round = 0, items = 0;
        unsigned p_phase[2] = {0, 0}, uses[2] = {0, 0};
        bool ok = true;
        const uint64_t q_operand = operand(smem_u32(base + M::kQ), 16, 1024), k_operand = operand(smem_u32(base + M::kKV), 16, 1024);
        const uint64_t v_operand = operand(smem_u32(base + M::kKV + M::kOperand), M::kChunk, 1024);
        const bool one = elect();
        while (left > 0 && ok) {
            const int n = (int)(left < at.tiles - at.tile ? left : at.tiles - at.tile);
            ok = warp_wait(&S.q_full, items & 1, failed);
            if (!ok) break;
            auto valid_of = [&](int i) { return i == 0 ? P.N : min(kTile, at.ctx - (i - 1) * kTile); };
            // Operands step by adding to the low word of their descriptors (a place in shared memory, by 16 bytes; it never carries): made
            // anew for every product they took longer than the products.
            // S of group g for the tile of keys i
            auto scores = [&](int g, int i) {
                const uint64_t q = q_operand + (kMT == 2 ? g * (M::kOperand >> 4) : 0), k = k_operand + next * (2 * M::kOperand >> 4);
                const int valid = valid_of(i);
                const uint32_t sh = valid == kTile ? shape<DT == DSSD_BF16>(128, 128, false) : shape<DT == DSSD_BF16>(128, (valid + 15) / 16 * 16, false);
                if (one) {
#pragma unroll
                    for (int x = 0; x < DP / 16; ++x) {
                        const uint32_t in = ((x / 4) * M::kChunk + (x % 4) * 32) >> 4;
                        mma_ss(tmem + g * 128, q + in, k + in, sh, x > 0);
                    }
                    mma_commit(&S.s_full[g]);
                }
                __syncwarp();
            };
            auto outputs = [&](int g, int i, bool add) {
                const uint64_t v = v_operand + stage * (2 * M::kOperand >> 4);
                constexpr uint32_t sh = shape<DT == DSSD_BF16>(128, DP, true);
                const int steps = (valid_of(i) + 15) / 16;
                const uint32_t o = tmem + 256 + g * 128, p = tmem + g * 128;
                if (one) {
                    if (steps == 8) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) mma_ts(o, p + x * 8, v + x * (2048 >> 4), sh, add || x > 0);
                    } else
                        for (int x = 0; x < steps; ++x) mma_ts(o, p + x * 8, v + x * (2048 >> 4), sh, add || x > 0);
                    mma_commit(&S.o_done[g]);
                }
                __syncwarp();
            };
            auto commit = [&](uint64_t *bar) {
                if (one) mma_commit(bar);
                __syncwarp();
            };
            auto step_next = [&]() {
                commit(&S.k_empty[next]);
                if (++next == M::kStages) next = 0, ++next_round;
            };
            auto key_tile = [&]() {
                const bool there = warp_wait(&S.k_full[next], next_round & 1, failed);
                tc_after();
                return there;
            };
            const int first = at.tile, last = at.tile + n - 1;
            // the S that need no P before them
            if (kMT == 2) {
                if (!(ok = key_tile())) break;
                scores(0, first);
                scores(1, first);
                step_next();
            } else
                for (int g = 0; g < 2 && g < n && ok; ++g) {
                    if (!(ok = key_tile())) break;
                    scores(g, first + g);
                    step_next();
                }
            for (int i = first; i <= last && ok; ++i) {
                for (int g = kMT == 2 ? 0 : (i - first) & 1; g < 2 && ok; g += kMT == 2 ? 1 : 2) {
                    const bool begin = i - first < (kMT == 2 ? 1 : 2);  // the group's first tile of this item
                    if (!(ok = warp_wait(&S.p_ready[g], p_phase[g], failed))) break;
                    p_phase[g] ^= 1;
                    if ((kMT == 1 || g == 0) && !(ok = warp_wait(&S.v_full[stage], round & 1, failed))) break;
                    if (begin) {
                        if (uses[g] && !(ok = warp_wait(&S.o_free[g], (uses[g] - 1) & 1, failed))) break;
                        ++uses[g];
                    }
                    tc_after();
                    outputs(g, i, !begin);
                    if (kMT == 1 || g == 1) commit(&S.v_empty[stage]);
                    // the group's next S, in the place of the P that was just used (products are done in order)
                    const int ahead = i + (kMT == 2 ? 1 : 2);
                    if (ahead <= last) {
                        if ((kMT == 1 || g == 0) && !(ok = key_tile())) break;
                        scores(g, ahead);
                        if (kMT == 1 || g == 1) step_next();
                    }
                }
                if (++stage == M::kStages) stage = 0, ++round;
            }
            if (ok) commit(&S.q_empty);
            ++items;
            left -= n;
            advance(P, at);
        }
        // the last arrival that the tensor core owes this CTA's shared memory
        if (ok && items) warp_wait(&S.q_empty, (items - 1) & 1, failed);
        if (!ok) {  // products in flight are done before their operands and tensor memory go
            if (one) mma_commit(&S.drained);
            __syncwarp();
            bar_drain(&S.drained, 0, failed);
        }
    } else if (warp >= 4) {
        // ---- softmax: a thread per row
        const int g = (warp - 4) / 4, m = kMT == 2 ? g : 0;  // group, tile of rows
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t sp = tmem + g * 128 + lanes, op = tmem + 256 + g * 128 + lanes;
        constexpr int kStep = kMT == 2 ? 1 : 2;  // between tiles of a group
        int stage = 0;
        unsigned round = 0, tiles = 0, halves = 0;
        bool ok = true;
        const long long range_start = left;  // (a segment that begins here is the piece's first)
        const int node_in = row / P.G;
        const int head_in = row - node_in * P.G;
        while (left > 0 && ok) {
            const int h = at.item / P.row_items, rt = at.item - h * P.row_items;
            const int n = (int)(left < at.tiles - at.tile ? left : at.tiles - at.tile);
            const int node = (rt * kMT + m) * P.nodes_per_tile + node_in;
            const bool in_tile = node_in < P.nodes_per_tile && node < P.N;
            bool there = in_tile;
            float top = DSSD_NEG_INF, sum = 0.f;  // the maximum that weights refer to, in units of S
            uint32_t sees[4] = {0, 0, 0, 0};      // the row's node's ancestors and itself
            bool no_key = false;                  // there is no node `row`
            if (at.tile == 0 && (kMT == 2 || g == 0)) {
                signed char *const parent = S.parent[warp - 4];
                bool bad = false;
                __syncwarp();
                for (int j = lane; j < P.N; j += 32) {
                    int p = j - 1;
                    if (j > 0 && P.parents) p = ld_after(P.parents + at.b * (P.N - 1) + j - 1);
                    bad |= j > 0 && p >= j;
                    parent[j] = (signed char)(j == 0 ? 0 : p >= j ? -1 : max(p, -1));
                }
                __syncwarp();
                if (in_tile) {
                    int up = node;
                    while (up > 0) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (up >> 5 == k) sees[k] |= 1u << (up & 31);
                        up = parent[up];
                    }
                    there = up == 0;  // else there is no way to the root, and no node here
                    sees[0] |= 1u;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (!there) sees[k] = 0;
                }
                if (row < P.N) {
                    int up = row;
                    while (up > 0) up = parent[up];
                    no_key = up < 0;
                    bad |= no_key && parent[row] >= 0;
                }
                if (bad && h == 0 && rt == 0 && m == 0 && P.flags) atomicOr(P.flags + at.b, DSSD_CACHE_FLAG_BAD_NODE);
            }
            bool begin = true;
            for (int x = 0; x < n; ++x) {
                if (kStep == 1 || (x & 1) == g) {
                    const int i = at.tile + x;
                    if (!(ok = warp_wait(&S.s_full[g], tiles & 1, failed))) break;
                    tc_after();
                    const int valid = i == 0 ? P.N : min(kTile, at.ctx - (i - 1) * kTile);
                    const bool masked = i == 0 || valid < kTile;
                    // columns that do not count become -inf
                    auto mask = [&](uint32_t (&s)[32], int part) {
                        const int v = valid - part * 32;
                        const uint32_t a = (i == 0 ? sees[part] : 0xffffffffu) & (v >= 32 ? 0xffffffffu : v > 0 ? (1u << v) - 1u : 0u);
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (!((a >> k) & 1u)) s[k] = 0xff800000u;
                    };
                    auto most = [&](const uint32_t (&s)[32]) {
                        float h4[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) h4[k] = __uint_as_float(s[k]);
#pragma unroll
                        for (int k = 4; k < 32; ++k) h4[k & 3] = fmaxf(h4[k & 3], __uint_as_float(s[k]));
                        return fmaxf(fmaxf(h4[0], h4[1]), fmaxf(h4[2], h4[3]));
                    };
                    // All of S twice, 32 columns at a time and the next on their way: once for the maximum, once for the weights.  (In registers at
                    // once, with the warps' registers shared out anew for it, it took as long.)
                    uint32_t sa[32], sb[32], sc[32];
                    float hi;
                    tmem_ld32(sp, sa);
                    tmem_ld_wait(sa);
                    tmem_ld32(sp + 32, sb);
                    if (masked) mask(sa, 0);
                    hi = most(sa);
                    tmem_ld_wait(sb);
                    tmem_ld32(sp + 64, sa);
                    if (masked) mask(sb, 1);
                    hi = fmaxf(hi, most(sb));
                    tmem_ld_wait(sa);
                    tmem_ld32(sp + 96, sb);
                    if (masked) mask(sa, 2);
                    hi = fmaxf(hi, most(sa));
                    tmem_ld_wait(sb);
                    tmem_ld32(sp, sa);
                    if (masked) mask(sb, 3);
                    hi = fmaxf(hi, most(sb));
                    bool o_known = begin;
                    const bool raise = hi > top && (hi - top) * P.c > 8.f;  // (top = -inf: the first keys that count)
                    if (__any_sync(0xffffffffu, raise)) {
                        const float f = raise ? (top == DSSD_NEG_INF ? 0.f : ex2((top - hi) * P.c)) : 1.f;
                        if (raise) top = hi;
                        sum *= f;
                        if (!begin) {
                            if (!(ok = warp_wait(&S.o_done[g], (tiles - 1) & 1, failed))) break;
                            o_known = true;
                            tc_after();
#pragma unroll 1
                            for (int y = 0; y < DP; y += 32) {
                                uint32_t o[32];
                                tmem_ld32(op + y, o);
                                tmem_ld_wait(o);
#pragma unroll
                                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                                tmem_st32(op + y, o);
                            }
                        }
                    }
                    const float ref = top == DSSD_NEG_INF ? 0.f : -top * P.c;
                    const f32x2 c2 = pack2(P.c, P.c), ref2 = pack2(ref, ref);
                    f32x2 part_sum[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
                    auto weigh = [&](const uint32_t (&s)[32], int part) {
                        uint32_t p[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float u, v;
                            unpack2(fma2(pack2(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), c2, ref2), u, v);
                            u = ex2(u);
                            v = ex2(v);
                            part_sum[k & 1] = add2(part_sum[k & 1], pack2(u, v));
                            p[k] = pack<DT>(u, v);
                        }
                        tmem_st16(sp + part * 16, p);
                    };
                    // (P of 32 columns takes the place of 16 columns of S that have been read)
                    tmem_ld_wait(sa);
                    tmem_ld32(sp + 32, sc);
                    if (masked) mask(sa, 0);
                    weigh(sa, 0);
                    tmem_ld_wait(sc);
                    tmem_ld32(sp + 64, sa);
                    if (masked) mask(sc, 1);
                    weigh(sc, 1);
                    tmem_ld_wait(sa);
                    if (masked) mask(sa, 2);
                    weigh(sa, 2);
                    weigh(sb, 3);
                    float even, odd;
                    unpack2(add2(part_sum[0], part_sum[1]), even, odd);
                    sum += even + odd;
                    tmem_st_wait();
                    tc_before();
                    if (masked && (kMT == 1 || g == 0)) {
                        // what lies behind the last key, or belongs to no node, is made zero: its weight is, but zero times NaN is not
                        if (!(ok = warp_wait(&S.v_full[stage], round & 1, failed))) break;
                        const int upto = (valid + 15) / 16 * 16;
                        if (row < upto && (row >= valid || (i == 0 && no_key))) {
                            unsigned char *v = base + M::kKV + stage * 2 * M::kOperand + M::kOperand + row * 128;
                            for (int y = 0; y < kChunks; ++y)
                                for (int z = 0; z < 128; z += 16) *reinterpret_cast<uint4 *>(v + y * M::kChunk + z) = make_uint4(0, 0, 0, 0);
                        }
                        fence_async();
                    }
                    // The tile before has to be in O before this one's weights are given away: a barrier tells its last two phases
                    // apart and no more.  (It is, as a rule.)
                    if (!o_known && !(ok = warp_wait(&S.o_done[g], (tiles - 1) & 1, failed))) break;
                    bar_arrive(&S.p_ready[g]);
                    ++tiles;
                    begin = false;
                }
                if (++stage == M::kStages) stage = 0, ++round;
            }
            if (!ok) break;
            const bool mine = !begin;  // this group had keys of the item (with one tile of it the second had none)
            if (mine && !(ok = warp_wait(&S.o_done[g], (tiles - 1) & 1, failed))) break;
            tc_after();
            const bool two = kMT == 1 && n > 1;
            float w0 = 1.f, w1 = 0.f;
            if (two) {
                if (g == 1) {
                    S.other[row] = make_float2(top, sum);
                    tc_before();
                    bar_arrive(&S.half);
                } else {
                    if (!(ok = warp_wait(&S.half, halves & 1, failed))) break;
                    tc_after();
                    const float2 ml = S.other[row];
                    const float t2 = fmaxf(top, ml.x), r = t2 == DSSD_NEG_INF ? 0.f : t2;
                    w0 = ex2((top - r) * P.c);
                    w1 = ex2((ml.x - r) * P.c);
                    sum = sum * w0 + ml.y * w1;
                    top = t2;
                }
                ++halves;
            }
            if (kMT == 2 || g == 0) {
                const bool whole = n == at.tiles;
                const int head = h * P.G + head_in;
                const long long r = (2ll * blockIdx.x + (left == range_start ? 0 : 1)) * (kMT * 128) + m * 128 + row;
                const float inv = 1.f / sum;
                if (whole) w0 *= inv, w1 *= inv;
                unsigned short *to = static_cast<unsigned short *>(P.o) + at.b * P.o_b + node * P.o_n + head * P.o_h;
                float *part = P.part + r * DP;
#pragma unroll 1
                for (int x = 0; x < DP; x += 32) {
                    uint32_t o[32];
                    __syncwarp();
                    tmem_ld32(op + x, o);
                    if (two) {
                        uint32_t o1[32];
                        tmem_ld32(op + 128 + x, o1);
                        tmem_ld_wait(o);
                        tmem_ld_wait(o1);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * w0 + __uint_as_float(o1[k]) * w1);
                    } else {
                        tmem_ld_wait(o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * w0);
                    }
                    if (whole && there) {
#pragma unroll
                        for (int k = 0; k < 32; k += 8)
                            if (x + k < P.D)
                                *reinterpret_cast<uint4 *>(to + x + k) =
                                    make_uint4(pack<DT>(__uint_as_float(o[k]), __uint_as_float(o[k + 1])), pack<DT>(__uint_as_float(o[k + 2]), __uint_as_float(o[k + 3])),
                                               pack<DT>(__uint_as_float(o[k + 4]), __uint_as_float(o[k + 5])), pack<DT>(__uint_as_float(o[k + 6]), __uint_as_float(o[k + 7])));
                    } else if (!whole && in_tile) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) *reinterpret_cast<uint4 *>(part + x + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    }
                }
                if (whole && there && P.lse) P.lse[(at.b * P.N + node) * (P.Hkv * P.G) + head] = top * P.scale + logf(sum);
                // a row without a node is marked by the piece that has tile 0: no sum of weights is negative
                if (!whole && in_tile) P.part_ml[r] = make_float2(top * P.c, there ? sum : -1.f);
                tc_before();
                bar_arrive(&S.o_free[g]);
                if (two) bar_arrive(&S.o_free[1]);
            }
            left -= n;
            advance(P, at);
        }
        if (!ok) {
            __syncwarp();
            tmem_ld_wait_all();
            tmem_st_wait();
        }
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (S.failed) give_up(P, S.place, S.count, kMT * 128);
    if (warp == 1) tmem_free(tmem, 512);
}

// Joins the pieces of items that lie in several: a CTA per item and eight rows, a warp per row.
template <int DT, int DP, int kMT>
__global__ void __launch_bounds__(kThreads) tree_join_kernel(const __grid_constant__ Geometry P)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rows = P.nodes_per_tile * P.G;  // of a tile
    const int c = blockIdx.x % kMaxCtas, x = (int)(blockIdx.x / kMaxCtas) * kWarps + warp;
    const int m = x / rows, row = x - m * rows;
    pdl_wait();
    pdl_trigger();
    const uint4 raw = ld_row16(P.joins + c);
    const int4 join = make_int4((int)raw.x, (int)raw.y, (int)raw.z, (int)raw.w);
    if (join.x < 0) return;
    const long long b = join.x;
    const int h = join.y / P.row_items, rt = join.y - h * P.row_items;
    const int node = (rt * kMT + m) * P.nodes_per_tile + row / P.G;
    if (m >= kMT || node >= P.N) return;
    // the item's pieces: the second half (or all) of the piece before this one, then the beginnings of this one and those after it
    const int count = join.w - c + 2;
    auto slot_row = [&](int k) { return (long long)(k == 0 ? join.z : 2 * (c + k - 1)) * (kMT * 128) + m * 128 + row; };
    float top = DSSD_NEG_INF;
    bool none = false;
    for (int k = lane; k < count; k += 32) {
        const float2 ml = P.part_ml[slot_row(k)];
        none |= ml.y < 0.f;
        top = fmaxf(top, ml.x);
    }
    if (__any_sync(0xffffffffu, none)) return;  // there is no node
    top = warp_max(top);
    const float ref = top == DSSD_NEG_INF ? 0.f : top;  // (no score above -inf: an empty sum)
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const bool mine = lane * 4 < DP;
#pragma unroll 4
    for (int k = 0; k < count; ++k) {
        const long long r = slot_row(k);
        const float2 ml = P.part_ml[r];
        const float w = ex2(ml.x - ref);
        sum += w * ml.y;
        if (mine) {
            const float4 v = *reinterpret_cast<const float4 *>(P.part + r * DP + lane * 4);
            o[0] += w * v.x, o[1] += w * v.y, o[2] += w * v.z, o[3] += w * v.w;
        }
    }
    const float inv = 1.f / sum;
    const int hq = h * P.G + row % P.G;
    if (lane * 4 < P.D) {
        unsigned short *to = static_cast<unsigned short *>(P.o) + b * P.o_b + node * P.o_n + hq * P.o_h + lane * 4;
        *reinterpret_cast<uint2 *>(to) = make_uint2(pack<DT>(o[0] * inv, o[1] * inv), pack<DT>(o[2] * inv, o[3] * inv));
    }
    // lse = ln 2 * log2 of the sum over all weights
    if (lane == 0 && P.lse) P.lse[(b * P.N + node) * (P.Hkv * P.G) + hq] = top * 0.693147180559945309f + logf(sum);
}

typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                           CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A map of 16-bit values: sizes from the innermost dimension on, strides (in elements) of the others, the box that a copy takes
template <int kDims>
bool encode(CUtensorMap *map, int dtype, const void *at, const int64_t (&size)[kDims], const int64_t (&stride)[kDims - 1], const int (&box)[kDims])
{
    static const Encode fn = driver_call<Encode>("cuTensorMapEncodeTiled");
    if (!fn) return false;
    cuuint64_t sizes[kDims], strides[kDims - 1];
    cuuint32_t boxes[kDims], ones[kDims];
    for (int i = 0; i < kDims; ++i) {
        sizes[i] = (cuuint64_t)size[i];
        boxes[i] = (cuuint32_t)box[i];
        ones[i] = 1;
        // (the stride of a dimension of one entry is never used, but has to be a stride)
        if (i) strides[i - 1] = size[i] > 1 ? (cuuint64_t)stride[i - 1] * 2 : 16;
    }
    return fn(map, dtype == DSSD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, kDims, const_cast<void *>(at), sizes, strides, boxes, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DT, int DP, int kMT>
cudaError_t launch_as(const Geometry &P, unsigned grid, unsigned join_grid, cudaStream_t stream)
{
    typedef Smem<DP, kMT> M;
    static PerContext allowed;
    const int ok = allowed.get([] {
        return (int)(cudaFuncSetAttribute(tree_attention_kernel<DT, DP, kMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)M::kBytes) == cudaSuccess);
    });
    if (!ok) {
        const cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? cudaErrorInvalidConfiguration : e;
    }
    const cudaError_t e = launch_pdl(tree_attention_kernel<DT, DP, kMT>, grid, kAttend, stream, P, M::kBytes);
    return e == cudaSuccess ? launch_pdl(tree_join_kernel<DT, DP, kMT>, join_grid, kThreads, stream, P) : e;
}

// values of a piece's row in the workspace, rows of a piece
int padded(int D) { return D <= 64 ? 64 : 128; }
int rows_of(int N, int Hq, int Hkv)
{
    const int per = 128 / (Hq / Hkv);
    return N <= per ? 128 : 256;
}

}  // namespace

size_t tree_attention_workspace(int B, int N, int Hq, int Hkv, int D)
{
    (void)B, (void)Hkv;
    // (no less for fewer key heads: rows by the query heads, of which each key head has a part)
    const size_t rows = (long long)N * Hq <= 64 ? 128 : 256;
    return 2 * (size_t)kMaxCtas * rows * ((size_t)padded(D) * 4 + 8) + (kMaxCtas * sizeof(int4) + 255) / 256 * 256;
}

cudaError_t tree_attention_launch(TreeAttentionParams &P, int dtype, void *workspace, cudaStream_t stream)
{
    Geometry g;
    const int G = P.Hq / P.Hkv, per = 128 / G;
    const int rows = rows_of(P.N, P.Hq, P.Hkv), mt = rows / 128;
    int box = P.page_size, r = 128;
    while (r) {
        const int k = box % r;
        box = r;
        r = k;
    }
    const bool none = P.num_pages == 0;
    const int64_t pages = none ? 1 : P.num_pages, page = none ? 1 : P.page_size;
    const void *kc = none ? P.k_new : P.k_cache, *vc = none ? P.v_new : P.v_cache;
    bool ok = encode<5>(&g.q, dtype, P.q, {P.D, G, P.Hkv, P.N, P.B}, {P.q_h, G * P.q_h, P.q_n, P.q_b}, {64, G, 1, per, 1});
    ok = ok && encode<4>(&g.k_new, dtype, P.k_new, {P.D, P.Hkv, P.N, P.B}, {P.new_h, P.new_n, P.new_b}, {64, 1, P.N, 1});
    ok = ok && encode<4>(&g.v_new, dtype, P.v_new, {P.D, P.Hkv, P.N, P.B}, {P.new_h, P.new_n, P.new_b}, {64, 1, P.N, 1});
    ok = ok && encode<4>(&g.k_cache, dtype, kc, {P.D, none ? 1 : P.Hkv, page, pages}, {P.cache_h, P.cache_t, P.cache_p}, {64, 1, box, 1});
    ok = ok && encode<4>(&g.v_cache, dtype, vc, {P.D, none ? 1 : P.Hkv, page, pages}, {P.cache_h, P.cache_t, P.cache_p}, {64, 1, box, 1});
    if (!ok) return cudaErrorInvalidValue;
    g.block_table = P.block_table;
    g.table_stride = P.table_stride;
    g.max_pages = P.max_pages, g.num_pages = P.num_pages, g.page_size = P.page_size;
    g.box_log = 0;
    while (1 << g.box_log < box) ++g.box_log;
    g.tile_pages = kTile / P.page_size, g.tile_rest = kTile % P.page_size;
    g.ctx_len = P.ctx_len, g.parents = P.parents;
    g.B = P.B, g.N = P.N, g.Hkv = P.Hkv, g.G = G, g.D = P.D;
    g.nodes_per_tile = per;
    g.row_items = (P.N + mt * per - 1) / (mt * per);
    g.scale = P.scale;
    g.c = P.scale * 1.4426950408889634074f;
    g.o = P.o;
    g.o_b = P.o_b, g.o_n = P.o_n, g.o_h = P.o_h;
    g.lse = P.lse;
    g.flags = P.flags;
    g.wait_cycles = P.wait_cycles > 0 ? P.wait_cycles : kCycles;
    g.withhold = P.withhold;
    const int dp = padded(P.D);
    g.part = static_cast<float *>(workspace);
    g.part_ml = reinterpret_cast<float2 *>(g.part + 2 * (size_t)kMaxCtas * rows * dp);
    g.joins = reinterpret_cast<int4 *>(g.part_ml + 2 * (size_t)kMaxCtas * rows);
    const unsigned join = (unsigned)kMaxCtas * (unsigned)(((P.N < mt * per ? P.N : mt * per) * G + kWarps - 1) / kWarps);
    const bool bf = dtype == DSSD_BF16;
    if (dp == 64) {
        if (mt == 1) return bf ? launch_as<DSSD_BF16, 64, 1>(g, kMaxCtas, join, stream) : launch_as<DSSD_F16, 64, 1>(g, kMaxCtas, join, stream);
        return bf ? launch_as<DSSD_BF16, 64, 2>(g, kMaxCtas, join, stream) : launch_as<DSSD_F16, 64, 2>(g, kMaxCtas, join, stream);
    }
    if (mt == 1) return bf ? launch_as<DSSD_BF16, 128, 1>(g, kMaxCtas, join, stream) : launch_as<DSSD_F16, 128, 1>(g, kMaxCtas, join, stream);
    return bf ? launch_as<DSSD_BF16, 128, 2>(g, kMaxCtas, join, stream) : launch_as<DSSD_F16, 128, 2>(g, kMaxCtas, join, stream);
}

}  // namespace dssd
