// Attention over the paged 8-bit cache for few query rows (wz_attend): up to 16
// rows (tokens x heads of the group) of a sequence and KV head, as in decoding.
//
// Bound by HBM: every code is read once, by TMA, and goes to the tensor cores as
// it is.  With few rows the tokens take the M side of the products:
//   S^T [128 tokens x N] = K [tokens x D] * (q1 | q2)^T        K: A, K-major
//   O^T [D x N]          = V^T [D x tokens] * (p1 | p2)^T      V: A, MN-major
// N = 2R columns: a query row and a row of weights are two e4m3 numbers each,
// hi and 32 times the rest, in two columns whose results are joined in fp32 (8
// significant bits and more; a query of bf16 is exact).  A thread then has one token
// and R rows, and no accumulator lanes stand idle.
// The weights of a tile are taken relative to the tile's own largest (weight x
// scale of V), so that their 8 bits never lose a tile whose weights are small
// beside another's; each tile's O^T is read back and added in fp32 registers.
//
// Work is the list of all tiles of all (sequence, KV head) items, item_cost more for
// each item's start and end, cut into one contiguous range per CTA, so that any
// mixture of lengths keeps every SM busy; a range finds its first item by a scan
// over the sequences' tile counts.  An item inside one range is finished there; the
// pieces of others are written unnormalised, and attend_join_kernel adds them in
// order.  Where the page table has room for kWholeTiles tiles a sequence at most,
// CTAs take whole items and nothing is joined: the second kernel and the pieces'
// way through memory take longer than the tiles that they would spread.
//   warps 0-3  weights: thread = token of S^T, channel of O^T
//   warp 4     TMA producer: K and V tiles of 16 KB in one ring
//   warp 5     TMEM allocation, MMA issuer (one thread)
// One query over 200,003 slots of 4 heads x 128 takes 40 us: 205 MB at 6.9 TB/s between
// the first copies' arrival (4 us) and the median CTA's end (33 us), then the slowest
// SMs' tails and the join (7 us).  64 queries over up to 18,699 slots 78 us for 454 MB
// (95 with a join whose loads wait for one another; 105 beside that with tiles' rows in byte
// stores, scalars by every thread and a join that scanned the lengths again).
// Every wait is bounded; where one gives up the kernel sets a status bit, ends
// its copies, frees tensor memory and returns.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "wz_attend.cuh"

namespace wz {

namespace {

constexpr int kFThreads = 192;
constexpr int kFMaxStages = 6;
constexpr float kPTop = 8.f;   // log2 of a tile's largest weight

// Tiles of a sequence up to which items are not cut.  741 slots (six tiles) of 4 KV heads
// through the binding: 10.0 us in pieces, 11.8 whole; a tile more takes a CTA 1 us, the
// second kernel 4 us of the device's time and 2 of the host's.
constexpr int kWholeTiles = 4;

// A piece of an item, as the weight warps see it.
struct Piece {
    int b, h, t0, t1, tiles, kv, x0, rows, minlim, maxlim;
    long long first;     // the item's first tile in the list of units
};

template <int R>
struct FewShared {
    uint64_t full[kFMaxStages], empty[kFMaxStages];
    uint64_t s_full[2], p_ready[2], o_full[2], q_ready[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
    int b0;                      // first sequence of the range
    long long unit0;             // first unit of the range among its heads' units
    long long scan[8];
    alignas(16) float wmax[2][4][R];
    // by item: factors of the rows' logits, slots that a row sees
    alignas(16) float rowf[2][R];
    int lim[2][R];
    int token[2][R], head[2][R];
    Piece piece[2];
    // per warp and buffer: what a tile's sums and those before it are multiplied by
    alignas(16) float beta[4][2][R], alpha[4][2][R];
    float lsum[4][R];
    uint32_t nan_bits[64];       // two channels a word: tokens minlim + i that some rows see and whose V is NaN there
};

template <int R>
struct FewShape {
    static constexpr int N = 2 * R;
    static constexpr int kStages = R == 8 ? 4 : 5;
    static constexpr int kCtas = R == 8 ? 3 : 2;      // per SM
    static constexpr int kItemCost = R == 8 ? 2 : 5;  // tiles that an item's start and end take the time of
    static constexpr int kTmem = 4 * N;               // S and O, two buffers each
    static constexpr int kOpBytes = N * 128;          // q or p operand, two buffers each
    static constexpr size_t kSmem =
        1024 + (size_t)kStages * kATileBytes + 4 * (size_t)kOpBytes + sizeof(FewShared<R>);
    static_assert(kCtas * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
};

// Verdict of the four weight warps (barrier 1): true where all said so.
__device__ __forceinline__ bool all_agree(bool ok) {
    int r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.s32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, 128, p;\n\t"
        "selp.s32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((int)ok)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ int few_tiles(const AttendParams &p, int b) {
    const int2 n = attend_lengths(p, b);
    return n.x > 0 ? (n.y + kATile - 1) / kATile : -1;   // -1: nothing is asked
}

// Units of an item of this many tiles: those that cost time or, whole, an answer.
__device__ __forceinline__ int few_units(const AttendParams &p, int tiles) {
    return tiles > 0 || (tiles == 0 && p.whole) ? tiles + p.item_cost : 0;
}

// Sum of x over the threads before this one and over all, blockDim.x a multiple of 32.
__device__ __forceinline__ long long block_scan(long long x, long long *sums, long long *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long v = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xFFFFFFFFu, v, d);
        if (lane >= d) v += o;
    }
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < warps; ++w) {
        const long long s = sums[w];
        if (w < warp) before += s;
        all += s;
    }
    *total = all;
    return before + v - x;
}

// Ranges that the units are cut into: none of them empty, so that the pieces of an
// item lie in consecutive CTAs.
__device__ __forceinline__ int few_ranges(const AttendParams &p, long long total) {
    return (int)min((long long)p.ctas, total);
}
// The range that unit a lies in.
__device__ __forceinline__ int few_range_of(const AttendParams &p, long long total, long long a) {
    return (int)(((a + 1) * few_ranges(p, total) - 1) / total);
}

// A walk over a CTA's range, piece by piece: tiles t0 .. t1-1 of item (b, h).
struct Walk {
    int b, h, tiles, t0, t1;
    int unit;                    // first unit of the range in this item
    long long item0, left;       // first unit of the item in the list; units left, this piece's included
    bool any;

    __device__ __forceinline__ void start(const AttendParams &p, int b0, long long unit0, long long first, long long n) {
        left = n;
        any = n > 0;
        if (!any) return;
        b = b0;
        tiles = few_tiles(p, b);
        const int units = few_units(p, tiles);
        h = (int)(unit0 / units);
        unit = (int)(unit0 - (long long)h * units);
        item0 = first - unit;
        settle(p);
    }
    // The next piece; any: whether there is one.
    __device__ __forceinline__ void next(const AttendParams &p) {
        skip(p);
        settle(p);
    }

private:
    __device__ __forceinline__ void skip(const AttendParams &p) {
        const int units = few_units(p, tiles);
        left -= units - unit;
        item0 += units;
        unit = 0;
        if (left > 0 && ++h == p.heads) {
            h = 0;
            do tiles = few_tiles(p, ++b);
            while (few_units(p, tiles) == 0);   // left > 0: a later sequence has units
        }
    }
    // Leaves out what asks nothing of this CTA: starts of items whose tiles are the
    // next CTA's or, whole, items that begin in the CTA before.
    __device__ __forceinline__ void settle(const AttendParams &p) {
        for (; left > 0; skip(p)) {
            if (p.whole) {
                t0 = 0;
                t1 = tiles;
                if (unit == 0) return;
            } else {
                t0 = max(unit - p.item_cost, 0);
                t1 = max((int)min((long long)unit + left, (long long)tiles + p.item_cost) - p.item_cost, 0);
                if (t1 > t0) return;
            }
        }
        any = false;
    }
};

}  // namespace

// R: rows that the operands have room for (N = 16 columns is the least for M = 128); U: rows
// that a call can have.  A row alone (single tokens, no grouped heads) is its own variant: 16
// sequences of up to 4,098 slots, 16 heads x 64, take 24 us so and 27 with eight rows' weights.
template <int R, int U>
__global__ void __launch_bounds__(kFThreads, FewShape<R>::kCtas)
attend_few_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendParams p) {
    using Sh = FewShape<R>;
    constexpr int N = Sh::N;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *qs = ring + (size_t)Sh::kStages * kATileBytes;
    uint8_t *ps = qs + 2 * Sh::kOpBytes;
    FewShared<R> *S = reinterpret_cast<FewShared<R> *>(ps + 2 * Sh::kOpBytes);
    volatile int *abort_flag = &S->abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int s = 0; s < Sh::kStages; ++s) {
            ptx::mbar_init(&S->full[s], 1);
            ptx::mbar_init(&S->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&S->s_full[i], 1);
            ptx::mbar_init(&S->p_ready[i], 4);
            ptx::mbar_init(&S->o_full[i], 1);
            ptx::mbar_init(&S->q_ready[i], 4);
        }
        ptx::mbar_init(&S->drain, 1);
        S->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == 5) {
        ptx::tmem_alloc(&S->tmem_base, Sh::kTmem);
        ptx::tmem_relinquish();
    }
    if (tid == 128) {
        ptx::prefetch_tmap(&maps.k);
        ptx::prefetch_tmap(&maps.v);
    }
    pdl_wait();
    pdl_trigger();

    // this CTA's range of units
    const int per = (p.B + kFThreads - 1) / kFThreads;
    const int blo = min(p.B, tid * per), bhi = min(p.B, blo + per);
    long long mine = 0, total;
    for (int b = blo; b < bhi; ++b) {
        mine += few_units(p, few_tiles(p, b));
        if (blockIdx.x == 0 && !attend_lengths_sound(p, b)) kv_report(p.status);
    }
    const long long before = block_scan(mine, S->scan, &total);
    total *= p.heads;
    const int ranges = few_ranges(p, total);
    const bool busy = (int)blockIdx.x < ranges;
    const long long t0 = busy ? total * blockIdx.x / ranges : 0, t1 = busy ? total * (blockIdx.x + 1) / ranges : 0;
    if (busy && before * p.heads <= t0 && t0 < (before + mine) * p.heads) {
        long long at = before * p.heads;
        int b = blo;
        for (long long n; (n = (long long)few_units(p, few_tiles(p, b)) * p.heads) + at <= t0; ++b) at += n;
        S->b0 = b;
        S->unit0 = t0 - at;
    }
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;

    Walk w;
    w.start(p, S->b0, S->unit0, t0, t1 - t0);

    if (warp == 4) {
        // ---------------- TMA producer: lane = page of the tile ----------------
        const uint64_t pol = ptx::policy_evict_first();
        const int pages_tile = kATile / p.P, box = p.P * 128;
        const int absent = (int)(p.pages * p.heads);   // past the cache: zeros
        int seq = 0;                                   // copies issued: K, V, K, V, ..
        auto slab = [&](const Walk &u, int kv, int tile) {
            const int t = tile * kATile + (lane << p.shift);
            int pg = -1;
            if (lane < pages_tile && tile < u.t1 && t < kv) pg = attend_page(p, u.b, t);
            return pg < 0 ? absent : pg * p.heads + u.h;
        };
        int znext = absent;
        if (w.any) znext = slab(w, attend_lengths(p, w.b).y, w.t0);
        while (w.any && __all_sync(0xFFFFFFFFu, !*abort_flag)) {
            const Walk now = w;
            const int n = now.t1 - now.t0, kv = attend_lengths(p, now.b).y;
            bool ok = true;
            int zafter = absent;                       // of the next piece's first tile
            if (n == 0) {
                w.next(p);
                if (w.any) zafter = slab(w, attend_lengths(p, w.b).y, w.t0);
            }
            for (int i = 0; i < n && ok; ++i) {
                const int z = znext;
                if (i + 1 < n) znext = slab(now, kv, now.t0 + i + 1);
                for (int c = 0; c < 2; ++c, ++seq) {
                    const int st = seq % Sh::kStages;
                    ok = ptx::mbar_wait(&S->empty[st], ((uint32_t)(seq / Sh::kStages) & 1u) ^ 1u, wait_limit(p));
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) {
                        attend_fail(p, abort_flag);
                        break;
                    }
                    if (lane == 0) ptx::mbar_arrive_expect_tx(&S->full[st], kATileBytes);
                    __syncwarp();
                    if (lane < pages_tile)
                        ptx::tma_load_3d(ring + (size_t)st * kATileBytes + (size_t)lane * box, c ? &maps.v : &maps.k,
                                         &S->full[st], 0, 0, z, pol);
                }
                if (i == 0) {
                    w.next(p);
                    if (w.any) zafter = slab(w, attend_lengths(p, w.b).y, w.t0);
                }
            }
            if (!ok) break;
            znext = zafter;
        }
        for (int s = max(0, seq - Sh::kStages); s < seq; ++s)   // the copies have landed
            ptx::mbar_wait(&S->full[s % Sh::kStages], (uint32_t)(s / Sh::kStages) & 1u, kATimeoutNs);
    } else if (warp == 5) {
        if (ptx::elect_one()) {
            // ---------------- MMA issuer ----------------
            const uint32_t id_s = ptx::idesc_e4m3(128, N, false, false), id_o = ptx::idesc_e4m3(128, N, true, true);
            const uint32_t ring32 = ptx::smem_u32(ring);
            const uint64_t k_desc = ptx::smem_desc(ring32, 16, 1024, 2);
            const uint64_t v_desc = ptx::smem_desc(ring32, 16, 1024, 2);     // 8 tokens of 128 channels: 1 KB
            const uint64_t q_desc = ptx::smem_desc(ptx::smem_u32(qs), 16, 1024, 2);
            // weights: N bytes a token, 8 tokens after 8 tokens; 16 bytes without, 32 with a 32-byte swizzle
            const uint64_t p_desc = ptx::smem_desc(ptx::smem_u32(ps), 8 * N, 8 * N, N == 16 ? 0 : 6);
            const bool wide = p.D > 64;
            int k = 0, item = 0;                                             // tiles and items begun
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (ok && !ptx::mbar_wait(bar, parity, wait_limit(p))) {
                    attend_fail(p, abort_flag);
                    ok = false;
                }
                return ok;
            };
            for (; w.any && ok; ++item) {
                const int n = w.t1 - w.t0;
                if (!wait(&S->q_ready[item & 1], (uint32_t)(item >> 1) & 1u)) break;
                const uint64_t bq = q_desc + (uint64_t)(item & 1) * (Sh::kOpBytes >> 4);
                for (int i = 0; i <= n; ++i, ++k) {
                    if (i < n) {
                        const int seq = 2 * k, st = seq % Sh::kStages;
                        if (!wait(&S->full[st], (uint32_t)(seq / Sh::kStages) & 1u)) break;
                        ptx::tc_fence_after();
                        const uint64_t a = k_desc + (uint64_t)st * (kATileBytes >> 4);
    #pragma unroll
                        for (int j = 0; j < 4; ++j)   // K = 32 bytes along the swizzled row
                            if (j < 2 || wide)
                                ptx::mma_e4m3(tmem + (uint32_t)((k & 1) * N), a + (uint64_t)(2 * j), bq + (uint64_t)(2 * j),
                                              id_s, j > 0);
                        ptx::mma_commit(&S->empty[st]);
                        ptx::mma_commit(&S->s_full[k & 1]);
                    }
                    if (i == 0) w.next(p);   // its loads run beside the first weights
                    if (i > 0) {
                        const int j = k - 1, seq = 2 * j + 1, st = seq % Sh::kStages;
                        if (!wait(&S->p_ready[j & 1], (uint32_t)(j >> 1) & 1u) ||
                            !wait(&S->full[st], (uint32_t)(seq / Sh::kStages) & 1u))
                            break;
                        ptx::tc_fence_after();
                        const uint64_t a = v_desc + (uint64_t)st * (kATileBytes >> 4);
                        const uint64_t bp = p_desc + (uint64_t)(j & 1) * (Sh::kOpBytes >> 4);
    #pragma unroll
                        for (int s = 0; s < kATile / 32; ++s)   // 32 tokens: four groups of 8 rows of V
                            ptx::mma_e4m3(tmem + (uint32_t)((2 + (j & 1)) * N), a + (uint64_t)(s * (4096 >> 4)),
                                          bp + (uint64_t)(s * (32 * N >> 4)), id_o, s > 0);
                        ptx::mma_commit(&S->empty[st]);
                        ptx::mma_commit(&S->o_full[j & 1]);
                    }
                }
                --k;   // the last round began no tile
            }
            ptx::mma_commit(&S->drain);
            ptx::mbar_wait(&S->drain, 0, kATimeoutNs);
        }
    } else {
        // ---------------- weights ----------------
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16);
        int k = 0;
        bool ok = true;
        int item = 0;
        // Queries, limits and first scales of w's piece for item number `it`, in the buffers of its parity.
        auto page_of = [&](const Piece &u, int tile) {
            const int t = tile * kATile + tid;
            return tile < u.t1 && t < u.kv ? attend_page(p, u.b, t) : -1;
        };
        auto scales_of = [&](const Piece &u, int pg) {
            return pg < 0 ? make_float2(0.f, 0.f)
                          : make_float2(p.k_scale[(size_t)pg * p.heads + u.h], p.v_scale[(size_t)pg * p.heads + u.h]);
        };
        int pg = -1, pg_next = -1;   // pages of this thread's token: the next tile's, the one's after
        float2 sc;                   // scales of the next tile's
        auto prepare = [&](int it, int &pg, int &pg_next, float2 &sc) {
            Piece u;
            const int2 len = attend_lengths(p, w.b);
            u.b = w.b;
            u.h = w.h;
            u.t0 = w.t0;
            u.t1 = w.t1;
            u.tiles = w.tiles;
            u.first = w.item0 + p.item_cost;
            u.kv = len.y;
            u.x0 = p.cu[u.b];
            u.rows = min(len.x, p.most) * p.G;   // tokens past them, reported above, are left out
            // row c = token c / G, head c % G of the group
            uint2 raw[R / 4];
            int tok[R / 4];
#pragma unroll
            for (int j = 0; j < R / 4; ++j) {
                const int c = warp + 4 * j, i = c / p.G, hq = u.h * p.G + c - i * p.G;
                tok[j] = i;
                raw[j] = query_load(p, c < u.rows ? p.q + (size_t)(u.x0 + i) * p.q_stride + (size_t)hq * p.D : nullptr);
                if (lane == 0) {
                    S->token[it & 1][c] = u.x0 + i;
                    S->head[it & 1][c] = hq;
                }
            }
            pg = page_of(u, u.t0);
            pg_next = page_of(u, u.t0 + 1);
            sc = scales_of(u, pg);
            u.minlim = max(0, min(u.kv, attend_visible(p, 0, len.x, u.kv)));
            u.maxlim = u.rows > 0 ? max(0, min(u.kv, attend_visible(p, (u.rows - 1) / p.G, len.x, u.kv))) : 0;
            uint8_t *dst = qs + (size_t)(it & 1) * Sh::kOpBytes;
#pragma unroll
            for (int j = 0; j < R / 4; ++j) {
                const int c = warp + 4 * j;
                const QueryPiece v = query_piece<true>(raw[j]);
                *reinterpret_cast<uint32_t *>(dst + c * 128 + ((4 * lane) ^ ((c & 7) << 4))) = v.hi;
                *reinterpret_cast<uint32_t *>(dst + (R + c) * 128 + ((4 * lane) ^ (((R + c) & 7) << 4))) = v.lo;
                if (lane == 0) {
                    S->rowf[it & 1][c] = v.factor * p.scale2;
                    S->lim[it & 1][c] = c < u.rows ? max(0, min(u.kv, attend_visible(p, tok[j], len.x, u.kv))) : 0;
                }
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&S->q_ready[it & 1]);
            if (tid == 0) S->piece[it & 1] = u;
        };
        if (tid < 64) S->nan_bits[tid] = 0;
        if (w.any) prepare(0, pg, pg_next, sc);
        ok = all_agree(ok);   // the first item's factors and limits are there; a later one's before its tiles
        while (w.any && ok) {
            const Piece cur = S->piece[item & 1];
            int after_pg = -1, after_pg_next = -1;
            float2 after_sc = sc;
            bool more = false;
            const int n = cur.t1 - cur.t0, kv = cur.kv, rows = cur.rows, h = cur.h, x0 = cur.x0;
            const int minlim = cur.minlim, maxlim = cur.maxlim, ib = item & 1;
            const bool whole = n == cur.tiles;

            float acc[U], l[U], run = -INFINITY;   // run: lane c's maximum of row c so far
#pragma unroll
            for (int c = 0; c < U; ++c) acc[c] = l[c] = 0.f;

            auto read_output = [&](int kk) {   // O^T of tile kk into the sums
                ok = ptx::mbar_wait(&S->o_full[kk & 1], (uint32_t)(kk >> 1) & 1u, wait_limit(p)) && ok;
                ptx::tc_fence_after();
                uint32_t o[N / 16][16];
#pragma unroll
                for (int j = 0; j < N / 16; ++j)
                    ptx::tmem_ld_32x32b_x16(lane_base + (uint32_t)((2 + (kk & 1)) * N + 16 * j), o[j]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < N / 16; ++j) ptx::reg_fence16(o[j]);
#pragma unroll
                for (int c = 0; c < U; c += 4) {
                    const float4 al = *reinterpret_cast<const float4 *>(&S->alpha[warp][kk & 1][c]);
                    const float4 be = *reinterpret_cast<const float4 *>(&S->beta[warp][kk & 1][c]);
                    const float a4[4] = {al.x, al.y, al.z, al.w}, b4[4] = {be.x, be.y, be.z, be.w};
#pragma unroll
                    for (int u = 0; u < 4 && c + u < U; ++u) {
                        const int c1 = c + u, c2 = R + c + u;
                        const float sum = fmaf(__uint_as_float(o[c2 / 16][c2 % 16]), 1.f / kRest,
                                               __uint_as_float(o[c1 / 16][c1 % 16]));
                        acc[c1] = fmaf(acc[c1], a4[u], sum * b4[u]);
                    }
                }
            };

            // A thread's `ok` is its own from a wait to the next verdict: the loops are left on verdicts
            // alone, so that no warp is missing where the others wait for it.
            int i = 0;
            for (; i < n; ++i, ++k) {
                const int tile = cur.t0 + i, t = tile * kATile + tid;
                const float2 sc_now = sc;
                const int pg_now = pg;
                pg = pg_next;
                sc = scales_of(cur, pg);
                pg_next = page_of(cur, tile + 2);
                if (pg_now < 0 && t < kv) kv_report(p.status);

                ok = ptx::mbar_wait(&S->s_full[k & 1], (uint32_t)(k >> 1) & 1u, wait_limit(p)) && ok;
                ptx::tc_fence_after();
                float x[U];
                {
                    uint32_t s[N / 16][16];
#pragma unroll
                    for (int j = 0; j < N / 16; ++j)
                        ptx::tmem_ld_32x32b_x16(lane_base + (uint32_t)((k & 1) * N + 16 * j), s[j]);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < N / 16; ++j) ptx::reg_fence16(s[j]);
                    float rf[(U + 3) / 4 * 4];
#pragma unroll
                    for (int c = 0; c < U; c += 4)
                        *reinterpret_cast<float4 *>(&rf[c]) = *reinterpret_cast<const float4 *>(&S->rowf[ib][c]);
                    // base-2 logit + log2 of V's scale: the weight of a code of V
                    const float lv = pg_now < 0 ? -INFINITY : __log2f(sc_now.y);
#pragma unroll
                    for (int c = 0; c < U; ++c) {
                        const int c2 = R + c;
                        const float dot = fmaf(__uint_as_float(s[c2 / 16][c2 % 16]), 1.f / kRest,
                                               __uint_as_float(s[c / 16][c % 16]));
                        x[c] = fmaf(dot * sc_now.x, rf[c], lv);
                    }
                }
                if ((tile + 1) * kATile > minlim) {
#pragma unroll
                    for (int c = 0; c < U; ++c)
                        if (t >= S->lim[ib][c]) x[c] = -INFINITY;
                }
                float(*wm)[R] = S->wmax[k & 1];
#pragma unroll
                for (int c = 0; c < U; c += 4) {
                    float m[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) m[u] = c + u < U ? warp_max(x[(c + u) % U]) : -INFINITY;
                    if (lane == 0) *reinterpret_cast<float4 *>(&wm[warp][c]) = make_float4(m[0], m[1], m[2], m[3]);
                }
                ok = all_agree(ok);
                if (!ok) break;
                uint32_t codes[N / 4] = {};
#pragma unroll
                for (int c = 0; c < U; c += 4) {
                    float m4[4];
                    *reinterpret_cast<float4 *>(m4) = *reinterpret_cast<const float4 *>(&wm[0][c]);
#pragma unroll
                    for (int u = 1; u < 4; ++u) {
                        const float4 o = *reinterpret_cast<const float4 *>(&wm[u][c]);
                        m4[0] = fmaxf(m4[0], o.x);
                        m4[1] = fmaxf(m4[1], o.y);
                        m4[2] = fmaxf(m4[2], o.z);
                        m4[3] = fmaxf(m4[3], o.w);
                    }
                    uint32_t hi = 0, lo = 0;
#pragma unroll
                    for (int u = 0; u < 4 && c + u < U; u += 2) {
                        // relative to the tile's largest, which becomes 2^kPTop
#pragma unroll
                        for (int v = u; v < u + 2 && c + v < U; ++v)
                            x[c + v] = ex2(x[c + v] - ((m4[v] == -INFINITY ? 0.f : m4[v]) - kPTop));
                        // number and rest in f16, whose 11 bits hold both
                        const __half2 wt = __floats2half2_rn(x[c + u], c + u + 1 < U ? x[(c + u + 1) % U] : 0.f);
                        const uint32_t q = e4m3x2(wt);
                        const __half2 rest = __hfma2(half2_of_e4m3((uint16_t)q), __float2half2_rn(-kRest),
                                                     __hmul2(wt, __float2half2_rn(kRest)));
                        hi |= q << (8 * u);
                        lo |= e4m3x2(rest) << (8 * u);
                    }
                    codes[c / 4] = hi;
                    codes[(R + c) / 4] = lo;
                }
                uint8_t *pb = ps + (size_t)(k & 1) * Sh::kOpBytes + tid * N;
#pragma unroll
                for (int j = 0; j < N / 16; ++j)
                    *reinterpret_cast<uint4 *>(pb + 16 * (N == 16 ? 0 : j ^ ((tid >> 2) & 1))) =
                        make_uint4(codes[4 * j], codes[4 * j + 1], codes[4 * j + 2], codes[4 * j + 3]);
                if ((tile + 1) * kATile > minlim) {
                    // rows of V that a weight of 0 must not meet: past the sequence, or
                    // NaN where only some rows see the token
                    const int seq = 2 * k + 1, st = seq % Sh::kStages;
                    ok = ptx::mbar_wait(&S->full[st], (uint32_t)(seq / Sh::kStages) & 1u, wait_limit(p)) && ok;
                    uint4 *row = reinterpret_cast<uint4 *>(ring + (size_t)st * kATileBytes + (size_t)tid * 128);
                    if (t >= maxlim) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) row[j] = make_uint4(0, 0, 0, 0);
                    } else if (t >= minlim) {
                        for (int j = 0; j < 32; ++j) {
                            uint32_t *word = reinterpret_cast<uint32_t *>(row) + j;
                            const uint32_t v = *word, bad = __vcmpeq4(v & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                            if (bad) {
                                *word = v & ~bad;
                                const int ch = ((j >> 2) ^ (tid & 7)) * 16 + (j & 3) * 4;
                                for (int u = 0; u < 4; ++u)
                                    if ((bad >> (8 * u)) & 1u)
                                        atomicOr(&S->nan_bits[(ch + u) >> 1], 1u << (t - minlim + 16 * ((ch + u) & 1)));
                            }
                        }
                    }
                }
                ptx::tc_fence_before();
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&S->p_ready[k & 1]);
                // sums, while the products run
                if (lane < U) {
                    const float m = fmaxf(fmaxf(wm[0][lane], wm[1][lane]), fmaxf(wm[2][lane], wm[3][lane]));
                    const float top = fmaxf(run, m), to = top == -INFINITY ? 0.f : top;
                    S->alpha[warp][k & 1][lane] = ex2(run - to);
                    S->beta[warp][k & 1][lane] = ex2(m - to - kPTop);
                    run = top;
                }
                __syncwarp();
                const float inv_v = pg_now < 0 ? 0.f : __frcp_rn(sc_now.y);
#pragma unroll
                for (int c = 0; c < U; c += 4) {
                    const float4 al = *reinterpret_cast<const float4 *>(&S->alpha[warp][k & 1][c]);
                    const float4 be = *reinterpret_cast<const float4 *>(&S->beta[warp][k & 1][c]);
                    const float a4[4] = {al.x, al.y, al.z, al.w}, b4[4] = {be.x, be.y, be.z, be.w};
#pragma unroll
                    for (int u = 0; u < 4 && c + u < U; ++u)
                        l[c + u] = fmaf(l[c + u], a4[u], x[c + u] * inv_v * b4[u]);
                }
                if (i > 0) read_output(k - 1);
                if (i == 0) {   // the next item's first products follow this one's last
                    w.next(p);
                    more = w.any;
                    if (more) prepare(item + 1, after_pg, after_pg_next, after_sc);
                }
            }
            if (i < n) break;
            if (n > 0) {
                read_output(k - 1);
            } else {
                ok = all_agree(ok);   // the buffers are the last item's but one
                if (!ok) break;
                w.next(p);
                more = w.any;
                if (more) prepare(item + 1, after_pg, after_pg_next, after_sc);
            }
            // sums over the tokens: halves of the rows change lanes until a lane has one row
#pragma unroll
            for (int half = U / 2, d = 16; half; half >>= 1, d >>= 1) {
                const bool up = lane & d;
#pragma unroll
                for (int c = 0; c < half; ++c) {
                    const float give = up ? l[c] : l[half + c], keep = up ? l[half + c] : l[c];
                    l[c] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, d);
                }
            }
#pragma unroll
            for (int d = 16 / U; d; d >>= 1) l[0] += __shfl_xor_sync(0xFFFFFFFFu, l[0], d);
            if (lane % (32 / U) == 0) S->lsum[warp][lane / (32 / U)] = l[0];
            ok = all_agree(ok);
            if (!ok) break;
            const uint32_t nan_at = S->nan_bits[tid >> 1] >> (16 * (tid & 1)) & 0xFFFFu;
            const size_t slot = 2 * (size_t)blockIdx.x + (cur.t0 == 0 ? 1 : 0);
            // lane c: the sum of row c, its reciprocal for all lanes
            const int cl = lane % U;
            const float L = (S->lsum[0][cl] + S->lsum[1][cl]) + (S->lsum[2][cl] + S->lsum[3][cl]);
            const float inv_mine = L == 0.f ? 0.f : 1.f / L;
            if (warp == 0 && lane < rows) {
                if (!whole)
                    p.ml[slot * R + lane] = make_float2(run, L);
                else if (p.lse)
                    p.lse[(size_t)S->token[ib][lane] * p.Hq + S->head[ib][lane]] =
                        L == 0.f ? -INFINITY : (run + log2f(L)) * kLn2;
            }
#pragma unroll
            for (int c = 0; c < U; ++c) {
                const float inv = __shfl_sync(0xFFFFFFFFu, inv_mine, c);
                if (c >= rows) continue;
                float o = acc[c];
                if (nan_at) {   // tokens minlim .. lim - 1 are those that this row sees and some other does not
                    const uint32_t sees = (1u << min(max(S->lim[ib][c] - minlim, 0), 16)) - 1u;
                    if (nan_at & sees) o = NAN;
                }
                if (whole) {
                    const int x = S->token[ib][c];
                    if (tid < p.D && wz_in_range(p.status, x < p.T))
                        p.out[(size_t)x * p.out_stride + (size_t)S->head[ib][c] * p.D + tid] =
                            __float2bfloat16_rn(o * inv);
                } else if (wz_in_range(p.status, slot < 2 * (size_t)p.ctas)) {
                    p.part[(slot * R + c) * 128 + tid] = o;
                }
            }
            if (tid == 0 && cur.t0 == 0 && !p.whole) {
                // where the join finds the item's pieces: this CTA and those after it
                const int pieces = whole ? 1 : few_range_of(p, total, cur.first + cur.tiles - 1) - (int)blockIdx.x + 1;
                p.spans[(size_t)x0 * p.heads + h] = make_int2((int)blockIdx.x, pieces);
            }
            __syncwarp();   // both channels of a word are this warp's
            if (nan_at) S->nan_bits[tid >> 1] = 0;
            pg = after_pg;
            pg_next = after_pg_next;
            sc = after_sc;
            ++item;
            if (!more) break;
        }
        if (!ok) attend_fail(p, abort_flag);
    }
    __syncthreads();
    if (warp == 5) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, Sh::kTmem);
    }
}

// Adds the pieces of the items that several CTAs hold, and answers the rows of
// sequences without slots.  A warp per row (BY_ROW; a block per item) where items have
// few pieces, else a block per row, whose warps take every sixteenth piece each.
template <int R, bool BY_ROW>
__global__ void __launch_bounds__(512) attend_join_kernel(const __grid_constant__ AttendParams p) {
    constexpr int kWarps = BY_ROW ? R : 16, kBatch = 8;   // kBatch: pieces whose loads are in flight
    __shared__ float sums[kWarps][128];
    __shared__ float2 ml[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = (int)blockIdx.x / p.heads, h = (int)blockIdx.x - b * p.heads;
    // lengths are older than the kernel before, which started this one after its own wait
    const int2 len = attend_lengths(p, b);
    const int x0 = p.cu[b];
    pdl_wait();
    pdl_trigger();
    // Those that the kernel before formed.  (Where the compiler sees that they are R at most it
    // gives the loads of a batch of pieces 42 registers instead of 63 and one waits for the
    // other: 64 ragged queries 97 us instead of 78, 741 slots 9.3 instead of 8.7.)
    const int rows = min(len.x, p.most) * p.G;
    if (rows == 0) return;
    const int2 span = len.y > 0 ? p.spans[(size_t)x0 * p.heads + h] : make_int2(0, 0);
    if (span.y == 1) return;   // one CTA had the whole item
    // never written: the kernel before gave up (any numbers, so no sum of them)
    if (span.x < 0 || span.y < 0 || span.x > p.ctas - span.y) return;
    for (int c = BY_ROW ? warp : (int)blockIdx.y; c < rows; c += R) {
        float m = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        constexpr int kStep = BY_ROW ? 1 : kWarps;
        for (int j0 = BY_ROW ? 0 : warp; j0 < span.y; j0 += kBatch * kStep) {
            float2 pm[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int j = j0 + u * kStep;
                // the first piece is its CTA's last item, the others are their CTAs' first
                const size_t at = (2 * (size_t)(span.x + j) + (j == 0 ? 1 : 0)) * R + c;
                pm[u] = j < span.y ? p.ml[at] : make_float2(-INFINITY, 0.f);
                v[u] = j < span.y ? *reinterpret_cast<const float4 *>(p.part + at * 128 + 4 * lane)
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) top = fmaxf(top, pm[u].x);
            const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(m - ref);
            m = top;
            L *= f0;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] *= f0;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const float f = ex2(pm[u].x - ref);
                L = fmaf(pm[u].y, f, L);
                o[0] = fmaf(v[u].x, f, o[0]);
                o[1] = fmaf(v[u].y, f, o[1]);
                o[2] = fmaf(v[u].z, f, o[2]);
                o[3] = fmaf(v[u].w, f, o[3]);
            }
        }
        if (!BY_ROW) {
            *reinterpret_cast<float4 *>(&sums[warp][4 * lane]) = make_float4(o[0], o[1], o[2], o[3]);
            if (lane == 0) ml[warp] = make_float2(m, L);
            __syncthreads();
            if (warp != 0) return;
            m = -INFINITY;
            for (int k = 0; k < kWarps; ++k) m = fmaxf(m, ml[k].x);
            const float ref = m == -INFINITY ? 0.f : m;
            L = o[0] = o[1] = o[2] = o[3] = 0.f;
            for (int k = 0; k < kWarps; ++k) {
                const float f = ex2(ml[k].x - ref);
                const float4 s = *reinterpret_cast<const float4 *>(&sums[k][4 * lane]);
                L = fmaf(ml[k].y, f, L);
                o[0] = fmaf(s.x, f, o[0]);
                o[1] = fmaf(s.y, f, o[1]);
                o[2] = fmaf(s.z, f, o[2]);
                o[3] = fmaf(s.w, f, o[3]);
            }
        }
        const int i = c / p.G, hq = h * p.G + c - i * p.G;
        const size_t x = (size_t)(x0 + i);
        const float inv = L == 0.f ? 0.f : 1.f / L;
        if (4 * lane < p.D && wz_in_range(p.status, x < (size_t)p.T)) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(o[0] * inv, o[1] * inv);
            const __nv_bfloat162 d = __floats2bfloat162_rn(o[2] * inv, o[3] * inv);
            *reinterpret_cast<uint2 *>(p.out + x * p.out_stride + (size_t)hq * p.D + 4 * lane) =
                make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&d));
        }
        if (lane == 0 && p.lse) p.lse[x * p.Hq + hq] = L == 0.f ? -INFINITY : (m + log2f(L)) * kLn2;
    }
}

namespace {

template <int R, int U>
cudaError_t launch_few(const AttendMaps &maps, AttendParams p, int max_new, int sms, cudaStream_t s) {
    using Sh = FewShape<R>;
    cudaError_t e = allow_smem((const void *)attend_few_kernel<R, U>, Sh::kSmem);
    if (e != cudaSuccess) return e;
    const int64_t items = (int64_t)p.B * p.heads;
    const int64_t tiles = ((int64_t)p.max_pages * p.P + kATile - 1) / kATile;
    p.whole = tiles <= kWholeTiles;
    p.most = U / p.G;
    // 0: a CTA for each tile; whole items have at least the unit that an empty one is found by
    p.item_cost = p.whole || items * tiles > (int64_t)sms * Sh::kCtas ? Sh::kItemCost : 0;
    // no more CTAs than items or tiles there can be
    p.ctas = (int)std::min<int64_t>({(int64_t)sms * Sh::kCtas, kFewSlots / 2, p.whole ? items : items * tiles});
    void *args[] = {const_cast<AttendMaps *>(&maps), &p};
    e = launch_kernel((const void *)attend_few_kernel<R, U>, dim3(p.ctas), dim3(kFThreads), Sh::kSmem, s, args, true);
    if (e != cudaSuccess || p.whole) return e;
    void *jargs[] = {&p};
    const bool by_row = p.ctas <= 8 * items;   // a batch of pieces to an item, if all are alike
    return launch_kernel(by_row ? (const void *)attend_join_kernel<R, true> : (const void *)attend_join_kernel<R, false>,
                         dim3((unsigned)items, by_row ? 1 : (unsigned)std::min<int64_t>((int64_t)max_new * p.G, R)),
                         dim3(by_row ? 32 * R : 512), 0, s, jargs, true);
}

}  // namespace

cudaError_t launch_attend_few(const AttendMaps &maps, const AttendParams &p, int max_new, int sms, cudaStream_t s) {
    const int64_t rows = (int64_t)max_new * p.G;
    return rows <= 1   ? launch_few<8, 1>(maps, p, max_new, sms, s)
           : rows <= 8 ? launch_few<8, 8>(maps, p, max_new, sms, s)
                       : launch_few<16, 16>(maps, p, max_new, sms, s);
}

}  // namespace wz
