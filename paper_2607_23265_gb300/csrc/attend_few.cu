// Attention over the paged 8-bit cache for few query rows (wz_attend): up to 16
// rows (tokens x heads of the group) of a sequence and KV head, as in decoding.
//
// Bound by HBM: every code is read once, by TMA, and goes to the tensor cores as
// it is.  With few rows the tokens take the M side of the products:
//   S^T [128 tokens x N] = K [tokens x D] * (q1 | q2)^T        K: A, K-major
//   O^T [D x N]          = V^T [D x tokens] * (p1 | p2)^T      V: A, MN-major
// N = 2R columns: a query row and a row of weights are two e4m3 numbers each,
// hi and 32 times the rest, in two columns whose results are joined in fp32 (8
// significant bits and more; a query of bf16 is exact).  A thread then has one token and R rows:
// no row waits for 128 lanes of idle accumulators.
// The weights of a tile are taken relative to the tile's own largest (weight x
// scale of V), so that their 8 bits never lose a tile whose weights are small
// beside another's; each tile's O^T is read back and added in fp32 registers.
//
// Work is the list of all tiles of all (sequence, KV head) items, cut into one
// contiguous range per CTA, so that any mixture of lengths keeps every SM busy;
// a range finds its first item by a scan over the sequences' tile counts.  An
// item inside one range is finished there; the pieces of others are written
// unnormalised, and attend_join_kernel adds them in order.
//   warps 0-3  weights: thread = token of S^T, channel of O^T
//   warp 4     TMA producer: K and V tiles of 16 KB in one ring
//   warp 5     TMEM allocation, MMA issuer (one thread)
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
constexpr float kPScale = 256.f;   // a tile's largest weight

template <int R>
struct FewShared {
    uint64_t full[kFMaxStages], empty[kFMaxStages];
    uint64_t s_full[2], p_ready[2], o_full[2];
    uint64_t q_ready, drain;
    uint32_t tmem_base;
    int abort;
    int b0;                      // first sequence of the range
    long long tile0;             // first tile of the range among the tiles of its heads
    long long scan[8];
    float wmax[2][4][R];
    float rowf[R];
    int lim[R];
    float lsum[4][R];
    int nan_min[128];            // per channel: the first token that some rows see and whose V is NaN there
};

template <int R>
struct FewShape {
    static constexpr int N = 2 * R;
    static constexpr int kStages = R == 8 ? 4 : 5;
    static constexpr int kCtas = R == 8 ? 3 : 2;      // per SM
    static constexpr int kTmem = 4 * N;               // S and O, two buffers each
    static constexpr int kOpBytes = N * 128;          // q or p operand
    static constexpr size_t kSmem =
        1024 + (size_t)kStages * kATileBytes + 3 * (size_t)kOpBytes + sizeof(FewShared<R>);
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
    return n.x > 0 ? (n.y + kATile - 1) / kATile : 0;
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

// Ranges that the tiles are cut into: none of them empty, so that the pieces of an
// item lie in consecutive CTAs.
__device__ __forceinline__ int few_ranges(const AttendParams &p, long long total) {
    return (int)min((long long)p.ctas, total);
}
__device__ __forceinline__ void few_range(const AttendParams &p, long long total, int cta, long long *t0,
                                          long long *t1) {
    const int n = few_ranges(p, total);
    *t0 = cta < n ? total * cta / n : 0;
    *t1 = cta < n ? total * (cta + 1) / n : 0;
}
// The range that tile a lies in.
__device__ __forceinline__ int few_range_of(const AttendParams &p, long long total, long long a) {
    return (int)(((a + 1) * few_ranges(p, total) - 1) / total);
}

// A walk over the tiles of a CTA's range, item by item.
struct Walk {
    int b, h, tile, tiles;       // this item's next tile and its tiles
    long long left;              // tiles left in the range
    __device__ __forceinline__ void start(const AttendParams &p, int b0, long long tile0, long long n) {
        b = b0;
        left = n;
        tiles = n > 0 ? few_tiles(p, b) : 1;
        h = (int)(tile0 / tiles);
        tile = (int)(tile0 - (long long)h * tiles);
    }
    __device__ __forceinline__ int count() const { return (int)min((long long)(tiles - tile), left); }
    __device__ __forceinline__ void next(const AttendParams &p) {
        left -= count();
        tile = 0;
        if (left > 0 && ++h == p.heads) {
            h = 0;
            do tiles = few_tiles(p, ++b);
            while (tiles == 0);   // left > 0: a later sequence has tiles
        }
    }
};

}  // namespace

template <int R>
__global__ void __launch_bounds__(kFThreads, FewShape<R>::kCtas)
attend_few_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendParams p) {
    using Sh = FewShape<R>;
    constexpr int N = Sh::N;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *qs = ring + (size_t)Sh::kStages * kATileBytes;
    uint8_t *ps = qs + Sh::kOpBytes;
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
        }
        ptx::mbar_init(&S->q_ready, 1);
        ptx::mbar_init(&S->drain, 1);
        S->abort = 0;
        S->b0 = 0;
        S->tile0 = 0;
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

    // this CTA's range of tiles
    const int per = (p.B + kFThreads - 1) / kFThreads;
    const int blo = min(p.B, tid * per), bhi = min(p.B, blo + per);
    long long mine = 0, total;
    for (int b = blo; b < bhi; ++b) {
        mine += few_tiles(p, b);
        if (blockIdx.x == 0 && !attend_lengths_sound(p, b)) kv_report(p.status);
    }
    const long long before = block_scan(mine, S->scan, &total);
    total *= p.heads;
    long long t0, t1;
    few_range(p, total, (int)blockIdx.x, &t0, &t1);
    if (t1 > t0 && before * p.heads <= t0 && t0 < (before + mine) * p.heads) {
        long long at = before * p.heads;
        int b = blo;
        for (long long n; (n = (long long)few_tiles(p, b) * p.heads) + at <= t0; ++b) at += n;
        S->b0 = b;
        S->tile0 = t0 - at;
    }
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;

    Walk w;
    w.start(p, S->b0, S->tile0, t1 - t0);

    if (warp == 4) {
        // ---------------- TMA producer: lane = page of the tile ----------------
        const uint64_t pol = ptx::policy_evict_first();
        const int pages_tile = kATile / p.P, box = p.P * 128;
        const int absent = (int)(p.pages * p.heads);   // past the cache: zeros
        int seq = 0;                                   // copies issued: K, V, K, V, ..
        for (; w.left > 0 && !*abort_flag; w.next(p)) {
            const int kv = attend_lengths(p, w.b).y;
            bool ok = true;
            const int n = w.count();
            int z = absent, znext = absent;
            auto slab = [&](int tile) {
                const int t = tile * kATile + lane * p.P;
                int pg = -1;
                if (lane < pages_tile && t < kv) pg = attend_page(p, w.b, t);
                return pg < 0 ? absent : pg * p.heads + w.h;
            };
            znext = slab(w.tile);
            for (int i = 0; i < n && ok; ++i) {
                z = znext;
                if (i + 1 < n) znext = slab(w.tile + i + 1);
                for (int c = 0; c < 2; ++c, ++seq) {
                    const int st = seq % Sh::kStages;
                    ok = ptx::mbar_wait(&S->empty[st], ((uint32_t)(seq / Sh::kStages) & 1u) ^ 1u, kATimeoutNs);
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
            }
            if (!ok) break;
        }
        for (int s = max(0, seq - Sh::kStages); s < seq; ++s)   // the copies have landed
            ptx::mbar_wait(&S->full[s % Sh::kStages], (uint32_t)(s / Sh::kStages) & 1u, kATimeoutNs);
    } else if (warp == 5) {
        if (lane == 0) {
            // ---------------- MMA issuer ----------------
            const uint32_t id_s = ptx::idesc_e4m3(128, N, false, false), id_o = ptx::idesc_e4m3(128, N, true, false);
            const uint32_t ring32 = ptx::smem_u32(ring);
            const uint64_t k_desc = ptx::smem_desc(ring32, 16, 1024, 2);
            const uint64_t v_desc = ptx::smem_desc(ring32, 16, 1024, 2);     // 8 tokens of 128 channels: 1 KB
            const uint64_t q_desc = ptx::smem_desc(ptx::smem_u32(qs), 16, 1024, 2);
            const uint64_t p_desc = ptx::smem_desc(ptx::smem_u32(ps), 16, 1024, 2);
            const int ksteps = (p.D + 31) >> 5;
            int k = 0, item = 0;                                             // tiles and items begun
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (ok && !ptx::mbar_wait(bar, parity, kATimeoutNs)) {
                    attend_fail(p, abort_flag);
                    ok = false;
                }
                return ok;
            };
            for (; w.left > 0 && ok && !*abort_flag; w.next(p), ++item) {
                const int n = w.count();
                if (!wait(&S->q_ready, (uint32_t)item & 1u)) break;
                for (int i = 0; i <= n; ++i, ++k) {
                    if (i < n) {
                        const int seq = 2 * k, st = seq % Sh::kStages;
                        if (!wait(&S->full[st], (uint32_t)(seq / Sh::kStages) & 1u)) break;
                        ptx::tc_fence_after();
                        const uint64_t a = k_desc + (uint64_t)st * (kATileBytes >> 4);
                        for (int j = 0; j < ksteps; ++j)   // K = 32 bytes along the swizzled row
                            ptx::mma_e4m3(tmem + (uint32_t)((k & 1) * N), a + (uint64_t)(2 * j),
                                          q_desc + (uint64_t)(2 * j), id_s, j > 0);
                        ptx::mma_commit(&S->empty[st]);
                        ptx::mma_commit(&S->s_full[k & 1]);
                    }
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
                                          bp + (uint64_t)(2 * s), id_o, s > 0);
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
        for (; w.left > 0; w.next(p)) {
            const int2 len = attend_lengths(p, w.b);
            const int kv = len.y, n = w.count(), h = w.h, b = w.b;
            const int x0 = p.cu[b];
            int rows = len.x * p.G;
            if (rows > R) {   // more tokens than max_new
                kv_report(p.status);
                rows = R / p.G * p.G;
            }
            const int ntok = rows / p.G;   // tokens that are answered
            // the item's queries: row c = token c / G, head c % G of the group
            for (int c = warp; c < R; c += 4) {
                const int i = c / p.G, g = c - i * p.G;
                const QueryPiece v = query_piece<true>(query_load(
                    p, c < rows ? p.q + (size_t)(x0 + i) * p.q_stride + (size_t)(h * p.G + g) * p.D : nullptr));
                *reinterpret_cast<uint32_t *>(qs + c * 128 + ((4 * lane) ^ ((c & 7) << 4))) = v.hi;
                *reinterpret_cast<uint32_t *>(qs + (R + c) * 128 + ((4 * lane) ^ (((R + c) & 7) << 4))) = v.lo;
                if (lane == 0) {
                    S->rowf[c] = v.factor * p.scale2;
                    S->lim[c] = c < rows ? min(kv, attend_visible(p, i, len.x, kv)) : 0;
                }
            }
            S->nan_min[tid] = INT32_MAX;
            ptx::fence_proxy_async_smem();
            ok = all_agree(ok);
            if (!ok) break;
            if (tid == 0) ptx::mbar_arrive(&S->q_ready);
            int minlim = kv, maxlim = 0;
            for (int c = 0; c < rows; ++c) {
                minlim = min(minlim, S->lim[c]);
                maxlim = max(maxlim, S->lim[c]);
            }

            float acc[R], l[R], run[R], alpha[R], beta[R];
#pragma unroll
            for (int c = 0; c < R; ++c) acc[c] = l[c] = 0.f, run[c] = -INFINITY;

            // scales of this thread's token: loaded a tile ahead, its page two
            auto page_of = [&](int tile) {
                const int t = tile * kATile + tid;
                return t < kv ? attend_page(p, b, t) : -1;
            };
            auto scales_of = [&](int pg) {
                return pg < 0 ? make_float2(0.f, 0.f)
                              : make_float2(p.k_scale[(size_t)pg * p.heads + h], p.v_scale[(size_t)pg * p.heads + h]);
            };
            int pg = page_of(w.tile), pg_next = n > 1 ? page_of(w.tile + 1) : -1;
            float2 sc = scales_of(pg);

            auto read_output = [&](int kk) {   // O^T of tile kk into the sums
                ok = ptx::mbar_wait(&S->o_full[kk & 1], (uint32_t)(kk >> 1) & 1u, kATimeoutNs) && ok;
                ptx::tc_fence_after();
                uint32_t o[N / 16][16];
#pragma unroll
                for (int j = 0; j < N / 16; ++j)
                    ptx::tmem_ld_32x32b_x16(lane_base + (uint32_t)((2 + (kk & 1)) * N + 16 * j), o[j]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < N / 16; ++j) ptx::reg_fence16(o[j]);
#pragma unroll
                for (int c = 0; c < R; ++c) {
                    const int c2 = R + c;
                    const float sum = fmaf(__uint_as_float(o[c2 / 16][c2 % 16]), 1.f / kRest,
                                           __uint_as_float(o[c / 16][c % 16]));
                    acc[c] = fmaf(acc[c], alpha[c], sum * beta[c]);
                }
            };

            for (int i = 0; i < n; ++i, ++k) {
                const int tile = w.tile + i, t = tile * kATile + tid;
                const float2 sc_now = sc;
                const int pg_now = pg;
                pg = pg_next;
                sc = scales_of(pg);
                pg_next = i + 2 < n ? page_of(tile + 2) : -1;
                if (pg_now < 0 && t < kv) kv_report(p.status);

                ok = ptx::mbar_wait(&S->s_full[k & 1], (uint32_t)(k >> 1) & 1u, kATimeoutNs) && ok;
                ptx::tc_fence_after();
                float x[R];
                {
                    uint32_t s[N / 16][16];
#pragma unroll
                    for (int j = 0; j < N / 16; ++j)
                        ptx::tmem_ld_32x32b_x16(lane_base + (uint32_t)((k & 1) * N + 16 * j), s[j]);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < N / 16; ++j) ptx::reg_fence16(s[j]);
                    // base-2 logit + log2 of V's scale: the weight of a code of V
                    const float lv = pg_now < 0 ? -INFINITY : log2f(sc_now.y);
#pragma unroll
                    for (int c = 0; c < R; ++c) {
                        const int c2 = R + c;
                        const float dot = fmaf(__uint_as_float(s[c2 / 16][c2 % 16]), 1.f / kRest,
                                               __uint_as_float(s[c / 16][c % 16]));
                        x[c] = fmaf(dot * sc_now.x, S->rowf[c], lv);
                    }
                }
                if ((tile + 1) * kATile > minlim) {
#pragma unroll
                    for (int c = 0; c < R; ++c)
                        if (t >= S->lim[c]) x[c] = -INFINITY;
                }
                float (*wm)[R] = S->wmax[k & 1];
#pragma unroll
                for (int c = 0; c < R; ++c) {
                    const float m = warp_max(x[c]);
                    if (lane == 0) wm[warp][c] = m;
                }
                ok = all_agree(ok);
                if (!ok) break;
                const float inv_v = pg_now < 0 ? 0.f : 1.f / sc_now.y;
                uint8_t *pb = ps + (size_t)(k & 1) * Sh::kOpBytes;
                float a_now[R], b_now[R];
#pragma unroll
                for (int c = 0; c < R; c += 2) {
                    float wgt[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int cc = c + u;
                        const float m = fmaxf(fmaxf(wm[0][cc], wm[1][cc]), fmaxf(wm[2][cc], wm[3][cc]));
                        const float ref = m == -INFINITY ? 0.f : m;
                        const float top = fmaxf(run[cc], m), tref = top == -INFINITY ? 0.f : top;
                        const float wt = ex2(x[cc] - ref);
                        a_now[cc] = ex2(run[cc] - tref);
                        b_now[cc] = ex2(m - tref);
                        run[cc] = top;
                        l[cc] = fmaf(l[cc], a_now[cc], wt * inv_v * b_now[cc]);
                        wgt[u] = wt * kPScale;
                    }
                    const uint32_t p1 = e4m3x2(wgt[0], wgt[1]);
                    const float2 f = __half22float2(half2_of_e4m3((uint16_t)p1));
                    const uint32_t p2 = e4m3x2((wgt[0] - f.x) * kRest, (wgt[1] - f.y) * kRest);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int r1 = c + u, r2 = R + c + u;
                        pb[r1 * 128 + (tid ^ ((r1 & 7) << 4))] = (uint8_t)(p1 >> (8 * u));
                        pb[r2 * 128 + (tid ^ ((r2 & 7) << 4))] = (uint8_t)(p2 >> (8 * u));
                    }
                }
                if ((tile + 1) * kATile > minlim) {
                    // rows of V that a weight of 0 must not meet: past the sequence, or
                    // NaN where only some rows see the token
                    const int seq = 2 * k + 1, st = seq % Sh::kStages;
                    ok = ptx::mbar_wait(&S->full[st], (uint32_t)(seq / Sh::kStages) & 1u, kATimeoutNs) && ok;
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
                                    if ((bad >> (8 * u)) & 1u) atomicMin(&S->nan_min[ch + u], t);
                            }
                        }
                    }
                }
                ptx::tc_fence_before();
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&S->p_ready[k & 1]);
                if (i > 0) read_output(k - 1);
#pragma unroll
                for (int c = 0; c < R; ++c) {
                    alpha[c] = a_now[c];
                    beta[c] = b_now[c] * (1.f / kPScale);
                }
            }
            if (!ok) break;   // agreed on: every warp of the four leaves here
            read_output(k - 1);
            // sums over the tokens
#pragma unroll
            for (int c = 0; c < R; ++c) {
                float s = l[c];
#pragma unroll
                for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
                if (lane == 0) S->lsum[warp][c] = s;
            }
            ok = all_agree(ok);
            if (!ok) break;
            const int nan_at = S->nan_min[tid];
            const bool whole = n == w.tiles;
            const size_t slot = 2 * (size_t)blockIdx.x + (w.tile == 0 ? 1 : 0);
#pragma unroll
            for (int c = 0; c < R; ++c) {
                if (c >= rows) continue;
                const float L = S->lsum[0][c] + S->lsum[1][c] + S->lsum[2][c] + S->lsum[3][c];
                float o = S->lim[c] > nan_at ? NAN : acc[c];
                if (whole) {
                    const int i = c / p.G, hq = h * p.G + c - i * p.G;
                    o = L == 0.f ? 0.f : o / L;
                    if (tid < p.D && wz_in_range(p.status, i < ntok && x0 + i < p.T))
                        p.out[(size_t)(x0 + i) * p.out_stride + (size_t)hq * p.D + tid] = __float2bfloat16_rn(o);
                    if (tid == 0 && p.lse)
                        p.lse[(size_t)(x0 + i) * p.Hq + hq] = L == 0.f ? -INFINITY : (run[c] + log2f(L)) * kLn2;
                } else if (wz_in_range(p.status, slot < 2 * (size_t)p.ctas)) {
                    p.part[(slot * R + c) * 128 + tid] = o;
                    if (tid == 0) p.ml[slot * R + c] = make_float2(run[c], L);
                }
            }
        }
        if (!ok) attend_fail(p, abort_flag);
    }
    __syncthreads();
    if (warp == 5) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, Sh::kTmem);
    }
}

// Row c of item (b, h): adds the pieces that several CTAs hold, in their order, or
// writes the answer of a sequence without tokens.
template <int R>
__global__ void __launch_bounds__(512) attend_join_kernel(const __grid_constant__ AttendParams p) {
    __shared__ long long scan[16];
    __shared__ long long before_b;
    __shared__ float fac[2 * 512];
    __shared__ float red[16], sums[4][128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();
    const int b = (int)blockIdx.x / p.heads, h = (int)blockIdx.x - b * p.heads, c = blockIdx.y;
    const int2 len = attend_lengths(p, b);
    const int i = c / p.G, g = c - i * p.G;
    if (i >= len.x) return;
    const size_t x = (size_t)(p.cu[b] + i);
    const int hq = h * p.G + g;
    const int tiles = few_tiles(p, b);
    if (tiles == 0) {
        if (tid < p.D) p.out[x * p.out_stride + (size_t)hq * p.D + tid] = __float2bfloat16_rn(0.f);
        if (tid == 0 && p.lse) p.lse[x * p.Hq + hq] = -INFINITY;
        return;
    }
    const int per = (p.B + (int)blockDim.x - 1) / (int)blockDim.x;
    const int blo = min(p.B, tid * per), bhi = min(p.B, blo + per);
    long long mine = 0, total;
    for (int j = blo; j < bhi; ++j) mine += few_tiles(p, j);
    const long long before = block_scan(mine, scan, &total);
    if (blo <= b && b < bhi) {
        long long at = before;
        for (int j = blo; j < b; ++j) at += few_tiles(p, j);
        before_b = at;
    }
    __syncthreads();
    total *= p.heads;
    const long long a0 = before_b * p.heads + (long long)h * tiles, a1 = a0 + tiles - 1;
    const int c0 = few_range_of(p, total, a0), c1 = few_range_of(p, total, a1);
    if (c0 == c1) return;   // one CTA had the whole item
    const int np = c1 - c0 + 1;   // at most p.ctas <= 1024
    const auto slot = [&](int j) { return 2 * (size_t)(c0 + j) + (j == 0 ? 1 : 0); };
    float m = -INFINITY;
    for (int j = tid; j < np; j += blockDim.x) {
        const float2 v = p.ml[slot(j) * R + c];
        fac[j] = v.x;
        m = fmaxf(m, v.x);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if (lane == 0) red[warp] = m;
    __syncthreads();
    for (int j = 0; j < (int)(blockDim.x >> 5); ++j) m = fmaxf(m, red[j]);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int j = tid; j < np; j += blockDim.x) fac[j] = ex2(fac[j] - ref);
    __syncthreads();
    // quarter of the pieces x channel
    const int quarter = tid >> 7, ch = tid & 127;
    const int lo = np * quarter / 4, hi = np * (quarter + 1) / 4;
    float o = 0.f, L = 0.f;
#pragma unroll 4
    for (int j = lo; j < hi; ++j) {
        const float f = fac[j];
        const size_t s = slot(j) * R + c;
        o = fmaf(p.part[s * 128 + ch], f, o);
        L = fmaf(p.ml[s].y, f, L);
    }
    sums[quarter][ch] = o;
    if (ch == 0) red[quarter] = L;
    __syncthreads();
    if (quarter == 0 && ch < p.D) {
        L = (red[0] + red[1]) + (red[2] + red[3]);
        o = (sums[0][ch] + sums[1][ch]) + (sums[2][ch] + sums[3][ch]);
        p.out[x * p.out_stride + (size_t)hq * p.D + ch] = __float2bfloat16_rn(L == 0.f ? 0.f : o / L);
        if (ch == 0 && p.lse) p.lse[x * p.Hq + hq] = L == 0.f ? -INFINITY : (m + log2f(L)) * kLn2;
    }
}

namespace {

template <int R>
cudaError_t launch_few(const AttendMaps &maps, AttendParams p, int max_new, int sms, cudaStream_t s) {
    using Sh = FewShape<R>;
    cudaError_t e = allow_smem((const void *)attend_few_kernel<R>, Sh::kSmem);
    if (e != cudaSuccess) return e;
    // no more CTAs than tiles there can be
    const int64_t most = (int64_t)p.B * p.heads * (((int64_t)p.max_pages * p.P + kATile - 1) / kATile);
    p.ctas = (int)std::min<int64_t>({(int64_t)sms * Sh::kCtas, kFewSlots / 2, most});
    void *args[] = {const_cast<AttendMaps *>(&maps), &p};
    e = launch_kernel((const void *)attend_few_kernel<R>, dim3(p.ctas), dim3(kFThreads), Sh::kSmem, s, args, true);
    if (e != cudaSuccess) return e;
    void *jargs[] = {&p};
    const int rows = std::min<int64_t>((int64_t)max_new * p.G, R);
    return launch_kernel((const void *)attend_join_kernel<R>, dim3((unsigned)(p.B * p.heads), rows), dim3(512), 0, s,
                         jargs, true);
}

}  // namespace

cudaError_t launch_attend_few(const AttendMaps &maps, const AttendParams &p, int max_new, int sms, cudaStream_t s) {
    return (int64_t)max_new * p.G <= 8 ? launch_few<8>(maps, p, max_new, sms, s)
                                       : launch_few<16>(maps, p, max_new, sms, s);
}

}  // namespace wz
