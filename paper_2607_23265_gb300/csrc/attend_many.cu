// Attention over the paged 8-bit cache for many query rows (wz_attend): prompts,
// questions, anything beyond 16 rows (tokens x heads of the group) a sequence and
// KV head.
//
// Bound by the tensor cores.  A CTA takes 256 rows of one sequence and KV head as two
// row tiles of 128 that take turns: while one tile's weights are formed, the other's
// products run.
//   S [128 rows x 128 tokens] = (q1 + q2) K^T    e4m3: a query is two codes a channel,
//                                                both into one accumulator
//   O [128 rows x D]         += W V              f16: weights from tensor memory (they
//                                                take the place of S), V from shared memory
// The codes of K go to the tensor cores as they are.  Those of V are converted to
// f16 once for both row tiles, because weights in f16 need no second number: 11
// bits down to 2^-17 of the running maximum and steps of 2^-27 of it below, so that
// the many small weights of a long context are not lost beside one large one.  The
// scales of V's pages multiply the weights, those of K's the logits, one of each for 16
// tokens.  A thread of warps 0-7 has one row: maximum, weights and sum need no other
// lane; its 128 logits stay in registers (setmaxnreg).
// The maximum that weights are relative to follows the true one only when that is
// 2^12 above it (2^8: one tile in five of logits of a few units, a fifth of the time):
// the tile's weights are formed without waiting for its maximum, and where it turns
// out so O is rescaled in tensor memory and they are formed again.
// Where a call has 128 rows at most a sequence and KV head, both tiles hold the same rows
// (paired) and take the tiles of tokens in turn; their pieces are added as those of splits.
//   warps 0-3, 4-7  weights of row tile 0, 1
//   warps 8-11      V to f16
//   warps 12, 14    TMA producers: rings of K and of V tiles
//   warp 13         TMEM allocation, MMA issuer (one thread)
// Tensor memory: S (then W) of the tiles in columns 0 and 128, O in 256 and 384.
// A prompt of 6,151 tokens of 28 heads x 128 takes 260 us (1,040 TFLOP/s): 4,100 cycles for
// each 256 x 128 block, of which a row tile's chain is 300 to read S, 1,200 to 1,900 to
// form the weights (floor of both tiles' exponentials on an SM sub-partition: 1,300), 400
// to store them, and 600 + 600 in its products; then starts and ends of CTAs.  What these
// cost: queries loaded under a condition, each load behind the one before, 7,000 cycles; the
// first tile's weights formed twice 2,500; columns hidden one by one, logit and weight,
// 4,000 a tile (292 us with all three).
// Measured slower, against 290: halves of 64 tokens with the logits one half ahead (342: N =
// 64 products cost what N = 128 cost), two threads to a row (301).
// Every wait is bounded; where one gives up the kernel sets a status bit, ends its
// copies, frees tensor memory and returns.
#include <cfloat>
#include <cstring>
#include <type_traits>

#include "wz_attend.cuh"

namespace wz {

namespace {

constexpr int kMThreads = 16 * 32;   // four warpgroups; two warps of the last have nothing to do
constexpr int kMKStages = 3, kMVStages = 2;
constexpr int kMTmem = 512;
constexpr float kMTop = 3.f;     // a row's largest weight is about 2^3 ..
constexpr float kMSlack = 12.f;  // .. and at most 2^15, below f16's largest

struct ManyShared {
    uint64_t k_full[kMKStages], k_empty[kMKStages], v_full[kMVStages], v_empty[kMVStages];
    uint64_t w_full[2], w_empty[2];              // V in f16
    uint64_t s_full[2], p_ready[2], o_full[2];   // by row tile
    uint64_t q_ready, drain;
    uint32_t tmem_base;
    int abort;
    float rowf[kManyRows];
    int any_nan;
    int nan_min[128];                            // per channel: first token that some rows see and whose V is NaN
};

constexpr int kMQBytes = 4 * 128 * 128;          // row tiles x (codes, rests)
constexpr size_t kMSmem =
    1024 + kMQBytes + (size_t)(kMKStages + kMVStages) * kATileBytes + 2 * 2 * (size_t)kATileBytes + sizeof(ManyShared);
static_assert(kMSmem <= 227 * 1024, "shared memory of the CTA");

// What a CTA does: rows r0 .. r1-1 of (b, h), tiles t0 .. t1-1 of 128 slots.
struct ManyItem {
    int b, h, r0, r1, n, kv, x0;   // n: the sequence's tokens of q
    int t0, t1;
};

__device__ __forceinline__ bool many_item(const AttendParams &p, int row_tiles, int splits, int idx, ManyItem *it) {
    uint32_t at = (uint32_t)idx, s = 0;
    if (splits > 1) {
        s = at % (uint32_t)splits;
        at /= (uint32_t)splits;
    }
    it->h = (int)(at % (uint32_t)p.heads);
    at /= (uint32_t)p.heads;
    it->b = p.B > 1 ? (int)(at % (uint32_t)p.B) : 0;
    const int rt = row_tiles - 1 - (int)(p.B > 1 ? at / (uint32_t)p.B : at);   // the longest rows of causal calls first
    const int2 len = attend_lengths(p, it->b);
    const int64_t rows = (int64_t)len.x * p.G;
    if ((int64_t)rt * kManyRows >= rows) return false;
    it->n = len.x;
    it->kv = len.y;
    it->x0 = p.cu[it->b];
    it->r0 = rt * kManyRows;
    it->r1 = (int)min(rows, (int64_t)it->r0 + kManyRows);
    const int most = min(it->kv, attend_visible(p, (it->r1 - 1) / p.G, it->n, it->kv));
    const uint32_t tiles = (uint32_t)(most + kATile - 1) / kATile;   // below 2^24, splits at most 32
    it->t0 = splits > 1 ? (int)(tiles * s / (uint32_t)splits) : 0;
    it->t1 = splits > 1 ? (int)(tiles * (s + 1) / (uint32_t)splits) : (int)tiles;
    return true;
}

// The largest of three, given as bits.
__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return r;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Columns from rel on are not seen: logits of -infinity.
__device__ __forceinline__ void hide(uint32_t (&s)[4][32], int rel) {
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        if (!__any_sync(0xFFFFFFFFu, 16 * g + 16 > rel)) continue;
        uint32_t *x = s[g / 2] + 16 * (g % 2);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (16 * g + j >= rel) x[j] = 0xFF800000u;
    }
}

// Factor of 16 columns' logits: not 0, for those of -infinity.
__device__ __forceinline__ float factor(float k, float rowf) {
    const float a = k * rowf;
    return a == 0.f ? FLT_MIN : a;
}

// The largest of 16 logits.
__device__ __forceinline__ float max16(const uint32_t *x) {
    float m = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int j = 3; j < 15; j += 2) m = max3(__float_as_uint(m), x[j], x[j + 1]);
    return fmaxf(m, __uint_as_float(x[15]));
}

// A row's largest logit with its weight of V; lanes 0-7 hold the scales of 16 tokens each.
__device__ __forceinline__ float largest(const uint32_t (&s)[4][32], float my_k, float my_lv, float rowf) {
    float top = -INFINITY;
#pragma unroll
    for (int g = 0; g < 8; ++g)
        top = fmaxf(top, fmaf(max16(s[g / 2] + 16 * (g % 2)), factor(__shfl_sync(0xFFFFFFFFu, my_k, g), rowf),
                              __shfl_sync(0xFFFFFFFFu, my_lv, g)));
    return top;
}

// A row's 128 logits to weights in f16, 16 to the first half of each s[c].  top: as
// above, add: the weights' sum.
__device__ __forceinline__ void weights(uint32_t (&s)[4][32], float my_k, float my_lv, float my_inv, float rowf,
                                        float base, float &top, float &add) {
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        const uint32_t *x = s[g / 2] + 16 * (g % 2);
        const float a = factor(__shfl_sync(0xFFFFFFFFu, my_k, g), rowf), lv = __shfl_sync(0xFFFFFFFFu, my_lv, g);
        top = fmaxf(top, fmaf(max16(x), a, lv));
        const f2_t a2 = pack2(a, a), off2 = pack2(lv + base, lv + base);
        f2_t part[2] = {0, 0};   // zeros
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float2 v = unpack2(fma2(pack2(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), a2, off2));
            const float w0 = ex2(v.x), w1 = ex2(v.y);
            part[(j / 2) % 2] = add2(part[(j / 2) % 2], pack2(w0, w1));
            s[g / 2][8 * (g % 2) + j / 2] = pack_half2(w0, w1);   // past the logits that are still to come
        }
        const float2 both = unpack2(add2(part[0], part[1]));
        add = fmaf(both.x + both.y, __shfl_sync(0xFFFFFFFFu, my_inv, g), add);
    }
}

}  // namespace

// PAIRED: a variant of its own, since the choice at run time costs every call 3 % (260 us to 267).
template <bool PAIRED>
__global__ void __launch_bounds__(kMThreads, 1)
attend_many_kernel(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendParams p, int row_tiles,
                   int splits) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *qs = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *kring = qs + kMQBytes;
    uint8_t *vring = kring + (size_t)kMKStages * kATileBytes;
    uint8_t *wring = vring + (size_t)kMVStages * kATileBytes;      // V in f16: two buffers of 32 KB
    ManyShared *S = reinterpret_cast<ManyShared *>(wring + 4 * (size_t)kATileBytes);
    volatile int *abort_flag = &S->abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    pdl_wait();
    pdl_trigger();
    ManyItem it;
    if (!many_item(p, row_tiles, splits, (int)blockIdx.x, &it)) {
        if (tid == 0 && !attend_lengths_sound(p, it.b)) kv_report(p.status);
        return;
    }
    if (tid == 0 && !attend_lengths_sound(p, it.b)) kv_report(p.status);
    if (tid == 0) {
        for (int s = 0; s < kMKStages; ++s) {
            ptx::mbar_init(&S->k_full[s], 1);
            ptx::mbar_init(&S->k_empty[s], 1);
        }
        for (int s = 0; s < kMVStages; ++s) {
            ptx::mbar_init(&S->v_full[s], 1);
            ptx::mbar_init(&S->v_empty[s], 4);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&S->w_full[i], 4);
            ptx::mbar_init(&S->w_empty[i], 1);
            ptx::mbar_init(&S->s_full[i], 1);
            ptx::mbar_init(&S->p_ready[i], 4);
            ptx::mbar_init(&S->o_full[i], 1);
        }
        ptx::mbar_init(&S->q_ready, 8);
        ptx::mbar_init(&S->drain, 1);
        S->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    if (tid < 128) S->nan_min[tid] = INT32_MAX;
    if (tid == 128) S->any_nan = 0;
    if (warp == 13) {
        ptx::tmem_alloc(&S->tmem_base, kMTmem);
        ptx::tmem_relinquish();
    }
    if (warp == 12 && lane == 0) {
        ptx::prefetch_tmap(&maps.k);
        ptx::prefetch_tmap(&maps.v);
    }
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;
    const int n = it.t1 - it.t0;
    if (PAIRED) it.r1 = min(it.r1, it.r0 + 128);          // more tokens than max_new, reported above
    const int qtiles = PAIRED || it.r1 - it.r0 > 128 ? 2 : 1;
    const int stride = PAIRED ? 2 : 1;                    // tiles from one of a row tile's to its next
    const int minlim = max(0, min(it.kv, attend_visible(p, it.r0 / p.G, it.n, it.kv)));
    const int maxlim = max(0, min(it.kv, attend_visible(p, (it.r1 - 1) / p.G, it.n, it.kv)));

    // 512 threads start with 128 registers: 256 x 184 + 128 x 64 + 128 x 80 = 512 x 128
    if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == 12 || warp == 14) {
            // ---------------- TMA producers of K and of V: lane = page of the tile ----------------
            const bool v = warp == 14;
            const int stages = v ? kMVStages : kMKStages;
            uint64_t *full = v ? S->v_full : S->k_full, *empty = v ? S->v_empty : S->k_empty;
            uint8_t *ring = v ? vring : kring;
            const CUtensorMap *map = v ? &maps.v : &maps.k;
            const uint64_t pol = ptx::policy_evict_last();   // other row tiles read the same slots
            const int pages_tile = kATile / p.P, box = p.P * 128;
            const int absent = (int)(p.pages * p.heads);     // past the cache: zeros
            auto slab = [&](int tile) {
                const int t = tile * kATile + (lane << p.shift);
                int pg = -1;
                if (lane < pages_tile && tile < it.t1 && t < it.kv) {
                    pg = attend_page(p, it.b, t);
                    if (pg < 0) kv_report(p.status);
                }
                return pg < 0 ? absent : pg * p.heads + it.h;
            };
            int znext = slab(it.t0), done = 0, st = 0;
            uint32_t phase = 0;
            for (int i = 0; i < n; ++i) {
                const int z = znext;
                znext = slab(it.t0 + i + 1);
                const bool ok = __all_sync(0xFFFFFFFFu, warp_wait(p, &empty[st], phase ^ 1u) && !*abort_flag);
                if (!ok) {
                    attend_fail(p, abort_flag);
                    break;
                }
                if (lane == 0) ptx::mbar_arrive_expect_tx(&full[st], kATileBytes);
                __syncwarp();
                if (lane < pages_tile)
                    ptx::tma_load_3d(ring + (size_t)st * kATileBytes + (size_t)lane * box, map, &full[st], 0, 0, z, pol);
                done = i + 1;
                if (++st == stages) {
                    st = 0;
                    phase ^= 1u;
                }
            }
            for (int i = max(0, done - stages); i < done; ++i)   // the copies have landed
                ptx::mbar_wait(&full[i % stages], (uint32_t)(i / stages) & 1u, kATimeoutNs);
        } else if (warp == 13 && ptx::elect_one()) {
            // ---------------- MMA issuer ----------------
            const uint32_t id_s = ptx::idesc_e4m3(128, 128, false, false), id_o = ptx::idesc_f16(128, p.D, false, true);
            const uint64_t q_desc = ptx::smem_desc(ptx::smem_u32(qs), 16, 1024, 2);
            const uint64_t k_desc = ptx::smem_desc(ptx::smem_u32(kring), 16, 1024, 2);
            const uint64_t w_desc = ptx::smem_desc(ptx::smem_u32(wring), kATileBytes, 1024, 2);   // 64 channels: 16 KB
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                if (ok && !ptx::mbar_wait(bar, parity, wait_limit(p))) {
                    attend_fail(p, abort_flag);
                    ok = false;
                }
                return ok;
            };
            // S of row tile q for tile i: 32 channels of the codes, of the rests, of the codes ..
            auto logits = [&](auto q_, int i) {
                constexpr int q = decltype(q_)::value;
                const uint64_t a = q_desc + (uint64_t)(q * 2) * (kATileBytes >> 4);
                const uint64_t b = k_desc + (uint64_t)(i % kMKStages) * (kATileBytes >> 4);
                const uint32_t d = tmem + (uint32_t)(q * 128);
                constexpr uint64_t rest = kATileBytes >> 4;
                if (p.D > 64) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        ptx::mma_e4m3(d, a + (uint64_t)(j & 1) * rest + (uint64_t)(2 * (j >> 1)),
                                      b + (uint64_t)(2 * (j >> 1)), id_s, j > 0);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        ptx::mma_e4m3(d, a + (uint64_t)(j & 1) * rest + (uint64_t)(2 * (j >> 1)),
                                      b + (uint64_t)(2 * (j >> 1)), id_s, j > 0);
                }
                if (PAIRED || q == qtiles - 1) ptx::mma_commit(&S->k_empty[i % kMKStages]);
                ptx::mma_commit(&S->s_full[q]);
            };
            // O of row tile q after its weights of tile i, then its logits of the next tile
            auto step = [&](auto q_, int i) {
                constexpr int q = decltype(q_)::value;
                const uint32_t par = (uint32_t)(PAIRED ? i >> 1 : i) & 1u;
                if ((PAIRED || q == 0) && !wait(&S->w_full[i & 1], (uint32_t)(i >> 1) & 1u)) return;
                if (!wait(&S->p_ready[q], par)) return;
                ptx::tc_fence_after();
                const uint64_t b = w_desc + (uint64_t)(i & 1) * (2 * kATileBytes >> 4);
#pragma unroll
                for (int s = 0; s < kATile / 16; ++s)   // 16 tokens: 8 columns of W, two groups of 8 rows of V
                    ptx::mma_f16_ta(tmem + (uint32_t)(256 + q * 128), tmem + (uint32_t)(q * 128 + 8 * s),
                                    b + (uint64_t)(s * (2048 >> 4)), id_o, s > 0 || i >= stride);
                if (PAIRED || q == qtiles - 1) ptx::mma_commit(&S->w_empty[i & 1]);
                ptx::mma_commit(&S->o_full[q]);
                const int next = i + stride;
                if (next >= n) return;
                if ((PAIRED || q == 0) && !wait(&S->k_full[next % kMKStages], (uint32_t)(next / kMKStages) & 1u)) return;
                // S takes the place of the weights: their products have to be complete
                if (!wait(&S->o_full[q], par)) return;
                ptx::tc_fence_after();
                logits(q_, next);
            };
            constexpr std::integral_constant<int, 0> q0{};
            constexpr std::integral_constant<int, 1> q1{};
            if (n > 0 && wait(&S->q_ready, 0) && wait(&S->k_full[0], 0)) {
                ptx::tc_fence_after();
                logits(q0, 0);
                if (PAIRED && n > 1 && wait(&S->k_full[1], 0)) {
                    ptx::tc_fence_after();
                    logits(q1, 1);
                }
                if (!PAIRED && qtiles == 2) logits(q1, 0);
                for (int i = 0; i < n && ok; ++i) {
                    if (!PAIRED || i % 2 == 0) step(q0, i);
                    if ((PAIRED ? i % 2 == 1 : qtiles == 2) && ok) step(q1, i);
                }
            }
            ptx::mma_commit(&S->drain);
            ptx::mbar_wait(&S->drain, 0, kATimeoutNs);
        }
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ---------------- V to f16: a warp takes two rows x four pieces of 16 channels at a time ----------------
        const int c4 = lane & 3, odd = (lane >> 2) & 1, far = (lane >> 3) & 1, pair = lane >> 4;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int vs = i % kMVStages, base = (it.t0 + i) * kATile;
            ok = warp_wait(p, &S->v_full[vs], (uint32_t)(i / kMVStages) & 1u) &&
                 warp_wait(p, &S->w_empty[i & 1], ((uint32_t)(i >> 1) & 1u) ^ 1u);
            ok = __all_sync(0xFFFFFFFFu, ok && !*abort_flag);
            if (!ok) {
                attend_fail(p, abort_flag);
                break;
            }
            const uint8_t *src = vring + (size_t)vs * kATileBytes;
            uint8_t *dst = wring + (size_t)(i & 1) * (2 * kATileBytes) + (size_t)far * kATileBytes;
            const bool mixed = base + kATile > minlim;
            const int t0 = (warp - 8) * 32 + 2 * pair + odd;   // and every fourth row from here
            for (int g0 = 0; g0 < 8; g0 += 4) {
                uint32_t in[4][4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int t = t0 + 4 * (g0 + g);
                    const uint4 v = *reinterpret_cast<const uint4 *>(src + t * 128 + (((far * 4 + c4) ^ (t & 7)) << 4));
                    in[g][0] = v.x;
                    in[g][1] = v.y;
                    in[g][2] = v.z;
                    in[g][3] = v.w;
                }
                if (mixed) {
                    // codes that a weight of 0 must not meet
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int t = base + t0 + 4 * (g0 + g);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (t >= maxlim) in[g][j] = 0;
                            const uint32_t bad = __vcmpeq4(in[g][j] & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
                            if (bad && t >= minlim) {
                                for (int u = 0; u < 4; ++u)
                                    if ((bad >> (8 * u)) & 1u)
                                        atomicMin(&S->nan_min[far * 64 + c4 * 16 + 4 * j + u], t);
                                in[g][j] &= ~bad;
                                S->any_nan = 1;
                            }
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int t = t0 + 4 * (g0 + g), x = t & 7;
                    uint32_t o[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const __half2 a = half2_of_e4m3((uint16_t)(in[g][j] & 0xFFFFu));
                        const __half2 b = half2_of_e4m3((uint16_t)(in[g][j] >> 16));
                        o[2 * j] = *reinterpret_cast<const uint32_t *>(&a);
                        o[2 * j + 1] = *reinterpret_cast<const uint32_t *>(&b);
                    }
                    *reinterpret_cast<uint4 *>(dst + t * 128 + (((2 * c4) ^ x) << 4)) =
                        make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4 *>(dst + t * 128 + (((2 * c4 + 1) ^ x) << 4)) =
                        make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(&S->v_empty[vs]);
                ptx::mbar_arrive(&S->w_full[i & 1]);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        // ---------------- weights ----------------
        const int q = warp >> 2, row = tid;               // this thread's row of the CTA's two tiles
        const int same = PAIRED ? q * 128 : 0;            // paired: both hold the same rows
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes + (uint32_t)(q * 128), o_at = lanes + (uint32_t)(256 + q * 128);
        const uint32_t flip = p.scale2 < 0.f ? 0x80808080u : 0u;   // logits' factors are positive
        {
            // eight lanes to a row, 16 channels to a lane; all of a warp's rows in flight
            const int sub = lane & 7, r0 = warp * 32 + (lane >> 3);
            uint4 raw[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // every lane loads, so that no load waits for the one before: past the rows the last
                const int at = min(it.r0 + r0 - same + 4 * j, it.r1 - 1), i = at / p.G, g = at - i * p.G;
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (size_t)(it.x0 + i) * p.q_stride +
                                                                   (size_t)(it.h * p.G + g) * p.D +
                                                                   (16 * sub < p.D ? 16 * sub : 0));
                raw[j][0] = src[0];
                raw[j][1] = src[1];
            }
            uint32_t most[8];   // bits of the largest magnitude: as floats, and infinities and NaN above all
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool none = it.r0 + r0 - same + 4 * j >= it.r1 || 16 * sub >= p.D;
                uint32_t m = 0;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    uint32_t &w = (&raw[j][u / 4].x)[u % 4];
                    w = none ? 0 : w;
                    m = max(m, max((w << 16) & 0x7FFFFFFFu, w & 0x7FFF0000u));
                }
                most[j] = m;
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1)
#pragma unroll
                for (int j = 0; j < 8; ++j) most[j] = max(most[j], __shfl_xor_sync(0xFFFFFFFFu, most[j], d));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = r0 + 4 * j;
                const uint32_t w[8] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w,
                                       raw[j][1].x, raw[j][1].y, raw[j][1].z, raw[j][1].w};
                const uint32_t m = most[j];
                const bool finite = m < 0x7F800000u;
                int e = 134 - (int)(m >> 23);   // takes the largest to [128, 256)
                e = m == 0 || !finite ? 0 : min(e, 126);
                const float up = __uint_as_float((uint32_t)(e + 127) << 23);
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    // f16 holds the 8 bits of a bf16 number, and what the code leaves of it
                    const __half2 x = __floats2half2_rn(__uint_as_float(w[u] << 16) * up,
                                                        __uint_as_float(w[u] & 0xFFFF0000u) * up);
                    const uint32_t c = e4m3x2(x);
                    const uint32_t d = e4m3x2(__hsub2(x, half2_of_e4m3((uint16_t)c)));
                    hi[u / 2] = u % 2 ? hi[u / 2] | c << 16 : c;
                    lo[u / 2] = u % 2 ? lo[u / 2] | d << 16 : d;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    hi[u] = finite ? hi[u] ^ flip : 0;
                    lo[u] = finite ? lo[u] ^ flip : 0;
                }
                uint8_t *dst = qs + (size_t)(q * 2) * kATileBytes + (r & 127) * 128 + ((sub ^ (r & 7)) << 4);
                *reinterpret_cast<uint4 *>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(dst + kATileBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                if (sub == 0)
                    S->rowf[r] = finite ? __uint_as_float((uint32_t)(127 - e) << 23) * fabsf(p.scale2) : NAN;
            }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&S->q_ready);
        const float rowf = S->rowf[row];   // this warp's rows
        const int at = it.r0 + row - same, tok = at / p.G;
        const bool real = at < it.r1;
        const int lim = real ? max(0, min(it.kv, attend_visible(p, tok, it.n, it.kv))) : 0;

        float ref = -INFINITY, sum = 0.f;
        bool ok = true;
        const int steps = PAIRED ? (n + 1 - q) / 2 : q < qtiles ? n : 0;
        const int first = it.t0 + (PAIRED ? q : 0);   // this row tile's first
        // lane l < 8: scales of the l-th 16 tokens of a tile, loaded one tile ahead, their page two
        auto page_of = [&](int tile) {
            const int t = tile * kATile + 16 * lane;
            return lane < 8 && tile < it.t1 && t < it.kv ? attend_page(p, it.b, t) : -1;
        };
        auto scales_of = [&](int pg) {
            return pg < 0 ? make_float2(1.f, 0.f)
                          : make_float2(p.k_scale[(size_t)pg * p.heads + it.h], p.v_scale[(size_t)pg * p.heads + it.h]);
        };
        int pg_next = steps > 0 ? page_of(first + stride) : -1;
        float2 next = scales_of(steps > 0 ? page_of(first) : -1);
        // factor of the logits, log2 and reciprocal of V's scale
        float my_k, my_lv, my_inv;
        auto take_scales = [&](int tile_after) {
            my_k = next.x;
            my_lv = next.y > 0.f ? __log2f(next.y) : -INFINITY;
            my_inv = next.y > 0.f ? __frcp_rn(next.y) : 0.f;
            next = scales_of(pg_next);
            pg_next = page_of(tile_after);
        };
        take_scales(first + 2 * stride);
        for (int i = 0; i < steps; ++i) {
            const int tile = first + i * stride, rel = lim - tile * kATile;   // columns of the tile that this row sees
            const bool mixed = (tile + 1) * kATile > minlim;
            ok = warp_wait(p, &S->s_full[q], (uint32_t)i & 1u);
            ok = __all_sync(0xFFFFFFFFu, ok && !*abort_flag);
            if (!ok) break;
            ptx::tc_fence_after();
            uint32_t s[4][32];
            // Weights relative to the maximum of the tiles before; where this tile's is too
            // far above it, once more relative to that.
            for (;;) {
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32b_x32(s_at + (uint32_t)(32 * c), s[c]);
                float top = -INFINITY, add = 0.f;
                ptx::tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::reg_fence32(s[c]);
                if (mixed) hide(s, rel);
                if (i == 0) ref = largest(s, my_k, my_lv, rowf);   // else most rows would come here twice
                const float base = kMTop - (ref == -INFINITY ? 0.f : ref);
                weights(s, my_k, my_lv, my_inv, rowf, base, top, add);
                const bool rise = top > ref + kMSlack;
                if (!__any_sync(0xFFFFFFFFu, rise)) {
                    sum += add;
                    break;
                }
                const float to = rise ? top : ref, f = rise ? ex2(ref - to) : 1.f;
                ref = to;
                sum *= f;
                if (i > 0) {   // the products of the tile before are complete: S followed them
                    for (int c = 0; c < p.D; c += 16) {
                        uint32_t o[16];
                        ptx::tmem_ld_32x32b_x16(o_at + (uint32_t)c, o);
                        ptx::tmem_ld_wait();
                        ptx::reg_fence16(o);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                        ptx::tmem_st_32x32b_x16(o_at + (uint32_t)c, o);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
                ptx::tmem_st_32x32b_x16(s_at + (uint32_t)(16 * c), *reinterpret_cast<const uint32_t(*)[16]>(&s[c]));
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&S->p_ready[q]);
            take_scales(tile + 3 * stride);
        }
        if (ok && steps > 0) {
            ok = ptx::mbar_wait(&S->o_full[q], (uint32_t)(steps - 1) & 1u, wait_limit(p));
            ok = __all_sync(0xFFFFFFFFu, ok);
        }
        if (!ok) attend_fail(p, abort_flag);
        ptx::tc_fence_after();
        if (ok && q < qtiles) {
            const int hq = it.h * p.G + at - tok * p.G;
            const size_t x = (size_t)(it.x0 + tok);
            if (lim == 0) sum = 0.f;   // a row that sees nothing: NaN where its query, and so its factor, is
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const bool nans = *reinterpret_cast<volatile int *>(&S->any_nan);
            uint32_t o[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (32 * c < p.D) ptx::tmem_ld_32x32b_x32(o_at + (uint32_t)(32 * c), o[c]);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 4; ++c) ptx::reg_fence32(o[c]);
            // Rows go through shared memory (the queries' place: their products are complete),
            // 256 bytes a row at a time, so that a warp's stores are whole rows: row by row of
            // its own a thread takes ten times as long.
            uint8_t *stage = qs + (size_t)(q * 2) * kATileBytes + (size_t)(warp & 3) * 32 * 256;
            auto flush = [&](void *dst, int bytes) {   // dst: where this thread's row goes, or null
                __syncwarp();
                const unsigned long long mine = reinterpret_cast<unsigned long long>(dst);
#pragma unroll 4
                for (int k = 0; k < 16; ++k) {
                    const int r = 2 * k + (lane >> 4), c = lane & 15;
                    const unsigned long long to = __shfl_sync(0xFFFFFFFFu, mine, r);
                    if (to && 16 * c < bytes)
                        *reinterpret_cast<uint4 *>(to + 16 * c) =
                            *reinterpret_cast<const uint4 *>(stage + r * 256 + ((c ^ (r & 15)) << 4));
                }
                __syncwarp();
            };
            auto put = [&](int c, uint4 v) {           // 16 bytes of this thread's row
                *reinterpret_cast<uint4 *>(stage + lane * 256 + ((c ^ (lane & 15)) << 4)) = v;
            };
            if (sum == 0.f || nans) {
#pragma unroll
                for (int j = 0; j < 128; ++j) {
                    if (sum == 0.f) o[j / 32][j % 32] = 0;
                    if (lim > S->nan_min[j]) o[j / 32][j % 32] = __float_as_uint(NAN);
                }
            }
            if (splits == 1 && !PAIRED) {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const __nv_bfloat162 v =
                            __floats2bfloat162_rn(__uint_as_float(o[c / 4][8 * (c % 4) + 2 * j]) * inv,
                                                  __uint_as_float(o[c / 4][8 * (c % 4) + 2 * j + 1]) * inv);
                        w[j] = *reinterpret_cast<const uint32_t *>(&v);
                    }
                    put(c, make_uint4(w[0], w[1], w[2], w[3]));
                }
                const bool in = wz_in_range(p.status, !real || x < (size_t)p.T) && real;
                flush(in ? p.out + x * p.out_stride + (size_t)hq * p.D : nullptr, 2 * p.D);
            } else {
#pragma unroll
                for (int part = 0; part < 2; ++part) {
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const uint32_t *f = &o[2 * part + c / 8][4 * (c % 8)];
                        put(c, make_uint4(f[0], f[1], f[2], f[3]));
                    }
                    float *to = p.part + ((size_t)blockIdx.x * kManyRows + row) * 128 + 64 * part;
                    flush(real ? to : nullptr, 4 * (p.D - 64 * part));
                }
            }
            if (real) {
                if (splits > 1 || PAIRED)
                    p.ml[(size_t)blockIdx.x * kManyRows + row] = make_float2(ref - kMTop, sum);
                else if (p.lse)
                    p.lse[x * p.Hq + hq] = sum == 0.f ? -INFINITY : (ref - kMTop + log2f(sum)) * kLn2;
            }
        }
    }
    __syncthreads();
    if (warp == 13) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, kMTmem);
    }
}

// Adds the pieces of each row, in order; a warp per row.
__global__ void __launch_bounds__(256)
attend_merge_kernel(const __grid_constant__ AttendParams p, int row_tiles, int splits, int paired) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int idx = (int)blockIdx.x / (kManyRows / 8), row = (int)blockIdx.x % (kManyRows / 8) * 8 + (threadIdx.x >> 5);
    ManyItem it;
    if (!many_item(p, row_tiles, splits, idx * splits, &it) || it.r0 + row >= it.r1) return;
    if (paired && row >= kManyRows / 2) return;
    // pieces of `step` rows: a CTA's, or of either of its tiles
    const int pieces = paired ? 2 * splits : splits, step = paired ? kManyRows / 2 : kManyRows;
    const size_t first = (size_t)idx * splits * kManyRows + row;
    float m = -INFINITY;
    for (int s = 0; s < pieces; ++s) m = fmaxf(m, p.ml[first + (size_t)s * step].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < pieces; ++s) {
        const size_t at = first + (size_t)s * step;
        const float2 ml = p.ml[at];
        const float f = ex2(ml.x - ref);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * lane < p.D) v = *reinterpret_cast<const float4 *>(p.part + at * 128 + 4 * lane);
        L = fmaf(ml.y, f, L);
        o[0] = fmaf(v.x, f, o[0]);
        o[1] = fmaf(v.y, f, o[1]);
        o[2] = fmaf(v.z, f, o[2]);
        o[3] = fmaf(v.w, f, o[3]);
    }
    const int tok = (it.r0 + row) / p.G, hq = it.h * p.G + (it.r0 + row) - tok * p.G;
    const size_t x = (size_t)(it.x0 + tok);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (4 * lane < p.D && wz_in_range(p.status, x < (size_t)p.T)) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(o[0] * inv, o[1] * inv);
        const __nv_bfloat162 b = __floats2bfloat162_rn(o[2] * inv, o[3] * inv);
        *reinterpret_cast<uint2 *>(p.out + x * p.out_stride + (size_t)hq * p.D + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
    if (lane == 0 && p.lse) p.lse[x * p.Hq + hq] = L == 0.f ? -INFINITY : (m + log2f(L)) * kLn2;
}

cudaError_t launch_attend_many(const AttendMaps &maps, const AttendParams &p, int max_new, int splits, int paired,
                               cudaStream_t s) {
    const void *kernel = paired ? (const void *)attend_many_kernel<true> : (const void *)attend_many_kernel<false>;
    cudaError_t e = allow_smem(kernel, kMSmem);
    if (e != cudaSuccess) return e;
    int row_tiles = (int)(((int64_t)max_new * p.G + kManyRows - 1) / kManyRows);
    const int64_t items = (int64_t)row_tiles * p.B * p.heads;
    if (items * splits > INT32_MAX) return cudaErrorInvalidValue;
    void *args[] = {const_cast<AttendMaps *>(&maps), const_cast<AttendParams *>(&p), &row_tiles, &splits};
    e = launch_kernel(kernel, dim3((unsigned)(items * splits)), dim3(kMThreads), kMSmem, s,
                      args, true);
    if (e != cudaSuccess || (splits == 1 && !paired)) return e;
    void *margs[] = {const_cast<AttendParams *>(&p), &row_tiles, &splits, &paired};
    return launch_kernel((const void *)attend_merge_kernel, dim3((unsigned)(items * (kManyRows / 8))), dim3(256), 0, s,
                         margs, true);
}

}  // namespace wz
