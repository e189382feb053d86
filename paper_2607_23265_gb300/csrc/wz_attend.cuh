// What the attention kernels over the paged 8-bit cache share (wz_attend).
#pragma once

#include <cfloat>
#include <cmath>

#include <cuda.h>
#include <cuda_bf16.h>

#include "wz_internal.cuh"
#include "wz_kv.cuh"
#include "wz_ptx.cuh"

namespace wz {

constexpr int kATile = 128;                  // tokens of a tile
constexpr int kATileBytes = kATile * 128;    // its codes of one KV head, rows of 128 bytes
constexpr int kFewSlots = 960;               // pieces of items that several CTAs share: two a CTA
constexpr int kManyRows = 256;               // query rows of a CTA of attend_many
constexpr int kManySlots = 320;              // pieces of its row tiles
constexpr double kSplitTiles = 3;            // what a CTA's start and end cost, in tiles
constexpr uint64_t kATimeoutNs = 2000000000ull;   // limit of every wait
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendMaps {
    CUtensorMap k, v;
};

struct AttendParams {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    int64_t q_stride, out_stride;
    float *lse;
    const int32_t *cu, *kv_len, *table;
    const float *k_scale, *v_scale;
    float *part;             // unnormalised outputs of pieces [slot][rows of a slot][128]
    float2 *ml;              // their maxima (base 2) and sums
    int2 *spans;             // by first token and KV head: first CTA and pieces of an item
    int64_t pages;
    int T, B, Hq, heads, G, D, P, max_pages, max_new, causal;
    int shift;               // log2(P)
    int ctas;                // CTAs that share the work
    int whole, item_cost;    // attend_few: items are not cut; tiles that an item's start and end count as
    int most;                // attend_few: tokens of a sequence that its rows have room for, max_new or more
    float scale2;            // scale * log2(e)
    int *status;
#ifdef WZ_CHECKED
    uint64_t wait_ns;        // limit of the waits that a warp gives up on (a test's may be short)
#endif
};

// Limit of a wait for another warp, a copy or a product that the kernel gives up on.  Waits for
// what is in flight when it ends, after it gave up too, keep kATimeoutNs.
__device__ __forceinline__ uint64_t wait_limit(const AttendParams &p) {
#ifdef WZ_CHECKED
    return p.wait_ns;
#else
    return kATimeoutNs;
#endif
}

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The most slots of a sequence: what the table has room for; tiles past them are counted in int too.
__device__ __forceinline__ int64_t attend_most(const AttendParams &p) {
    return min((int64_t)p.max_pages * p.P, (int64_t)INT32_MAX - 2 * kATile);
}

// Tokens of q and slots of sequence b; no tokens where its lengths make no sense.
__device__ __forceinline__ int2 attend_lengths(const AttendParams &p, int b) {
    const int x0 = p.cu[b], x1 = p.cu[b + 1];
    const int64_t most = attend_most(p);
    int kv = p.kv_len[b];
    if (kv < 0) kv = 0;
    if (kv > most) kv = (int)most;
    const bool sound = x0 >= 0 && x1 >= x0 && x1 <= p.T;
    return make_int2(sound ? x1 - x0 : 0, kv);
}

// Whether the lengths are what the call said: attend_lengths has to change nothing and
// no sequence has more tokens than max_new.
__device__ __forceinline__ bool attend_lengths_sound(const AttendParams &p, int b) {
    const int x0 = p.cu[b], x1 = p.cu[b + 1], kv = p.kv_len[b];
    return x0 >= 0 && x1 >= x0 && x1 <= p.T && x1 - x0 <= p.max_new && kv >= 0 &&
           kv <= attend_most(p);
}

// Slots that token i of n sees.
__device__ __forceinline__ int attend_visible(const AttendParams &p, int i, int n, int kv) {
    if (!p.causal) return kv;
    const int v = kv - n + i + 1;
    return v < 0 ? 0 : v;
}

// Page of token t of sequence b, or -1.
__device__ __forceinline__ int attend_page(const AttendParams &p, int b, int t) {
    const int pg = p.table[(size_t)b * p.max_pages + (t >> p.shift)];
    return pg >= 0 && pg < p.pages ? pg : -1;
}

// A barrier's phase, waited for by a whole warp; the same answer in every lane, false
// where the wait gave up.  (Lane 0 alone, the others behind it, took longer: a prompt of 6,151
// tokens 510 us instead of 451, when that was its time; 260 now.)
__device__ __forceinline__ bool warp_wait(const AttendParams &p, uint64_t *bar, uint32_t parity) {
    return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar, parity, wait_limit(p)));
}

__device__ __forceinline__ void attend_fail(const AttendParams &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

// The second e4m3 number of a pair stands for what the first leaves, at most 1/32 of
// the largest (half a step at 256 is 8).  In an accumulator of its own it is kept
// 32 times as large, which keeps 8 bits of weights down to 2^-15 of the largest.
constexpr float kRest = 32.f;

struct QueryPiece {
    uint32_t hi, lo;   // e4m3 codes of four channels: number and rest
    float factor;      // what a dot with the codes is multiplied by; NaN where the row has infinities or NaN
};

// Channels 4 lane .. 4 lane + 3 of a query row; zeros for a null row.
__device__ __forceinline__ uint2 query_load(const AttendParams &p, const __nv_bfloat16 *row) {
    const int lane = threadIdx.x & 31;
    return row && 4 * lane < p.D ? *reinterpret_cast<const uint2 *>(row + 4 * lane) : make_uint2(0, 0);
}

// They as two e4m3 numbers each, times the power of two that takes the row's largest
// channel to [128, 256); by all lanes of a warp.  SCALED: the rest times kRest.
template <bool SCALED>
__device__ __forceinline__ QueryPiece query_piece(uint2 raw) {
    const float v[4] = {__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xFFFF0000u),
                        __uint_as_float(raw.y << 16), __uint_as_float(raw.y & 0xFFFF0000u)};
    const float m = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
    const bool finite = __all_sync(0xFFFFFFFFu, fabsf(v[0]) <= FLT_MAX && fabsf(v[1]) <= FLT_MAX &&
                                                    fabsf(v[2]) <= FLT_MAX && fabsf(v[3]) <= FLT_MAX);
    const uint32_t mb = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m));
    int e = 134 - (int)(mb >> 23);
    e = mb == 0 || !finite ? 0 : min(max(e, -126), 126);
    const float up = __uint_as_float((uint32_t)(e + 127) << 23);
    QueryPiece r;
    r.hi = r.lo = 0;
    r.factor = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : NAN;
    if (!finite) return r;
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        const float a = v[j] * up, b = v[j + 1] * up;
        const uint32_t q = e4m3x2(a, b);
        const float2 f = __half22float2(half2_of_e4m3((uint16_t)q));
        const float s = SCALED ? kRest : 1.f;
        r.hi |= q << (8 * j);
        r.lo |= e4m3x2((a - f.x) * s, (b - f.y) * s) << (8 * j);
    }
    return r;
}

cudaError_t launch_attend_few(const AttendMaps &maps, const AttendParams &p, int max_new, int sms, cudaStream_t s);
cudaError_t launch_attend_many(const AttendMaps &maps, const AttendParams &p, int max_new, int splits, int paired,
                               cudaStream_t s);

}  // namespace wz
