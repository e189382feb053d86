// What the attention kernels over the paged 8-bit cache share (wz_attend).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "wz_internal.cuh"
#include "wz_kv.cuh"
#include "wz_ptx.cuh"

namespace wz {

constexpr int kATile = 128;                  // tokens of a tile
constexpr int kATileBytes = kATile * 128;    // its codes of one KV head, rows of 128 bytes
constexpr int kFewSlots = 960;               // pieces of items that several CTAs share: two a CTA
constexpr uint64_t kATimeoutNs = 2000000000ull;
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
    int64_t pages;
    int T, B, Hq, heads, G, D, P, max_pages, causal;
    int ctas;                // CTAs that share the work
    float scale2;            // scale * log2(e)
    int *status;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Tokens of q and slots of sequence b; no tokens where its lengths make no sense.
__device__ __forceinline__ int2 attend_lengths(const AttendParams &p, int b) {
    const int x0 = p.cu[b], x1 = p.cu[b + 1];
    const int64_t most = min((int64_t)p.max_pages * p.P, (int64_t)INT32_MAX - 2 * kATile);
    int kv = p.kv_len[b];
    if (kv < 0) kv = 0;
    if (kv > most) kv = (int)most;
    const bool sound = x0 >= 0 && x1 >= x0 && x1 <= p.T;
    return make_int2(sound ? x1 - x0 : 0, kv);
}

// Whether attend_lengths had to change something.
__device__ __forceinline__ bool attend_lengths_sound(const AttendParams &p, int b) {
    const int x0 = p.cu[b], x1 = p.cu[b + 1], kv = p.kv_len[b];
    return x0 >= 0 && x1 >= x0 && x1 <= p.T && kv >= 0 && kv <= (int64_t)p.max_pages * p.P;
}

// Slots that token i of n sees.
__device__ __forceinline__ int attend_visible(const AttendParams &p, int i, int n, int kv) {
    if (!p.causal) return kv;
    const int v = kv - n + i + 1;
    return v < 0 ? 0 : v;
}

// Page of token t of sequence b, or -1.
__device__ __forceinline__ int attend_page(const AttendParams &p, int b, int t) {
    const int pg = p.table[(size_t)b * p.max_pages + t / p.P];
    return pg >= 0 && pg < p.pages ? pg : -1;
}

}  // namespace wz
