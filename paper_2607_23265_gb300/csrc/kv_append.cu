// Appending keys and values to the paged 8-bit cache, rotated by position on
// the way (wz_kv_append).
//
// A unit is one page of one sequence that the call writes to; a CTA takes a
// unit and a KV head and either its keys, its values or the queries of the
// head's group.  Keys and values of a page stay in registers between the two
// things that are done with them: the largest magnitude, which decides the
// page's scale, and the conversion to e4m3, so that they are read once.
// A thread's item is 16 channels of a token as two vectors of 8; the vectors of a
// rotated item hold both halves of its pairs, channels 8j.. and rot/2 + 8j..
//   half split    frequencies 8j .. 8j+7, pairs across the two vectors
//   interleaved   frequencies 4j .. 4j+3 in the first vector, rot/4 + 4j .. in
//                 the second, pairs inside each
// Bound by HBM for prompts and by a chain of dependent loads (lengths, table,
// rows, scale) for single tokens.
#include <cfloat>
#include <cstring>

#include "wz_internal.cuh"
#include "wz_kv.cuh"

namespace wz {

namespace {

struct AppendParams {
    uint8_t *cache[2];        // keys, values
    float *scale[2];
    const void *in[3];        // k, v, q
    void *q_out;
    int64_t in_stride[3], q_out_stride;
    int64_t pages;
    int heads, P, D, G, T, B;
    int ppb;                  // units a sequence (0: found through cu)
    const int32_t *cu, *start, *table;
    int max_pages;
    const float *rotation;
    int rows, rot, interleaved;
    const int32_t *positions;
    int axes, sec0, sec01;
    int *status;
};

struct Vec16 {
    float x[16];
};

__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *x) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float *x) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float *p, const float *x) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// First channels of the two vectors of item j.
__device__ __forceinline__ int2 item_channels(const AppendParams &p, int rot, int j) {
    const int pairs = rot >> 4;
    const int a = j < pairs ? 8 * j : rot + 16 * (j - pairs);
    return make_int2(a, j < pairs ? (rot >> 1) + 8 * j : a + 8);
}

struct Angles {
    float c[8], s[8];
};

// Position of frequency f of token x (its slot where no positions are given).
__device__ __forceinline__ int position(const AppendParams &p, int x, int slot, int f) {
    int pos = slot;
    if (p.axes == 3)
        pos = p.positions[(size_t)x * 3 + (f >= p.sec0) + (f >= p.sec01)];
    else if (p.positions)
        pos = p.positions[x];
    if (pos < 0 || pos >= p.rows) {
        kv_report(p.status);
        pos = 0;
    }
    return pos;
}

// Cosines and sines of rotated item j of token x: four frequencies at fa, four at fb.
__device__ __forceinline__ Angles item_angles(const AppendParams &p, int x, int slot, int j) {
    const int half = p.rot >> 1;
    const int f[2] = {p.interleaved ? 4 * j : 8 * j, p.interleaved ? (half >> 1) + 4 * j : 8 * j + 4};
    Angles g;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const bool split = p.axes == 3 && ((f[v] < p.sec0 && f[v] + 3 >= p.sec0) ||
                                           (f[v] < p.sec01 && f[v] + 3 >= p.sec01));
        if (split) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *row = p.rotation + (size_t)position(p, x, slot, f[v] + i) * p.rot;
                g.c[4 * v + i] = row[f[v] + i];
                g.s[4 * v + i] = row[half + f[v] + i];
            }
        } else {
            const float *row = p.rotation + (size_t)position(p, x, slot, f[v]) * p.rot;
            const float4 c = *reinterpret_cast<const float4 *>(row + f[v]);
            const float4 s = *reinterpret_cast<const float4 *>(row + half + f[v]);
            g.c[4 * v] = c.x; g.c[4 * v + 1] = c.y; g.c[4 * v + 2] = c.z; g.c[4 * v + 3] = c.w;
            g.s[4 * v] = s.x; g.s[4 * v + 1] = s.y; g.s[4 * v + 2] = s.z; g.s[4 * v + 3] = s.w;
        }
    }
    return g;
}

// Turns the pair (a, b).  Products and sums are rounded one by one, so that the
// result does not depend on how a compiler contracts them.
__device__ __forceinline__ void turn(float &a, float &b, float c, float s) {
    const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
    b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
    a = x;
}

__device__ __forceinline__ void turn_item(Vec16 &v, const Angles &g, bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(v.x[2 * i], v.x[2 * i + 1], g.c[i], g.s[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(v.x[i], v.x[8 + i], g.c[i], g.s[i]);
    }
}

__device__ __forceinline__ uint2 pack8(const float *x, float inv) {
    uint2 r;
    r.x = e4m3x2(x[0] * inv, x[1] * inv) | (e4m3x2(x[2] * inv, x[3] * inv) << 16);
    r.y = e4m3x2(x[4] * inv, x[5] * inv) | (e4m3x2(x[6] * inv, x[7] * inv) << 16);
    return r;
}

// Keys or values of `count` tokens from row `row0` of a page on.
template <typename Tin, int IT>
__device__ __forceinline__ void append_page(const AppendParams &p, int role, int head, int x0, int slot0, int count,
                                            int row0, int64_t page) {
    __shared__ uint32_t warp_max[8];
    const int items = p.D >> 4, rot = role == 0 ? p.rot : 0;
    const size_t block = (size_t)page * p.heads + head;
    uint8_t *dst = p.cache[role] + block * (size_t)(p.P * p.D);
    const float old = p.scale[role][block];
    Vec16 v[IT];
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int at = (int)threadIdx.x + t * (int)blockDim.x;
        const int r = at / items, j = at - r * items;
        if (r < count) {
            const int2 ch = item_channels(p, rot, j);
            const Tin *src = static_cast<const Tin *>(p.in[role]) + (size_t)(x0 + r) * p.in_stride[role] +
                             (size_t)head * p.D;
            load8(src + ch.x, v[t].x);
            load8(src + ch.y, v[t].x + 8);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[t].x[i] = 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int at = (int)threadIdx.x + t * (int)blockDim.x;
        const int r = at / items, j = at - r * items;
        if (r < count && j < rot >> 4) turn_item(v[t], item_angles(p, x0 + r, slot0 + r, j), p.interleaved);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float m = fabsf(v[t].x[i]);
            most = fmaxf(most, m <= FLT_MAX ? m : 0.f);   // infinities and NaN have no say in the scale
        }
    }
    const uint32_t wm = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));   // order of bits = order of floats >= 0
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = wm;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) all = max(all, warp_max[w]);
    const float fit = fitting_scale(all);
    const float now = row0 == 0 ? fit : fmaxf(old, fit);
    const float inv = 1.f / now;
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int at = (int)threadIdx.x + t * (int)blockDim.x;
        const int r = at / items, j = at - r * items;
        if (r < count && wz_in_range(p.status, row0 + r < p.P)) {
            const int2 ch = item_channels(p, rot, j);
            uint8_t *d = dst + (row0 + r) * p.D;
            *reinterpret_cast<uint2 *>(d + ch.x) = pack8(v[t].x, inv);
            *reinterpret_cast<uint2 *>(d + ch.y) = pack8(v[t].x + 8, inv);
        }
    }
    if (row0 > 0 && now > old) {
        // the rows that the page holds already, in the larger scale
        const float ratio = old * inv;
        for (int at = threadIdx.x; at < row0 * items; at += blockDim.x) {
            uint4 *d = reinterpret_cast<uint4 *>(dst + 16 * at);
            const uint4 w = *d;
            *d = make_uint4(e4m3x4_times(w.x, ratio), e4m3x4_times(w.y, ratio), e4m3x4_times(w.z, ratio),
                            e4m3x4_times(w.w, ratio));
        }
    }
    if (threadIdx.x == 0) p.scale[role][block] = now;   // every thread has read `old` before the barrier
}

// The group's queries of `count` tokens.
template <typename Tin>
__device__ __forceinline__ void rotate_queries(const AppendParams &p, int head, int x0, int slot0, int count) {
    const int items = p.D >> 4;
    for (int at = threadIdx.x; at < count * items; at += blockDim.x) {
        const int r = at / items, j = at - r * items;
        const int2 ch = item_channels(p, p.rot, j);
        const size_t x = (size_t)(x0 + r);
        const Tin *src = static_cast<const Tin *>(p.in[2]) + x * p.in_stride[2] + (size_t)head * p.G * p.D;
        Tin *dst = static_cast<Tin *>(p.q_out) + x * p.q_out_stride + (size_t)head * p.G * p.D;
        const bool turned = j < p.rot >> 4;
        Angles g{};
        if (turned) g = item_angles(p, x0 + r, slot0 + r, j);
#pragma unroll 4
        for (int h = 0; h < p.G; ++h) {
            Vec16 v;
            load8(src + (size_t)h * p.D + ch.x, v.x);
            load8(src + (size_t)h * p.D + ch.y, v.x + 8);
            if (turned) turn_item(v, g, p.interleaved);
            if (wz_in_range(p.status, x < (size_t)p.T)) {
                store8(dst + (size_t)h * p.D + ch.x, v.x);
                store8(dst + (size_t)h * p.D + ch.y, v.x + 8);
            }
        }
    }
}

}  // namespace

// Grid: units x KV heads x (keys, values, queries).
template <typename Tin, int IT>
__global__ void __launch_bounds__(256) kv_append_kernel(AppendParams p) {
    pdl_wait();
    pdl_trigger();
    int b, j;
    if (p.ppb) {
        b = (int)blockIdx.x / p.ppb;
        j = (int)blockIdx.x - b * p.ppb;
    } else {
        // sequence b has units cu[b] / P + 2b up to the next one's: enough for its
        // pages wherever it starts, and known without the sequences before it
        b = kv_find_sequence(p.cu, p.B, (int)blockIdx.x, p.P);
        j = (int)blockIdx.x - (p.cu[b] / p.P + 2 * b);
    }
    const int x0 = p.cu[b], x1 = p.cu[b + 1], s0 = p.start[b];
    if (x0 < 0 || x1 < x0 || x1 > p.T || s0 < 0 || s0 > INT32_MAX - (x1 - x0) - p.P || j < 0) {
        kv_report(p.status);
        return;
    }
    if (x0 == x1) return;
    const int col = s0 / p.P + j, end = s0 + (x1 - x0);
    if (j == 0 && p.ppb && (end + p.P - 1) / p.P - col > p.ppb) kv_report(p.status);   // more tokens than max_new
    const int64_t first = (int64_t)col * p.P;
    const int lo = first > s0 ? (int)min(first, (int64_t)end) : s0;
    const int hi = (int)min(first + p.P, (int64_t)end);
    if (lo >= hi) return;
    const int x = x0 + (lo - s0), role = blockIdx.z, head = blockIdx.y;
    if (role == 2) {
        rotate_queries<Tin>(p, head, x, lo, hi - lo);
        return;
    }
    const int64_t page = col < p.max_pages ? p.table[(size_t)b * p.max_pages + col] : -1;
    if (page < 0 || page >= p.pages) {
        kv_report(p.status);
        return;
    }
    append_page<Tin, IT>(p, role, head, x, lo, hi - lo, (int)(lo - first), page);
}

template <typename Tin>
static const void *append_kernel(int it) {
    return it == 1 ? (const void *)kv_append_kernel<Tin, 1>
                   : it == 2 ? (const void *)kv_append_kernel<Tin, 2> : (const void *)kv_append_kernel<Tin, 4>;
}

cudaError_t launch_kv_append(const wz_kv_append_args &a, cudaStream_t s) {
    AppendParams p;
    memset(&p, 0, sizeof(p));
    p.cache[0] = static_cast<uint8_t *>(a.cache.k);
    p.cache[1] = static_cast<uint8_t *>(a.cache.v);
    p.scale[0] = a.cache.k_scale;
    p.scale[1] = a.cache.v_scale;
    p.in[0] = a.k; p.in[1] = a.v; p.in[2] = a.q;
    p.in_stride[0] = a.k_stride; p.in_stride[1] = a.v_stride; p.in_stride[2] = a.q_stride;
    p.q_out = a.q_out; p.q_out_stride = a.q_out_stride;
    p.pages = a.cache.pages; p.heads = a.cache.heads; p.P = a.cache.page_tokens; p.D = a.cache.D;
    p.G = a.q ? a.Hq / p.heads : 0;
    p.T = (int)a.T; p.B = a.B;
    p.cu = a.cu; p.start = a.start; p.table = a.page_table; p.max_pages = a.max_pages;
    if (a.rotation) {
        p.rotation = a.rotation; p.rows = (int)a.rotation_rows; p.rot = a.rot; p.interleaved = a.interleaved != 0;
        p.positions = a.positions; p.axes = a.axes;
        p.sec0 = a.section[0]; p.sec01 = a.section[0] + a.section[1];
    }
    p.status = a.device_status;
    // pages that a sequence of max_new tokens can reach, wherever it starts
    const int most = a.max_new ? a.max_new : p.T;
    const int64_t ppb = ((int64_t)most + p.P - 2) / p.P + 1;
    int64_t units = (int64_t)p.T / p.P + 2 * (int64_t)p.B;
    if (ppb * p.B <= units) {
        p.ppb = (int)ppb;
        units = ppb * p.B;
    }
    const int threads = p.P > 64 ? 256 : 128;
    const int items = p.P * (p.D >> 4);
    const int it = items <= threads ? 1 : items <= 2 * threads ? 2 : 4;
    const void *fn = a.dtype == WZ_DTYPE_BF16 ? append_kernel<__nv_bfloat16>(it) : append_kernel<float>(it);
    void *args[] = {&p};
    return launch_kernel(fn, dim3((unsigned)units, (unsigned)p.heads, a.q ? 3u : 2u), dim3(threads), 0, s, args, true);
}

}  // namespace wz
