// Appending keys and values to the paged 8-bit cache, rotated by position on
// the way (wz_kv_append).
//
// A unit is one page of one sequence that the call writes to.  A CTA takes a unit
// and either the keys and values of some KV heads, as many as its threads have
// registers for, or the queries of some tokens.  Keys and values of a
// page stay in registers between the two things that are done with them: the
// largest magnitude, which decides the page's scale, and the conversion to e4m3, so
// that they are read once.  Each head has warps of its own.  The cosines and sines of
// the CTA's tokens come to shared memory once, by cp.async beside the rows' loads.
// A thread's item is 16 channels of a token as two vectors of 8; the vectors of a
// rotated item hold both halves of its pairs, channels 8j.. and rot/2 + 8j..
//   half split    frequencies 8j .. 8j+7, pairs across the two vectors
//   interleaved   frequencies 4j .. 4j+3 in the first vector, rot/4 + 4j .. in
//                 the second, pairs inside each
// Bound by HBM for prompts and by a chain of dependent loads (lengths, table,
// rows, scale) for single tokens.
#include <algorithm>
#include <cfloat>
#include <cstring>

#include "wz_internal.cuh"
#include "wz_kv.cuh"
#include "wz_ptx.cuh"

namespace wz {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kMaxPage = 128;   // tokens
static_assert(kMaxPage <= kAppendThreads, "a thread for each token of a page");

struct AppendParams {
    uint8_t *cache[2];        // keys, values
    float *scale[2];
    const void *in[3];        // k, v, q
    void *q_out;
    int64_t in_stride[3], q_out_stride;
    int64_t pages;
    int heads, P, D, Hq, T, B;
    int shift, items;         // log2(P), 16-channel items of a head
    uint32_t items_inv, quads_inv;   // for by(): items, groups of four frequencies
    int most;                 // new tokens of a sequence
    int ppb;                  // units a sequence (0: found through cu)
    const int32_t *cu, *start, *table;
    int max_pages;
    const float *rotation;
    int rows, rot, interleaved;
    const int32_t *positions;
    int axes, sec0, sec01;
    int wph;                  // warps of a KV head, a power of two
    int groups, parts;        // CTAs of a unit: groups of KV heads, parts of the queries
    int q_tokens;             // tokens of a part
    int step_j, step_h, step_r;   // kAppendThreads items as items, heads and tokens
    int rows_cta;             // most tokens of a CTA
    int *status;
};

// n / d for n * d < 2^20, inv = 2^20 / d + 1.
__device__ __forceinline__ int by(int n, uint32_t inv) { return (int)((uint32_t)n * inv >> 20); }

struct Vec16 {
    float x[16];
};

// Eight numbers as they are in memory.
template <typename Tin>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *x) const {
        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(r[i] << 16);
            x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
    }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = *reinterpret_cast<const float4 *>(p);
        b = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void get(float *x) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};
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

// Starts the copies of the rotation rows of tokens x0 .. x0 + count - 1 to `rows`
// [count][rot], four frequencies at a time.  `places` [count][axes]: room for the
// tokens' positions, read once, together.  outside[r]: token x0 + r has a position that the
// table does not, and neither key nor query of it is written; true for a thread that found one.
__device__ __forceinline__ bool fetch_angles(const AppendParams &p, float *rows, int *places, uint8_t *outside, int x0,
                                             int slot0, int count) {
    const int half = p.rot >> 1, quads = half >> 2;
    if (p.positions) {
        for (int at = threadIdx.x; at < count * p.axes; at += kAppendThreads)
            places[at] = p.positions[(size_t)x0 * p.axes + at];
        __syncthreads();
    }
    auto in_table = [&](int pos) { return pos >= 0 && pos < p.rows; };
    bool found = false;
    if (const int r = threadIdx.x; r < count) {   // a page has fewer tokens than the CTA threads
        if (!p.positions)
            found = !in_table(slot0 + r);
        else if (p.axes == 3)   // axes that some frequency takes
            found = (p.sec0 > 0 && !in_table(places[3 * r])) ||
                    (p.sec01 > p.sec0 && !in_table(places[3 * r + 1])) || (half > p.sec01 && !in_table(places[3 * r + 2]));
        else
            found = !in_table(places[r]);
        outside[r] = found;
        if (found) kv_report(p.status);
    }
    auto row_of = [&](int r, int f) {   // of frequency f of token x0 + r
        int pos = slot0 + r;
        if (p.positions) pos = p.axes == 3 ? places[3 * r + (f >= p.sec0) + (f >= p.sec01)] : places[r];
        return p.rotation + (size_t)(in_table(pos) ? pos : 0) * p.rot;
    };
    for (int at = threadIdx.x; at < count * quads; at += kAppendThreads) {
        const int r = by(at, p.quads_inv), f = 4 * (at - r * quads);
        float *dst = rows + r * p.rot + f;
        if (p.axes == 3 && ((f < p.sec0 && f + 3 >= p.sec0) || (f < p.sec01 && f + 3 >= p.sec01))) {
            for (int i = 0; i < 4; ++i) {   // sections that meet inside the four
                const float *src = row_of(r, f + i) + f + i;
                ptx::copy_async4(dst + i, src);
                ptx::copy_async4(dst + half + i, src + half);
            }
        } else {
            const float *src = row_of(r, f) + f;
            ptx::copy_async16_l1(dst, src);   // few rows serve most tokens of a grid
            ptx::copy_async16_l1(dst + half, src + half);
        }
    }
    return found;
}

// Two products.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// Turns the pairs (a.x, b.x) and (a.y, b.y).  Products and sums are rounded one by one,
// so that the result does not depend on how a compiler contracts them (packed sums of
// packed products come out contracted).
__device__ __forceinline__ void turn(float2 &a, float2 &b, float2 c, float2 s) {
    const float2 ac = mul2(a, c), bs = mul2(b, s), bc = mul2(b, c), as = mul2(a, s);
    a = {__fsub_rn(ac.x, bs.x), __fsub_rn(ac.y, bs.y)};
    b = {__fadd_rn(bc.x, as.x), __fadd_rn(bc.y, as.y)};
}

// Turns rotated item j by a token's row of angles.
template <bool INTER>
__device__ __forceinline__ void turn_item(const AppendParams &p, Vec16 &v, const float *row, int j) {
    const int half = p.rot >> 1;
    const int f[2] = {INTER ? 4 * j : 8 * j, INTER ? (half >> 1) + 4 * j : 8 * j + 4};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float4 c4 = *reinterpret_cast<const float4 *>(row + f[q]);
        const float4 s4 = *reinterpret_cast<const float4 *>(row + half + f[q]);
        const float2 c[2] = {{c4.x, c4.y}, {c4.z, c4.w}}, s[2] = {{s4.x, s4.y}, {s4.z, s4.w}};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // pairs of the first two and the last two frequencies of the four
            float *w = v.x + (INTER ? 8 * q + 4 * i : 4 * q + 2 * i);
            float *z = INTER ? w + 1 : w + 8;
            const int step = INTER ? 2 : 1;
            float2 a = {w[0], w[step]}, b = {z[0], z[step]};
            turn(a, b, c[i], s[i]);
            w[0] = a.x; w[step] = a.y;
            z[0] = b.x; z[step] = b.y;
        }
    }
}

__device__ __forceinline__ uint2 pack8(const float *x, float inv) {
    uint2 r;
    r.x = e4m3x2(x[0] * inv, x[1] * inv) | (e4m3x2(x[2] * inv, x[3] * inv) << 16);
    r.y = e4m3x2(x[4] * inv, x[5] * inv) | (e4m3x2(x[6] * inv, x[7] * inv) << 16);
    return r;
}

// Keys and values of `count` tokens from row `row0` of a page on, a head of each wph
// warps.  `page_at` is read beside the rows.
template <typename Tin, int IT, bool INTER>
__device__ __forceinline__ void append_page(const AppendParams &p, float *angles, int *places, uint8_t *outside,
                                            int group, int x0, int slot0, int count, int row0,
                                            const int32_t *page_at) {
    constexpr bool kBoth = IT * sizeof(Tin) <= 4;   // registers for the values' rows beside the keys'
    __shared__ uint32_t warp_max[2][kAppendThreads / 32];
    const int items = p.items;
    const int warp = threadIdx.x >> 5, first_warp = warp & ~(p.wph - 1), width = p.wph * 32;
    const int lane = threadIdx.x - first_warp * 32;   // among the head's threads
    const int head = group * (kAppendThreads / 32 / p.wph) + first_warp / p.wph;
    const bool mine = head < p.heads;
    Raw8<Tin> a[kBoth ? 2 : 1][IT], b[kBoth ? 2 : 1][IT];
    auto load = [&](int role, Raw8<Tin> (&lo)[IT], Raw8<Tin> (&hi)[IT]) {
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            if (t > 0 && t * width >= count * items) break;
            const int at = lane + t * width, r = by(at, p.items_inv), j = at - r * items;
            // Every thread loads, past the rows the first: under a condition loads wait for one
            // another (18,699 tokens 63 us, 32 x 577 in f32 48; so 58 and 44).
            const int2 ch = item_channels(p, role ? 0 : p.rot, j);
            const bool is = mine && r < count;
            const Tin *src = static_cast<const Tin *>(p.in[role]) + (size_t)(x0 + (is ? r : 0)) * p.in_stride[role] +
                             (is ? head * p.D : 0);
            lo[t].load(src + (is ? ch.x : 0));
            hi[t].load(src + (is ? ch.y : 0));
        }
    };
    const int page = page_at ? *page_at : -1;
    load(0, a[0], b[0]);
    if (kBoth) load(1, a[kBoth], b[kBoth]);
    const bool found = p.rot && fetch_angles(p, angles, places, outside, x0, slot0, count);
    if (page < 0 || page >= p.pages) {
        ptx::copy_async_wait_all();
        kv_report(p.status);
        return;
    }
    const size_t block = (size_t)page * p.heads + (mine ? head : 0);
    const float olds[2] = {p.scale[0][block], p.scale[1][block]};
    ptx::copy_async_wait_all();
    const bool some_outside = __syncthreads_or(found);
    uint32_t absent = 0;   // this thread's items whose key is left out
    if (some_outside)
        for (int t = 0; t < IT; ++t) {
            const int r = by(lane + t * width, p.items_inv);
            if (r < count && outside[r]) absent |= 1u << t;
        }
#pragma unroll
    for (int role = 0; role < 2; ++role) {
        const int rot = role ? 0 : p.rot;
        auto takes = [&](int t, int r) { return mine && r < count && !(role == 0 && (absent >> t & 1u)); };
        uint8_t *dst = p.cache[role] + block * (size_t)(p.P * p.D);
        const float old = olds[role];
        if (!kBoth && role) load(1, a[0], b[0]);
        Vec16 v[IT];
        float most = 0.f;
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int at = lane + t * width, r = by(at, p.items_inv), j = at - r * items;
            if (takes(t, r)) {
                a[kBoth ? role : 0][t].get(v[t].x);
                b[kBoth ? role : 0][t].get(v[t].x + 8);
                if (j < rot >> 4) turn_item<INTER>(p, v[t], angles + r * p.rot, j);
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(v[t].x[i]));   // leaves out NaN
            }
        }
        if (most > FLT_MAX) {   // and infinities have no say in the scale either
            most = 0.f;
#pragma unroll
            for (int t = 0; t < IT; ++t) {
                const int at = lane + t * width;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float m = fabsf(v[t].x[i]);
                    if (takes(t, by(at, p.items_inv)) && m <= FLT_MAX) most = fmaxf(most, m);
                }
            }
        }
        const uint32_t wm = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));   // >= 0: bits order as floats
        if ((threadIdx.x & 31) == 0) warp_max[role][warp] = wm;
        __syncthreads();
        uint32_t all = 0;
        for (int w = 0; w < p.wph; ++w) all = max(all, warp_max[role][first_warp + w]);
        const float fit = fitting_scale(all);
        const float now = row0 == 0 ? fit : fmaxf(old, fit);
        const float inv = 1.f / now;
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int at = lane + t * width, r = by(at, p.items_inv), j = at - r * items;
            if (takes(t, r) && wz_in_range(p.status, row0 + r < p.P)) {
                const int2 ch = item_channels(p, rot, j);
                uint8_t *d = dst + (row0 + r) * p.D;
                *reinterpret_cast<uint2 *>(d + ch.x) = pack8(v[t].x, inv);
                *reinterpret_cast<uint2 *>(d + ch.y) = pack8(v[t].x + 8, inv);
            }
        }
        if (mine && row0 > 0 && now > old) {
            // the rows that the page holds already, in the larger scale
            const float ratio = old * inv;
            for (int at = lane; at < row0 * items; at += width) {
                uint4 *d = reinterpret_cast<uint4 *>(dst + 16 * at);
                const uint4 w = *d;
                *d = make_uint4(e4m3x4_times(w.x, ratio), e4m3x4_times(w.y, ratio), e4m3x4_times(w.z, ratio),
                                e4m3x4_times(w.w, ratio));
            }
        }
        if (mine && lane == 0) p.scale[role][block] = now;   // every thread has read `old` before the barriers
    }
}

// Queries of tokens part * q_tokens .. of `count`: their heads lie side by side, so
// that the CTA reads and writes whole rows from one end to the other.
template <typename Tin, bool INTER>
__device__ __forceinline__ void rotate_queries(const AppendParams &p, float *angles, int *places, uint8_t *outside,
                                               int part, int x0, int slot0, int count) {
    constexpr int kAhead = 2;   // items of a thread whose loads are in flight
    const int items = p.items, heads = p.Hq;
    const int r0 = part * p.q_tokens, tokens = min(count - r0, p.q_tokens);
    if (tokens <= 0) return;
    x0 += r0;
    struct Place {
        int r, h, j;
    };
    auto advance = [&](Place &w) {   // kAppendThreads items on
        w.j += p.step_j;
        w.h += p.step_h;
        w.r += p.step_r;
        if (w.j >= items) {
            w.j -= items;
            ++w.h;
        }
        if (w.h >= heads) {
            w.h -= heads;
            ++w.r;
        }
    };
    Place at{0, by(threadIdx.x, p.items_inv), 0};
    at.j = (int)threadIdx.x - at.h * items;
    if (at.h >= heads) {
        at.r = at.h / heads;
        at.h -= at.r * heads;
    }
    Place ahead = at;
    Raw8<Tin> a[kAhead], b[kAhead];
    auto load = [&](int u) {
        const int2 ch = item_channels(p, p.rot, ahead.j);   // past the rows the first, as above
        const bool is = ahead.r < tokens;
        const Tin *src = static_cast<const Tin *>(p.in[2]) + (size_t)(x0 + (is ? ahead.r : 0)) * p.in_stride[2] +
                         (is ? ahead.h * p.D : 0);
        a[u].load(src + (is ? ch.x : 0));
        b[u].load(src + (is ? ch.y : 0));
        advance(ahead);
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(u);
    bool some_outside = false;
    if (p.rot) {
        const bool found = fetch_angles(p, angles, places, outside, x0, slot0 + r0, tokens);
        ptx::copy_async_wait_all();
        some_outside = __syncthreads_or(found);
    }
    while (at.r < tokens) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (at.r < tokens) {
                Vec16 v;
                a[u].get(v.x);
                b[u].get(v.x + 8);
                if (at.j < p.rot >> 4) turn_item<INTER>(p, v, angles + at.r * p.rot, at.j);
                const int2 ch = item_channels(p, p.rot, at.j);
                const size_t x = (size_t)(x0 + at.r);
                Tin *dst = static_cast<Tin *>(p.q_out) + x * p.q_out_stride + (size_t)at.h * p.D;
                if (!(some_outside && outside[at.r]) && wz_in_range(p.status, x < (size_t)p.T)) {
                    store8(dst + ch.x, v.x);
                    store8(dst + ch.y, v.x + 8);
                }
            }
            load(u);
            advance(at);
        }
    }
}

}  // namespace

// Grid: units x (groups of KV heads, parts of the queries), a
// unit's CTAs one after the other: they share its tokens' rows, and so DRAM pages.  18,699
// tokens of 28 + 4 + 4 heads x 128, at positions (t, i, j): 58 us (5.6 TB/s); 24 more with
// the units of one head after those of another.
template <typename Tin, int IT, bool INTER>
__global__ void __launch_bounds__(kAppendThreads, IT == 4 ? 2 : sizeof(Tin) == 2 ? 4 : 3)
kv_append_kernel(const __grid_constant__ AppendParams p) {
    extern __shared__ __align__(16) float angles[];      // [rows][rot], then the positions
    __shared__ uint8_t outside[kMaxPage];
    int *places = reinterpret_cast<int *>(angles + p.rows_cta * p.rot);
    pdl_wait();
    pdl_trigger();
    const int share = p.groups + p.parts, unit = (int)blockIdx.x / share, place = (int)blockIdx.x - unit * share;
    int b, j;
    if (p.ppb) {
        b = unit / p.ppb;
        j = unit - b * p.ppb;
    } else {
        // sequence b has units cu[b] / P + 2b up to the next one's: enough for its
        // pages wherever it starts, and known without the sequences before it
        b = kv_find_sequence(p.cu, p.B, unit, p.shift);
        j = unit - ((p.cu[b] >> p.shift) + 2 * b);
    }
    const int x0 = p.cu[b], x1 = p.cu[b + 1], s0 = p.start[b];
    if (x0 < 0 || x1 < x0 || x1 > p.T || s0 < 0 || s0 > INT32_MAX - (x1 - x0) - p.P || j < 0) {
        kv_report(p.status);
        return;
    }
    if (x0 == x1) return;
    if (j == 0 && x1 - x0 > p.most) kv_report(p.status);   // more tokens than max_new: the rest is left out
    const int col = (s0 >> p.shift) + j, end = s0 + min(x1 - x0, p.most);
    const int64_t first = (int64_t)col << p.shift;
    const int lo = first > s0 ? (int)min(first, (int64_t)end) : s0;
    const int hi = (int)min(first + p.P, (int64_t)end);
    if (lo >= hi) return;
    const int x = x0 + (lo - s0);
    if (place >= p.groups)
        rotate_queries<Tin, INTER>(p, angles, places, outside, place - p.groups, x, lo, hi - lo);
    else
        append_page<Tin, IT, INTER>(p, angles, places, outside, place, x, lo, hi - lo, (int)(lo - first),
                                    col < p.max_pages ? p.table + (size_t)b * p.max_pages + col : nullptr);
}

template <typename Tin, bool INTER>
static const void *append_kernel(int it) {
    return it == 1 ? (const void *)kv_append_kernel<Tin, 1, INTER>
                   : it == 2 ? (const void *)kv_append_kernel<Tin, 2, INTER>
                             : (const void *)kv_append_kernel<Tin, 4, INTER>;
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
    while (1 << p.shift < p.P) ++p.shift;
    p.items = p.D >> 4;
    p.items_inv = (1u << 20) / p.items + 1;
    p.Hq = a.Hq;
    p.T = (int)a.T; p.B = a.B;
    p.cu = a.cu; p.start = a.start; p.table = a.page_table; p.max_pages = a.max_pages;
    if (a.rotation) {
        p.rotation = a.rotation; p.rows = (int)a.rotation_rows; p.rot = a.rot; p.interleaved = a.interleaved != 0;
        p.positions = a.positions; p.axes = a.axes;
        p.quads_inv = (1u << 20) / (p.rot >> 3) + 1;
        p.sec0 = a.section[0]; p.sec01 = a.section[0] + a.section[1];
    }
    p.status = a.device_status;
    // pages that a sequence of max_new tokens can reach, wherever it starts
    const int most = p.most = a.max_new ? std::min(a.max_new, p.T) : p.T;
    const int64_t ppb = ((int64_t)most + p.P - 2) / p.P + 1;
    int64_t units = (int64_t)p.T / p.P + 2 * (int64_t)p.B;
    if (ppb * p.B <= units) {
        p.ppb = (int)ppb;
        units = ppb * p.B;
    }
    // The items of a page's head: two to a thread, or one where 32 are all; four only
    // for the largest pages.
    const int rows = std::min(p.P, most), items = p.P * p.items;
    const int it = items <= 32 ? 1 : items <= 2 * kAppendThreads ? 2 : 4;
    p.wph = 1;
    while (p.wph * 32 * it < items) p.wph *= 2;
    const int kv_heads = (kAppendThreads / 32) / p.wph;
    p.groups = (p.heads + kv_heads - 1) / kv_heads;
    if (a.q) {   // eight items of a query to a thread
        p.q_tokens = std::max(1, std::min(rows, 8 * kAppendThreads / (a.Hq * p.items)));
        p.parts = (rows + p.q_tokens - 1) / p.q_tokens;
        p.q_tokens = (rows + p.parts - 1) / p.parts;
        p.step_j = kAppendThreads % p.items;
        p.step_h = kAppendThreads / p.items % p.Hq;
        p.step_r = kAppendThreads / p.items / p.Hq;
    }
    p.rows_cta = rows;
    const size_t smem = (size_t)rows * (p.rot + (p.positions ? p.axes : 0)) * sizeof(float);
    const void *fn = a.dtype == WZ_DTYPE_BF16
                         ? (p.interleaved ? append_kernel<__nv_bfloat16, true>(it) : append_kernel<__nv_bfloat16, false>(it))
                         : (p.interleaved ? append_kernel<float, true>(it) : append_kernel<float, false>(it));
    // 48 KB a CTA need no leave, the kernel's static arrays included; asking takes host time,
    // and calls of a few tokens, which that matters to, have less than this
    cudaError_t e = smem > 32 * 1024 ? allow_smem(fn, smem) : cudaSuccess;
    if (e != cudaSuccess) return e;
    void *args[] = {&p};
    const int64_t grid = units * (p.groups + p.parts);
    if (grid > INT32_MAX) return cudaErrorInvalidValue;
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kAppendThreads), smem, s, args, true);
}

}  // namespace wz
