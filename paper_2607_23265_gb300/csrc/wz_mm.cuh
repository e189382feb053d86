// Matrix products of a decoder layer (wz_linear, wz_gated and their backward
// passes): what their kernels share.
//
//   D[i][j] = sum_k A[i][k] B[j][k],  A and B bf16, fp32 accumulation
//
// An operand is either K-major (k is contiguous in memory) or MN-major (its row
// index is), so that one layout in memory serves the forward product and both
// gradients: x W^T reads both K-major, d W reads W MN-major, d^T x both.
#pragma once

#include <cuda.h>

#include "wz_internal.cuh"
#include "wz_ptx.cuh"

namespace wz {

constexpr int kMmMaps = 8;
constexpr int kMmProblems = 3;
constexpr uint64_t kMmTimeoutNs = 2000000000ull;
// The tensor cores add 16 products and the sum so far at a time, each cut off two bits behind the 24 of a sum (which is the
// result, cut off again), so that long sums come out a little too small: by 2.5 units of the last place at an addition
// on average, 1.1e-5 of 4,224 terms of one sign and 5.8e-5 of 14,336 (two sums: 2.9e-6 and 2.2e-5); bias gradients, which are f32 and made of slopes at such sums, are 1.3e-6 off in norm
// with K = 1,152, 4.6e-6 with 3,584 and 9.4e-6 with 14,336 (bf16 results do not notice).  Two sums, of the even and of the
// odd steps of 64 along K, halve that (6.5e-7 with 1,152, 4.6e-6 with 14,336).  Products that are formed again for their
// slopes keep two in mm_pair.cu, in tiles of half the rows, when they have more steps than this or it costs next to
// nothing, and have a share of K for each as many steps in mm_few.cu.
constexpr int kLongSteps = 64;
// Pairs of SMs that row tiles and both gradients are planned for: a constant, so that workspace sizes and the cut of
// gradients do not depend on the device.  (Which kernel a product takes does: plan_mm_few asks for its SMs and places.)
constexpr int kPlanPairs = 76;

struct MmMaps {
    CUtensorMap m[kMmMaps];   // 2D, boxes 64 wide with 128-byte swizzle
};

// What is done with the sums.
enum MmEpilogue : int {
    kMmStore = 0,     // out = act(p) + residual, p = sum + bias; p kept in pre[0]
    kMmGated = 1,     // out = act(g) u; g and u kept in pre[0], pre[1]
    kMmSlope = 2,     // out = dy act'(p), and its sums over some rows in part[0]
    kMmGatedSlope = 3 // out = dout u act'(g), out2 = dout act(g), and their sums
};

__host__ __device__ constexpr bool mm_both(int epi) { return epi == kMmGated || epi == kMmGatedSlope; }

// Division of 0 .. 2^31 - 1 by a number that the host knows: n / d = (high(n mul) + n) >> shift with
// 2^(shift - 1) < d <= 2^shift and mul = 2^32 (2^shift - d) / d + 1 (Granlund and Montgomery).
struct MmDivisor {
    uint32_t mul, shift;
    void set(uint32_t d) {
        shift = 0;
        while (((uint64_t)1 << shift) < d) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ int divide(int n) const {
        return (int)((__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift);
    }
};

// A matrix in memory: [rows][cols], rows `stride` elements apart.
struct MmOperand {
    const void *base;
    int64_t rows;
    int cols;
    int64_t stride;
};

// One product of a launch.  With two segments the second continues the sums; in a gated
// launch b[0] and b[1] are the gate's and the up projection's weights.
struct MmProblem {
    int M, N;              // rows and columns of D
    int segments, steps;   // K segments of `steps` steps of 64
    int a_mn, b_mn;        // operands MN-major
    __nv_bfloat16 *out;    // [M] rows of N
    int64_t out_stride;
    MmOperand from_a[2], from_b[2];   // host: the operands
    int64_t room_rows, room_sums;     // rows at out and floats at sums that there is room for (the checked build's kernels look)
    // set by the launch
    int a[2], b[2];        // their tensor maps
    float *sums;           // pairs, K shared: [split][M][N] sums of the shares
    int tile_m;            // rows of a tile; pairs: 0 lets the launch choose them
    int mt, nt, tiles;     // tiles along M and N, and all of them (with shared K, of all shares)
    MmDivisor by_mt;       // mm_few.cu
    MmDivisor by_group, by_last;   // pairs: tiles of a group of row tiles, row tiles of the last one
    int head, from, skip;  //   its first tiles, for the pairs from one on, the turn's first
    int box_rows;          // a CTA's
    int split;             // shares of a tile's K
    int share, more;       //   K steps of a share, shares that have one more
};

// Bias gradients: db[i][n] = the sum of part[i][.][n], or of dy's rows.
struct MmSums {
    const float *part[2];
    float *db[2];                           // null: not wanted
    int64_t part_rows;
    const __nv_bfloat16 *dy;
    int64_t dy_stride, dy_rows;
    int N;
    int blocks;                             // of 32 columns of either, all together; 0: none
};

struct MmArgs {
    MmProblem prob[kMmProblems];
    MmSums sums;                            // mm_pair.cu, kMmStore: added up before a CTA's first tile
    int problems;
    int act;                                // WZ_ACT_*
    const float *bias[2];                   // [N]; null: none
    const __nv_bfloat16 *residual;          // kMmStore; null: none
    const __nv_bfloat16 *dy;                // the slopes' factor
    __nv_bfloat16 *pre[2];                  // kept products; null: none
    __nv_bfloat16 *out2;                    // kMmGatedSlope
    float *part[2];                         // [some rows][N] sums over rows; null: none
    int64_t room_part;                      // floats at each of them
    int64_t residual_stride, dy_stride, pre_stride[2], out2_stride;
    int maps;                               // tensor maps in use
    int second;                             // pairs: columns from the even steps' sums to the odd ones'; 0: one
    int cluster;                            // mm_few.cu: CTAs of a cluster, the ring,
    MmDivisor by_cluster;
    int stages, stage_bytes, ring_bytes;
    int sums_bytes;                         //   joined sums, at its end where they are
    int apart;                              //   apart from it,
    int chunk;                              //   rows of sums in shared memory at a time
    int *status;
    uint64_t wait_ns;
};

// ---- activations -------------------------------------------------------------
// An exponential is off by about 2^-23 for each unit of its argument (which carries 2^-24 itself), and so are the
// logistic function and what follows from it, far below 0: 2^-22 around 0, up to 2^-15 near -90.  Values in bf16
// do not notice; of a bias gradient's terms it is those of little weight.

__device__ __forceinline__ float mm_sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// tanh z = 2 sigmoid(2z) - 1, so that gelu_tanh is x sigmoid(2z).
__device__ __forceinline__ float mm_gelu_arg(float x) { return 1.5957691216057308f * x * (1.f + 0.044715f * x * x); }

// x sigmoid(z).  Below z = -87 the logistic function comes near the least normal number, where its reciprocal is cut to 0;
// it is exp(z) there, and its product with x, which stays normal down to -91, is exp(z + 32) times x exp(-32).
template <int ACT>
__device__ __forceinline__ bool mm_far1(float x) {
    return x < (ACT == WZ_ACT_SILU ? -87.f : -9.98f);   // z: x, or mm_gelu_arg(x)
}
template <int ACT>
__device__ __forceinline__ float mm_far_value(float x) {
    return x * 1.2664165549e-14f * __expf((ACT == WZ_ACT_SILU ? x : mm_gelu_arg(x)) + 32.f);
}

// The normal distribution's share below x, and exp(-x^2 / 2).  Below -|x| it is
// exp(-x^2 / 2) erfcx(|x| / sqrt 2) / 2, and the last factor t P(t) with t = 1 / (1 + 0.21 |x|):
// P was fitted for the least largest relative error over |x| <= 13 (2^-26; with fp32
// coefficients and steps 2^-21, beside the exponential's).  One reciprocal and one
// exponential, which the slope needs too: the slopes of 18,662 x 3584 products with
// erfcf and the exponential apart took 211 us.
__device__ __forceinline__ float mm_normal(float x, float &e) {
    const float t = __fdividef(1.f, fmaf(0.21f, fabsf(x), 1.f));
    float y = -7.219379397e-02f;
    y = fmaf(y, t, 2.862429807e-01f);
    y = fmaf(y, t, -3.358583682e-01f);
    y = fmaf(y, t, 3.560014568e-01f);
    y = fmaf(y, t, -9.866009608e-02f);
    y = fmaf(y, t, 1.269889168e-01f);
    y = fmaf(y, t, 6.861732179e-02f);
    y = fmaf(y, t, 8.515556234e-02f);
    y = fmaf(y, t, 8.370601885e-02f);
    e = __expf(-0.5f * x * x);
    y *= t * e;
    return x > 0.f ? 1.f - y : y;
}

template <int ACT>
__device__ __forceinline__ float mm_act1(float x) {
    float e;
    if constexpr (ACT == WZ_ACT_GELU) return x * mm_normal(x, e);
    if constexpr (ACT == WZ_ACT_GELU_TANH) return x * mm_sigmoid(mm_gelu_arg(x));
    if constexpr (ACT == WZ_ACT_SILU) return x * mm_sigmoid(x);
    return x;
}

// Whether some of x are far below 0, and then their activations (1 for the others); mm_put_far puts these, times a
// factor, where they belong.  Few products come near, so that a lane looks at the least of its numbers, and what is to
// be done about them stays out of the way, in local memory: asked for each number by itself, 5,103 x 1151 x 4607
// (M x K x N) with GELU took 58.5 us, so 55.8, as without; slopes of 741 x 1152 x 4616 formed again take 1.4 us
// longer for it (65.8 and 64.4 us with their products).
template <int ACT, int C>
__device__ __forceinline__ bool mm_far(const float (&x)[C], float (&there)[C]) {
    if constexpr (ACT == WZ_ACT_NONE || ACT == WZ_ACT_GELU) return false;
    float least = x[0];
#pragma unroll
    for (int j = 1; j < C; ++j) least = fminf(least, x[j]);
    const bool far = mm_far1<ACT>(least);
    if (far) {
#pragma unroll
        for (int j = 0; j < C; ++j) there[j] = x[j];
#pragma unroll 1
        for (int j = 0; j < C; ++j) there[j] = mm_far1<ACT>(there[j]) ? mm_far_value<ACT>(there[j]) : 1.f;
    }
    return far;
}

template <int C>
__device__ __forceinline__ void mm_far_times(bool far, float (&there)[C], const float (&factor)[C]) {
    if (far) {
#pragma unroll
        for (int j = 0; j < C; ++j) there[j] = there[j] <= 0.f ? there[j] * factor[j] : 0.f;
    }
}

template <bool TIMES, int C>
__device__ __forceinline__ void mm_put_far(bool far, const float (&there)[C], float (&y)[C]) {
    if (far) {
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (TIMES ? there[j] != 0.f : there[j] <= 0.f) y[j] = there[j];
    }
}

// Value and slope.  A factor that has become 0 wins over an x, or a power of it, that
// is infinite.
template <int ACT>
__device__ __forceinline__ void mm_slope1(float x, float &value, float &slope) {
    if constexpr (ACT == WZ_ACT_NONE) {
        value = x;
        slope = 1.f;
    } else if constexpr (ACT == WZ_ACT_GELU) {
        float e;
        const float phi = mm_normal(x, e);
        value = x * phi;
        slope = phi + (e > 0.f ? 0.3989422804014327f * x * e : 0.f);
    } else {
        const bool tanh_form = ACT == WZ_ACT_GELU_TANH;
        const float s = mm_sigmoid(tanh_form ? mm_gelu_arg(x) : x);
        const float t = s * (1.f - s);
        const float dz = tanh_form ? 1.5957691216057308f * (1.f + 0.134145f * x * x) : 1.f;
        value = x * s;
        slope = s + (t > 0.f ? x * t * dz : 0.f);
    }
}

// The same for two products at once, in packed fp32 instructions (the kernel of kept products is bound by the issue of
// instructions: 17 for a slope and its uses, 30 one by one).  GELU's slope is s below 0 and 1 - s above, s = the normal
// share below -|x| less |x| exp(-x^2 / 2) / sqrt(2 pi); |x| is cut at 1e10, where the exponential has become 0, so that
// infinities give 0 and 1.
__device__ __forceinline__ float mm_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float mm_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ f2_t both2(float x) { return pack2(x, x); }

constexpr float kFarW = 125.5f;   // of -z log2 e: 87 times it (mm_far1)

template <int ACT, bool VALUE>
__device__ __forceinline__ void mm_slope2(f2_t x, f2_t &value, f2_t &slope) {
    const float2 v = unpack2(x);
    if constexpr (ACT == WZ_ACT_NONE) {
        value = x;
        slope = both2(1.f);
    } else if constexpr (ACT == WZ_ACT_GELU) {
        const float a0 = fabsf(v.x), a1 = fabsf(v.y);
        const float2 u = unpack2(fma2(both2(0.21f), pack2(a0, a1), both2(1.f)));
        const f2_t t = pack2(mm_rcp(u.x), mm_rcp(u.y));
        f2_t y = both2(-7.219379397e-02f);
        y = fma2(y, t, both2(2.862429807e-01f));
        y = fma2(y, t, both2(-3.358583682e-01f));
        y = fma2(y, t, both2(3.560014568e-01f));
        y = fma2(y, t, both2(-9.866009608e-02f));
        y = fma2(y, t, both2(1.269889168e-01f));
        y = fma2(y, t, both2(6.861732179e-02f));
        y = fma2(y, t, both2(8.515556234e-02f));
        y = fma2(y, t, both2(8.370601885e-02f));
        const float2 w = unpack2(mul2(mul2(x, x), both2(-0.72134752044448f)));
        const f2_t e = pack2(mm_exp2(w.x), mm_exp2(w.y));
        y = mul2(y, mul2(t, e));
        const f2_t s = fma2(pack2(fminf(a0, 1e10f), fminf(a1, 1e10f)), mul2(e, both2(-0.3989422804014327f)), y);
        const float2 below = unpack2(s), above = unpack2(fma2(s, both2(-1.f), both2(1.f)));
        slope = pack2(v.x > 0.f ? above.x : below.x, v.y > 0.f ? above.y : below.y);
        if constexpr (VALUE) {
            const float2 n = unpack2(y), m = unpack2(fma2(y, both2(-1.f), both2(1.f)));
            value = mul2(x, pack2(v.x > 0.f ? m.x : n.x, v.y > 0.f ? m.y : n.y));
        }
    } else {
        constexpr bool kTanh = ACT == WZ_ACT_GELU_TANH;
        const f2_t square = mul2(x, x);
        // sigmoid(z) with z = x or the argument of mm_gelu_arg
        f2_t z = mul2(x, both2(kTanh ? -2.302208198f : -1.442695041f));   // - z log2 e
        if constexpr (kTanh) z = mul2(z, fma2(square, both2(0.044715f), both2(1.f)));
        const float2 w = unpack2(z);
        const float2 u = unpack2(add2(pack2(mm_exp2(w.x), mm_exp2(w.y)), both2(1.f)));
        const f2_t s = pack2(mm_rcp(u.x), mm_rcp(u.y));
        const f2_t t = mul2(s, fma2(s, both2(-1.f), both2(1.f)));
        f2_t xt = mul2(x, t);
        if constexpr (kTanh) xt = mul2(xt, fma2(square, both2(1.5957691216057308f * 0.134145f), both2(1.5957691216057308f)));
        const float2 a = unpack2(t), b = unpack2(xt);
        slope = add2(s, pack2(a.x > 0.f ? b.x : 0.f, a.y > 0.f ? b.y : 0.f));
        if constexpr (VALUE) {
            value = mul2(x, s);
            if (fmaxf(w.x, w.y) > kFarW) {   // (mm_far_value, in powers of two)
                const float2 n = unpack2(value);
                value = pack2(w.x > kFarW ? v.x * 0x1p-46f * mm_exp2(46.f - w.x) : n.x,
                              w.y > kFarW ? v.y * 0x1p-46f * mm_exp2(46.f - w.y) : n.y);
            }
        }
    }
}

// f(constant of type) for the call's activation.
template <typename F>
__device__ __forceinline__ void mm_with_act(int act, F f) {
    switch (act) {
        case WZ_ACT_GELU: f(std::integral_constant<int, WZ_ACT_GELU>()); break;
        case WZ_ACT_GELU_TANH: f(std::integral_constant<int, WZ_ACT_GELU_TANH>()); break;
        case WZ_ACT_SILU: f(std::integral_constant<int, WZ_ACT_SILU>()); break;
        default: f(std::integral_constant<int, WZ_ACT_NONE>()); break;
    }
}

// ---- rows of bf16 --------------------------------------------------------------

__device__ __forceinline__ uint32_t mm_pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// x[0 .. C) to p, of which the first n are inside the row; p is 16-byte aligned.
template <int C>
__device__ __forceinline__ void mm_store(__nv_bfloat16 *p, const float (&x)[C], int n) {
    if (n >= C) {
#pragma unroll
        for (int j = 0; j < C; j += 8)
            reinterpret_cast<uint4 *>(p)[j / 8] = make_uint4(mm_pack(x[j], x[j + 1]), mm_pack(x[j + 2], x[j + 3]),
                                                             mm_pack(x[j + 4], x[j + 5]), mm_pack(x[j + 6], x[j + 7]));
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (j < n) p[j] = __float2bfloat16_rn(x[j]);
    }
}

// C values from p, zeros from the n-th on.
template <int C>
__device__ __forceinline__ void mm_load(const __nv_bfloat16 *p, float (&x)[C], int n) {
    if (n >= C) {
        uint4 v[C / 8];
#pragma unroll
        for (int j = 0; j < C / 8; ++j) v[j] = reinterpret_cast<const uint4 *>(p)[j];
#pragma unroll
        for (int j = 0; j < C / 8; ++j) {
            float f[8];
            unpack(v[j], f, (__nv_bfloat16 *)nullptr);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[8 * j + i] = f[i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = j < n ? __bfloat162float(p[j]) : 0.f;
    }
}

// ---- finishing -------------------------------------------------------------------
// How mm_few.cu finishes sums: they go through shared memory, [row][output], and are finished row
// by row, four outputs to a lane: a warp reads and writes 256 (or 128) contiguous bytes.
// (mm_pair.cu finishes them where they are read.)

struct MmOutputs {
    int i, left;        // the lane's first output; how many there are from it on
    float b[2][4];      // biases
    float sum[2][4];    // of the slopes, over the rows that the lane has finished
};

template <bool BOTH>
__device__ __forceinline__ void mm_outputs(const MmArgs &p, const MmProblem &q, MmOutputs &o, int i) {
    o.i = i;
    o.left = q.N - i;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            o.b[w][j] = (w == 0 || BOTH) && p.bias[w] && j < o.left ? __ldg(p.bias[w] + i + j) : 0.f;
            o.sum[w][j] = 0.f;
        }
}

__device__ __forceinline__ void mm_load4(const __nv_bfloat16 *p, float (&x)[4], int left) {
    if (left >= 4) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = j < left ? __bfloat162float(p[j]) : 0.f;
    }
}

__device__ __forceinline__ void mm_store4(__nv_bfloat16 *p, const float (&x)[4], int left) {
    if (left >= 4) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(mm_pack(x[0], x[1]), mm_pack(x[2], x[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = __float2bfloat16_rn(x[j]);
    }
}

// Where the lane's outputs of a row are, in each array that the epilogue reads or writes.
template <int EPI>
struct MmAt {
    const __nv_bfloat16 *from;   // the residual, or dy; null: none
    __nv_bfloat16 *out, *out2, *pre0, *pre1;
    int64_t s_from, s_out, s_out2, s_pre0, s_pre1;
    __device__ __forceinline__ MmAt(const MmArgs &p, const MmProblem &q, int64_t row, int i) {
        const __nv_bfloat16 *base = EPI == kMmStore ? p.residual : EPI == kMmGated ? nullptr : p.dy;
        s_from = EPI == kMmStore ? p.residual_stride : p.dy_stride;
        from = base ? base + row * s_from + i : nullptr;
        s_out = q.out_stride, out = q.out + row * s_out + i;
        s_out2 = p.out2_stride, out2 = p.out2 + row * s_out2 + i;
        s_pre0 = p.pre_stride[0], pre0 = p.pre[0] ? p.pre[0] + row * s_pre0 + i : nullptr;
        s_pre1 = p.pre_stride[1], pre1 = p.pre[1] + row * s_pre1 + i;
    }
    __device__ __forceinline__ void advance(int rows) {
        if (from) from += rows * s_from;
        if (pre0) pre0 += rows * s_pre0;
        out += rows * s_out, out2 += rows * s_out2, pre1 += rows * s_pre1;
    }
};

// The residual, or dy, of U rows `step` apart, of which the first `count` (in steps) are there.
template <int EPI, int U>
__device__ __forceinline__ void mm_fetch(const MmAt<EPI> &at, int left, float (&other)[U][4], int step, int count) {
    if (EPI == kMmGated || !at.from) return;
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (k < count) mm_load4(at.from + k * step * at.s_from, other[k], left);
}

// Finishes and stores them: v holds the sums (g in a gated product, u its other ones).
template <int EPI, int ACT, int U>
__device__ __forceinline__ void mm_finish(const MmAt<EPI> &at, MmOutputs &o, float (&v)[U][4], float (&u)[U][4],
                                          const float (&other)[U][4], int step, int count) {
    const int left = o.left;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        if (k >= count) break;
        float y[4], z[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[k][j] += o.b[0][j];
            if constexpr (mm_both(EPI)) u[k][j] += o.b[1][j];
        }
        float there[4];
        if constexpr (EPI == kMmStore) {
            const bool far = mm_far<ACT>(v[k], there);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = mm_act1<ACT>(v[k][j]);
            mm_put_far<false>(far, there, y);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at.from) y[j] += other[k][j];
        } else if constexpr (EPI == kMmGated) {
            const bool far = mm_far<ACT>(v[k], there);
            mm_far_times(far, there, u[k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = mm_act1<ACT>(v[k][j]) * u[k][j];
            mm_put_far<true>(far, there, y);
        } else {
            const bool far = EPI == kMmGatedSlope && mm_far<ACT>(v[k], there);
            mm_far_times(far, there, other[k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float value, slope;
                mm_slope1<ACT>(v[k][j], value, slope);
                y[j] = (EPI == kMmSlope ? other[k][j] : other[k][j] * u[k][j]) * slope;
                z[j] = other[k][j] * value;
                o.sum[0][j] += y[j];
            }
            if constexpr (EPI == kMmGatedSlope) {
                mm_put_far<true>(far, there, z);
#pragma unroll
                for (int j = 0; j < 4; ++j) o.sum[1][j] += z[j];
            }
        }
        if constexpr (EPI == kMmStore || EPI == kMmGated)
            if (at.pre0) mm_store4(at.pre0 + k * step * at.s_pre0, v[k], left);
        if constexpr (EPI == kMmGated)
            if (at.pre0) mm_store4(at.pre1 + k * step * at.s_pre1, u[k], left);
        mm_store4(at.out + k * step * at.s_out, y, left);
        if constexpr (EPI == kMmGatedSlope) mm_store4(at.out2 + k * step * at.s_out2, z, left);
    }
}

// 32 columns of a bias gradient, by 16 warps: a lane has a column, a warp every 16th row, 16 of them
// on their way at a time; then the warps' sums in order.  barrier(): of the 16 warps.
constexpr int kSumRows = 16;

template <typename F>
__device__ __forceinline__ void mm_column_sums(const MmSums &p, int block, int thread, float (*sums)[33], F barrier) {
    const int columns = (p.N + 31) / 32, which = p.db[0] && block < columns ? 0 : 1;
    const float *part = p.part[which];
    const int c = thread & 31, r0 = thread >> 5;
    const int n = (which && p.db[0] ? block - columns : block) * 32 + c;
    float s = 0.f;
    if (n < p.N) {
        const auto add = [&](int64_t rows, auto value) {
            for (int64_t r = r0; r < rows; r += 16 * kSumRows) {
                float x[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = r + k * kSumRows < rows ? value(r + k * kSumRows) : 0.f;
#pragma unroll
                for (int d = 1; d < 16; d *= 2)
#pragma unroll
                    for (int k = 0; k < 16; k += 2 * d) x[k] += x[k + d];
                s += x[0];
            }
        };
        add(p.part_rows, [&](int64_t r) { return part[r * p.N + n]; });
        add(p.dy_rows, [&](int64_t r) { return __bfloat162float(p.dy[r * p.dy_stride + n]); });
    }
    sums[r0][c] = s;
    barrier();
    if (r0 == 0 && n < p.N) {
#pragma unroll
        for (int i = 1; i < kSumRows; ++i) s += sums[i][c];
        p.db[which][n] = s;
    }
}

// 16 columns of tensor memory (of the warp's 32 lanes).
__device__ __forceinline__ void mm_read16(uint32_t tcol, float (&x)[16]) {
    uint32_t v[16];
    ptx::tmem_ld_32x32b_x16(tcol, v);
    ptx::tmem_ld_wait();
    ptx::reg_fence16(v);
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(v[j]);
}

// ---- launches (arguments checked) ------------------------------------------------
// All with programmatic stream serialization, the first of a call too: each kernel waits for
// the grid before it, whoever's it is, before it touches memory, so that only its start
// overlaps that grid's end.

// The most rows of sums over rows that a launch writes for M rows: mm_pair.cu's up to eight for each of at most
// M / 128 + 3 row tiles.
__host__ __device__ inline int64_t mm_part_rows(int64_t M) { return (M + 15) / 16 + 32; }

// Tiles of 256 outputs x up to 256 rows on pairs of SMs (mm_pair.cu).  part_rows (nullable), here and
// below: the rows of sums that the launch writes.
int mm_pair_tile(int64_t M, int64_t output_tiles);   // their rows
cudaError_t launch_mm_pair(MmEpilogue epi, MmArgs &p, int sms, cudaStream_t s, int64_t *part_rows);

// One product in tiles of 16 to 256 rows on one SM or a pair, K shared by a cluster (mm_few.cu).
// False: it does not suit it.
struct MmFewPlan {
    bool pair;
    int split, tile_m;   // shares of K, rows of a tile
};
bool plan_mm_few(MmEpilogue epi, const MmArgs &p, int sms, MmFewPlan *plan);
cudaError_t launch_mm_few(MmEpilogue epi, MmArgs &p, const MmFewPlan &plan, cudaStream_t s,
                          int64_t *part_rows);

uint64_t mm_wait_ns();   // the limit of the products' waits

// A launch's tensor maps.
struct MmMapList {
    MmMaps maps;
    int count = 0;
    bool ok = true;
    MmMapList();
    int add(const MmOperand &o, int box_rows);
};

}  // namespace wz
