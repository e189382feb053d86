// A layer's matrix products and their gradients (wz_linear, wz_gated and their
// backward passes): the launches of a call, and the kernels beside the products.
//
//   mm_delta_kernel   d = dy act'(p), or dg = dout u act'(g) and du = dout act(g), from
//                     kept products, with column sums over 64 rows; or the sums alone
//   mm_join_kernel    products whose K was shared, and bias gradients where the products'
//                     kernel does not add them up (mm_column_sums)
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "wz_mm.cuh"

namespace wz {

namespace {

size_t pad256(size_t x) { return (x + 255) / 256 * 256; }

constexpr int kDeltaRows = 64, kDeltaCols = 256, kDeltaWarps = 8;

enum DeltaMode : int { kDeltaSums = 0, kDeltaSlope = 1, kDeltaGated = 2 };

struct DeltaArgs {
    const __nv_bfloat16 *dy, *pre[2];   // kDeltaSlope: p; kDeltaGated: g and u
    __nv_bfloat16 *d[2];
    float *part[2];                     // [ceil(M / 64)][N]; null: not wanted
    int64_t dy_stride, pre_stride[2], d_stride;
    int64_t M, room_rows, room_part;    // rows at d, floats at each part: see MmProblem
    int N, act;
    int *status;
};

}  // namespace

// A block takes 64 rows of 256 columns, a warp every eighth row, a lane eight columns: 16-byte
// loads and stores, the column sums in registers and then over the warps in a fixed order.
// GELU slopes and sums of 18,662 x 3584: 88 us (4.5 TB/s; HBM's floor is 59), bound by the issue of
// the slopes' instructions; one product at a time 117, with erfcf 211.  SiLU 78.
template <int MODE>
__global__ void __launch_bounds__(32 * kDeltaWarps) mm_delta_kernel(const __grid_constant__ DeltaArgs p) {
    __shared__ float sums[kDeltaWarps][kDeltaCols];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = (int)blockIdx.y * kDeltaCols + 8 * lane, left = p.N - n;
    const int64_t m0 = (int64_t)blockIdx.x * kDeltaRows;
    f2_t a0[4] = {}, a1[4] = {};   // (zero bits are zeros)
    if (left > 0) {
        mm_with_act(p.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            // (a batch of rows is on its way before the first of them is stored: the compiler keeps
            // loads behind stores that might be to the same place)
            constexpr int kBatch = 4, kArrays = MODE == kDeltaSums ? 1 : MODE == kDeltaSlope ? 2 : 3;
            const __nv_bfloat16 *from[3] = {p.dy + n, p.pre[0] + n, p.pre[1] + n};
            const int64_t strides[3] = {p.dy_stride, p.pre_stride[0], p.pre_stride[1]};
#pragma unroll
            for (int r0 = warp; r0 < kDeltaRows; r0 += kBatch * kDeltaWarps) {
                uint4 raw[kArrays][kBatch];
                const bool wide = left >= 8 && m0 + r0 + (kBatch - 1) * kDeltaWarps < p.M;
                if (wide) {
#pragma unroll
                    for (int k = 0; k < kBatch; ++k)
#pragma unroll
                        for (int a = 0; a < kArrays; ++a)
                            raw[a][k] = *reinterpret_cast<const uint4 *>(from[a] + (m0 + r0 + k * kDeltaWarps) * strides[a]);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int64_t m = m0 + r0 + k * kDeltaWarps;
                    if ((!wide && m >= p.M) || !wz_in_range(p.status, m < p.room_rows)) break;
                    f2_t dy[4], g[4], u[4];
                    const auto take = [&](int a, f2_t (&x)[4]) {
                        if (wide) {
                            unpack_pairs(raw[a < kArrays ? a : 0][k], x, (__nv_bfloat16 *)nullptr);
                        } else {
                            float y[8];
                            mm_load(from[a] + m * strides[a], y, left);
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[j] = pack2(y[2 * j], y[2 * j + 1]);
                        }
                    };
                    const auto put = [&](__nv_bfloat16 *to, const f2_t (&x)[4]) {
                        float y[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 v = unpack2(x[j]);
                            y[2 * j] = v.x;
                            y[2 * j + 1] = v.y;
                        }
                        mm_store(to, y, wide ? 8 : left);
                    };
                    take(0, dy);
                    if constexpr (MODE == kDeltaSums) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) a0[j] = add2(a0[j], dy[j]);
                    } else {
                        take(1, g);
                        if constexpr (MODE == kDeltaGated) take(2, u);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            f2_t value, slope;
                            mm_slope2<ACT, MODE == kDeltaGated>(g[j], value, slope);
                            if constexpr (MODE == kDeltaGated) {
                                g[j] = mul2(mul2(dy[j], u[j]), slope);
                                u[j] = mul2(dy[j], value);
                                a1[j] = add2(a1[j], u[j]);
                            } else {
                                g[j] = mul2(dy[j], slope);
                            }
                            a0[j] = add2(a0[j], g[j]);
                        }
                        put(p.d[0] + m * p.d_stride + n, g);
                        if constexpr (MODE == kDeltaGated) put(p.d[1] + m * p.d_stride + n, u);
                    }
                }
            }
        });
    }
#pragma unroll
    for (int i = 0; i < (MODE == kDeltaGated ? 2 : 1); ++i) {
        if (!p.part[i]) continue;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 v = unpack2(i ? a1[j] : a0[j]);
            sums[warp][8 * lane + 2 * j] = v.x;
            sums[warp][8 * lane + 2 * j + 1] = v.y;
        }
        __syncthreads();
        const int c = (int)blockIdx.y * kDeltaCols + (int)threadIdx.x;
        if (c < p.N) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kDeltaWarps; ++w) s += sums[w][threadIdx.x];
            const size_t at = (size_t)blockIdx.x * p.N + c;
            if (wz_in_range(p.status, at < (size_t)p.room_part)) p.part[i][at] = s;
        }
    }
}

namespace {

constexpr int kSumThreads = 32 * kSumRows;
constexpr int kJoinRows = 4;   // rows that a thread of a join takes
// Up to so many rows of dy are added up as they are, if need be by the last kernel, which is a kernel less before the
// products.
constexpr int64_t kFewSumRows = 1024;
// A CTA of the products adds up to so many blocks of 32 columns of them, or of sums over some rows, before its first
// tile; more are left to the last kernel (577 x 1152 x 3584 (M x K x N) 19.5 us with it, 15.8 without).
constexpr int kSumBlocksEach = 4;
// And of more rows where the first tile's products take longer: 13 / 2 cycles a row of a block.  4,096 rows of
// 3584 x 14336 (K x N) 434 us, with a kernel for sums over 64 rows before 460; 18,662 of 3584 x 3584 500 and 523;
// but 4,096 of 256 x 4608, whose tiles are short, 68 and 34.
constexpr int64_t kSumRowCycles2 = 13;

// What is left to add up when the products are done.
struct JoinArgs {
    MmSums sums;
    // products whose K was shared: out = the sum of sums[split][M][cols]
    struct {
        const float *sums;
        __nv_bfloat16 *out;
        int64_t out_stride, M, room_rows;
        int cols, split;
        unsigned first;        // its first block
    } join[kMmProblems];
    int joins;
    int *status;
};

}  // namespace

// The first blocks take 32 columns of a bias gradient each; the others 512 outputs of 16 rows of a
// shared product, a thread four outputs of four of them, in the shares' order.  (Four rows' loads are on
// their way at a time; the sums are mostly in L2.)
__global__ void __launch_bounds__(kSumThreads) mm_join_kernel(const __grid_constant__ JoinArgs p) {
    __shared__ float sums[kSumRows][33];
    pdl_wait();
    pdl_trigger();
    unsigned block = blockIdx.x;
    if ((int)block < p.sums.blocks) {
        mm_column_sums(p.sums, (int)block, (int)threadIdx.x, sums, [] { __syncthreads(); });
        return;
    }
    int i = 0;
    while (i + 1 < p.joins && block >= p.join[i + 1].first) ++i;
    const auto &j = p.join[i];
    const unsigned across = (unsigned)(j.cols + 511) / 512;
    block -= j.first;
    const int n = (int)(block % across) * 512 + 4 * (int)(threadIdx.x & 127), left = j.cols - n;
    const int64_t m0 = (int64_t)(block / across) * (4 * kJoinRows) + (int)(threadIdx.x >> 7);
    if (left <= 0) return;
    const int64_t plane = j.M * j.cols;
    if (!wz_in_range(p.status, m0 < j.room_rows)) return;
    const bool wide = left >= 4 && j.cols % 4 == 0;
    if (wide && m0 + 4 * (kJoinRows - 1) < j.M && wz_in_range(p.status, m0 + 4 * (kJoinRows - 1) < j.room_rows)) {
        float x[kJoinRows][4] = {};
        const float *from = j.sums + m0 * j.cols + n;
#pragma unroll 2
        for (int k = 0; k < j.split; ++k, from += plane) {
            float4 v[kJoinRows];
#pragma unroll
            for (int r = 0; r < kJoinRows; ++r) v[r] = __ldcs(reinterpret_cast<const float4 *>(from + 4 * r * (int64_t)j.cols));
#pragma unroll
            for (int r = 0; r < kJoinRows; ++r) x[r][0] += v[r].x, x[r][1] += v[r].y, x[r][2] += v[r].z, x[r][3] += v[r].w;
        }
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r) mm_store4(j.out + (m0 + 4 * r) * j.out_stride + n, x[r], 4);
        return;
    }
    for (int r = 0; r < kJoinRows; ++r) {
        const int64_t m = m0 + 4 * r;
        if (m >= j.M || !wz_in_range(p.status, m < j.room_rows)) break;
        const float *from = j.sums + m * j.cols + n;
        float x[4] = {};
        for (int k = 0; k < j.split; ++k, from += plane)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) x[e] += from[e];
        mm_store4(j.out + m * j.out_stride + n, x, left);
    }
}

namespace {

cudaError_t launch_delta(DeltaMode mode, DeltaArgs &p, cudaStream_t s) {
    const dim3 grid((unsigned)((p.M + kDeltaRows - 1) / kDeltaRows), (unsigned)((p.N + kDeltaCols - 1) / kDeltaCols));
    const void *fn = mode == kDeltaSums    ? (const void *)mm_delta_kernel<kDeltaSums>
                     : mode == kDeltaSlope ? (const void *)mm_delta_kernel<kDeltaSlope>
                                           : (const void *)mm_delta_kernel<kDeltaGated>;
    void *args[] = {&p};
    return launch_kernel(fn, grid, dim3(32 * kDeltaWarps), 0, s, args, true);
}

// Launches p's sums and joins, if there are any.
cudaError_t launch_join(JoinArgs &p, cudaStream_t s) {
    int64_t blocks = p.sums.blocks;
    for (int i = 0; i < p.joins; ++i) {
        p.join[i].first = (unsigned)blocks;
        blocks += (p.join[i].M + 4 * kJoinRows - 1) / (4 * kJoinRows) * ((p.join[i].cols + 511) / 512);
    }
    if (!blocks) return cudaSuccess;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    void *args[] = {&p};
    return launch_kernel((const void *)mm_join_kernel, dim3((unsigned)blocks), dim3(kSumThreads), 0, s, args, true);
}

__nv_bfloat16 *half(void *p) { return static_cast<__nv_bfloat16 *>(p); }
const __nv_bfloat16 *half(const void *p) { return static_cast<const __nv_bfloat16 *>(p); }

MmArgs mm_args(int act, int *status) {
    MmArgs p;
    memset(&p, 0, sizeof(p));
    p.problems = 1;
    p.act = act;
    p.status = status;
    p.wait_ns = mm_wait_ns();
    return p;
}

int64_t steps_of(int64_t k) { return (k + 63) / 64; }

// What there is room for, as the checked build's kernels are told (its test takes some away).
#ifdef WZ_CHECKED
int check_room = 0;   // bits: 1 the last row of outputs, 2 sums over rows but for the first, 4 shares' sums but for the first
int64_t room_rows(int64_t rows) { return rows - (check_room & 1); }
int64_t room_part(size_t bytes, int N) { return check_room & 2 ? N : (int64_t)(bytes / 4); }
int64_t room_sums(size_t bytes, int64_t plane) { return check_room & 4 ? plane : (int64_t)(bytes / 4); }
#else
int64_t room_rows(int64_t rows) { return rows; }
int64_t room_part(size_t bytes, int) { return (int64_t)(bytes / 4); }
int64_t room_sums(size_t bytes, int64_t) { return (int64_t)(bytes / 4); }
#endif

JoinArgs join_args(const float *part0, const float *part1, float *db0, float *db1, int64_t rows, int N, int *status) {
    JoinArgs j;
    memset(&j, 0, sizeof(j));
    j.status = status;
    MmSums &p = j.sums;
    p.part[0] = part0, p.part[1] = part1, p.db[0] = db0, p.db[1] = db1;
    p.part_rows = rows, p.N = N;
    p.blocks = ((db0 ? 1 : 0) + (db1 ? 1 : 0)) * ((N + 31) / 32);
    return j;
}

// One layer's gradients from d: dx = d W (+ d2 W2) and dW = d^T x (dW2 = d2^T x).
struct Gradients {
    int both;                       // 1 or 2 products
    const void *d[2], *w[2], *x;
    void *dx, *dw[2];
    int64_t d_stride, w_stride[2], x_stride, dx_stride, dw_stride[2];
    int64_t M;
    int N, K;
};

// How the gradients' products are cut: row tiles, and shares of K where tiles are too few or too long to come out even
// on the pairs of SMs.
struct GradientSplit {
    int dx, dw;              // shares
    int tile_x, tile_w;      // rows of a tile
};

// Units of one gradient's products: tiles times shares, and the cycles of one.
struct Units {
    int64_t n, cycles;
};

Units units(int64_t rows, int64_t outs, int64_t products, int64_t steps, int tile, int shares) {
    return Units{products * ((rows + tile - 1) / tile) * ((outs + 255) / 256) * shares,
                 std::max<int64_t>((steps + shares - 1) / shares * std::max(2 * tile, 256 + tile), 5000)};
}

// Cycles of a launch of both: the longest unit's, or all of them evenly.
int64_t launch_cycles(const Units &x, const Units &w) {
    const auto rounds = [](const Units &u) { return (u.n + kPlanPairs - 1) / kPlanPairs * u.cycles; };
    if (!x.n || !w.n) return rounds(x) + rounds(w);
    const Units &longer = x.cycles > w.cycles ? x : w;
    return std::max(rounds(longer), (x.n * x.cycles + w.n * w.cycles) / kPlanPairs + std::min(x.cycles, w.cycles) / 2);
}

// The rows dealt evenly to k tiles of at most 256, in thirty-twos; 0: they do not fit.
int tile_of(int64_t rows, int64_t k) {
    const int64_t tile = (rows + k * 32 - 1) / (k * 32) * 32;
    return tile <= 256 ? (int)tile : 0;
}

// Bytes of the shares' sums.
size_t shares_bytes(int64_t M, int N, int K, int both, int dx, int dw) {
    return (dx > 1 ? pad256((size_t)dx * (size_t)M * (size_t)K * 4) : 0) +
           (dw > 1 ? both * pad256((size_t)dw * (size_t)N * (size_t)K * 4) : 0);
}
constexpr size_t kMostSharesBytes = 48u << 20;

// A weight gradient's terms are the rows, of which there may be any number, and a sum on the tensor cores comes out too
// small by a part that grows with its terms (see kLongSteps): 3,000,000 rows of one sign, in eight shares, lost
// 3.1e-3, about a bf16 rounding (now 2e-4 to 4e-4).  So one sum takes 65,536 rows at most, as many as a forward product
// has terms, and loses about 4e-4 of terms of one sign; the shares' sums are added in fp32.
constexpr int64_t kMostSumSteps = 1024;
int least_shares(int64_t M) { return (int)std::max<int64_t>(1, (steps_of(M) + kMostSumSteps - 1) / kMostSumSteps); }

GradientSplit split_gradients(int64_t M, int N, int K, int both, bool dx, bool dw) {
    const int64_t sx = both * steps_of(N), sw = steps_of(M);
    const int64_t kx = (M + 255) / 256, kw = ((int64_t)N + 255) / 256;
    const int least_dw = dw ? least_shares(M) : 1;
    const size_t most = std::max(kMostSharesBytes, shares_bytes(M, N, K, both, 1, least_dw));
    GradientSplit best{1, least_dw, tile_of(M, kx), tile_of(N, kw)};
    int64_t least = INT64_MAX;
    const auto consider = [&](int tx, int tw, int a, int b) {
        if (!tx || !tw) return;
        const Units none{0, 0};
        int64_t t = launch_cycles(dx ? units(M, K, 1, sx, tx, a) : none, dw ? units(N, K, both, sw, tw, b) : none);
        // shares are written, read again and joined by a kernel (4,000 cycles and 2,600 bytes a cycle), and
        // something has to come of it: the model is not exact
        if (a > 1 || b > 1)
            t = (t + 4000 + ((a > 1 ? a * M : 0) + (b > 1 ? b * (int64_t)both * N : 0)) * K * 8 / 2600) * 17 / 16;
        if (t < least) {
            least = t;
            best = GradientSplit{a, b, tx, tw};
        }
    };
    // as few row tiles as hold the rows, or one or two more
    for (int64_t i = kx; i <= kx + (dx && kx <= 8 ? 2 : 0); ++i)
        for (int64_t j = kw; j <= kw + (dw && kw <= 8 ? 2 : 0); ++j) consider(tile_of(M, i), tile_of(N, j), 1, least_dw);
    // and more shares, unless the pairs have no less to do on the whole
    const Units x = dx ? units(M, K, 1, sx, best.tile_x, 1) : Units{0, 0},
                w = dw ? units(N, K, both, sw, best.tile_w, least_dw) : Units{0, 0};
    if (least <= (x.n * x.cycles + w.n * w.cycles) / kPlanPairs * 9 / 8) return best;
    const int tiles[2][2] = {{best.tile_x, best.tile_w}, {tile_of(M, kx), tile_of(N, kw)}};
    constexpr int kShares[] = {1, 2, 3, 4, 6, 8};
    for (const auto &t : tiles)
        for (int a : kShares)
            for (int more : kShares) {
                const int b = std::max(more, least_dw);
                if ((a > 1 && (!dx || sx < 2 * a)) || (b > 1 && (!dw || sw < 2 * b)) || (a == 1 && b == 1)) continue;
                if (shares_bytes(M, N, K, both, a, b) <= most) consider(t[0], t[1], a, b);
            }
    return best;
}

// The products of both gradients in one launch, with the bias gradients of `join` where they are few enough; what
// they leave to be joined goes into `join`.
// (shares_end: where the workspace ends)
cudaError_t launch_gradients(const Gradients &g, const GradientSplit &split, bool beside, char *shares,
                             const char *shares_end, JoinArgs &join, int *status, int sms, cudaStream_t s) {
    MmArgs p = mm_args(WZ_ACT_NONE, status);
    MmProblem in, weight[2];
    memset(&in, 0, sizeof(in));
    memset(weight, 0, sizeof(weight));
    in.M = (int)g.M, in.N = g.K, in.segments = g.both, in.steps = (int)steps_of(g.N);
    in.b_mn = 1;
    in.out = half(g.dx), in.out_stride = g.dx_stride, in.room_rows = room_rows(g.M);
    for (int i = 0; i < g.both; ++i) {
        const MmOperand d{g.d[i], g.M, g.N, g.d_stride};
        in.from_a[i] = d;
        in.from_b[i] = MmOperand{g.w[i], g.N, g.K, g.w_stride[i]};
        MmProblem &q = weight[i];
        q.M = g.N, q.N = g.K, q.segments = 1, q.steps = (int)steps_of(g.M);
        q.a_mn = q.b_mn = 1;
        q.out = half(g.dw[i]), q.out_stride = g.dw_stride[i], q.room_rows = room_rows(g.N);
        q.from_a[0] = d;
        q.from_b[0] = MmOperand{g.x, g.M, g.K, g.x_stride};
    }
    // (dx alone may suit the kernel for few tiles, which joins shares of K by itself)
    if (g.dx && !g.dw[0]) {
        MmFewPlan plan;
        p.prob[0] = in;
        if (plan_mm_few(kMmStore, p, sms, &plan)) return launch_mm_few(kMmStore, p, plan, s, nullptr);
    }
    in.tile_m = split.tile_x;
    weight[0].tile_m = weight[1].tile_m = split.tile_w;
    bool none_left = false;
    const auto add = [&](MmProblem &q, int shared) {
        q.split = shared;
        if (shared > 1) {
            q.sums = reinterpret_cast<float *>(shares);
            q.room_sums = room_sums((size_t)(shares_end - shares), (int64_t)q.M * q.N);
            shares += pad256((size_t)shared * (size_t)q.M * (size_t)q.N * 4);
            none_left = none_left || shares > shares_end;
            auto &j = join.join[join.joins++];
            j.sums = q.sums, j.out = q.out, j.out_stride = q.out_stride, j.M = q.M, j.cols = q.N, j.split = shared;
            j.room_rows = q.room_rows;
        }
        p.prob[p.problems++] = q;
    };
    // the longer tiles first, so that the shorter ones even out the ends
    const bool weights_first = g.dw[0] && (!g.dx || weight[0].steps / split.dw > in.steps * in.segments / split.dx);
    p.problems = 0;
    if (g.dx && !weights_first) add(in, split.dx);
    if (g.dw[0])
        for (int i = 0; i < g.both; ++i) add(weight[i], split.dw);
    if (g.dx && weights_first) add(in, split.dx);
    if (!p.problems) return cudaSuccess;
    if (none_left) return cudaErrorInvalidValue;
    if (beside || join.sums.blocks <= kSumBlocksEach * sms) {
        p.sums = join.sums;
        join.sums.blocks = 0;
    }
    return launch_mm_pair(kMmStore, p, sms, s, nullptr);
}

cudaError_t zero_rows(void *p, int64_t stride, int rows, int cols, cudaStream_t s) {
    return p ? cudaMemset2DAsync(p, (size_t)stride * 2, 0, (size_t)cols * 2, (size_t)rows, s) : cudaSuccess;
}

// Rows of d begin on 128 bytes: what does not comes into an SM as two lines for each box row.
int64_t delta_stride(int N) { return ((int64_t)N + 63) / 64 * 64; }

size_t delta_bytes(int64_t M, int N) { return pad256((size_t)M * (size_t)delta_stride(N) * 2); }

size_t part_bytes(int64_t M, int N) { return pad256((size_t)mm_part_rows(M) * (size_t)N * 4); }

// The forward products of a layer: x [M][K] with one or two weights [N][K].
void forward_product(MmArgs &p, int64_t M, int N, int K, const void *x, int64_t x_stride, const void *w0,
                     int64_t stride0, const void *w1, int64_t stride1) {
    MmProblem &q = p.prob[0];
    q.M = (int)M, q.N = N, q.segments = 1, q.steps = (int)steps_of(K);
    q.room_rows = room_rows(M);
    q.from_a[0] = MmOperand{x, M, K, x_stride};
    q.from_b[0] = MmOperand{w0, N, K, stride0};
    q.from_b[1] = MmOperand{w1, N, K, stride1};
}

// The products of a forward call, or of the slopes, with the kernel that suits their sizes.
cudaError_t launch_mm(MmEpilogue epi, MmArgs &p, int sms, cudaStream_t s, int64_t *part_rows) {
    MmFewPlan plan;
    if (plan_mm_few(epi, p, sms, &plan)) return launch_mm_few(epi, p, plan, s, part_rows);
    return launch_mm_pair(epi, p, sms, s, part_rows);
}

#ifdef WZ_CHECKED
uint64_t check_mm_wait_ns = kMmTimeoutNs;
#endif

}  // namespace

uint64_t mm_wait_ns() {
#ifdef WZ_CHECKED
    return check_mm_wait_ns;
#else
    return kMmTimeoutNs;
#endif
}

cudaError_t launch_linear(const wz_linear_args &a, cudaStream_t s) {
    const int sms = sm_count();
    if (sms < 2) return cudaErrorInvalidDevice;
    MmArgs p = mm_args(a.act, a.device_status);
    forward_product(p, a.M, a.N, a.K, a.x, a.x_stride, a.w, a.w_stride, nullptr, 0);
    p.prob[0].out = half(a.out), p.prob[0].out_stride = a.out_stride;
    p.bias[0] = a.bias;
    p.residual = half(a.residual), p.residual_stride = a.residual_stride;
    p.pre[0] = half(a.pre), p.pre_stride[0] = a.pre_stride;
    return launch_mm(kMmStore, p, sms, s, nullptr);
}

cudaError_t launch_gated(const wz_gated_args &a, cudaStream_t s) {
    const int sms = sm_count();
    if (sms < 2) return cudaErrorInvalidDevice;
    MmArgs p = mm_args(a.act, a.device_status);
    forward_product(p, a.M, a.N, a.K, a.x, a.x_stride, a.w_gate, a.w_gate_stride, a.w_up, a.w_up_stride);
    p.prob[0].out = half(a.out), p.prob[0].out_stride = a.out_stride;
    p.bias[0] = a.b_gate, p.bias[1] = a.b_up;
    p.pre[0] = half(a.gate), p.pre_stride[0] = a.gate_stride;
    p.pre[1] = half(a.up), p.pre_stride[1] = a.up_stride;
    return launch_mm(kMmGated, p, sms, s, nullptr);
}

namespace {

// Whether dy's sums are ready before the products of the first tiles.
bool sums_beside(int64_t M, int N, int K, const GradientSplit &split, bool dx, bool dw) {
    const Units none{0, 0}, x = dx ? units(M, K, 1, steps_of(N), split.tile_x, split.dx) : none,
                            w = dw ? units(N, K, 1, steps_of(M), split.tile_w, split.dw) : none;
    const int64_t ctas = 2 * std::min<int64_t>(kPlanPairs, x.n + w.n);
    return dw && M * (((N + 31) / 32 + ctas - 1) / ctas) * kSumRowCycles2 <= 2 * std::max(x.cycles, w.cycles);
}

// How a backward call is cut, and where its parts are in its workspace: d, sums over rows, shares' sums, as
// many as it needs.
struct BackwardLayout {
    GradientSplit split;
    bool beside = false, of_dy = false;   // dy is added up beside the products; without sums over some rows before
    size_t d[2], part[2] = {}, shares, total = 0;
    BackwardLayout(int64_t M, int N, int K, int both, bool dx, bool dw) : split(split_gradients(M, N, K, both, dx, dw)) {}
    size_t take(size_t bytes) {
        const size_t at = total;
        total += bytes;
        return at;
    }
    void place(int64_t M, int N, int K, int both, bool with_d, bool part0, bool part1) {
        for (int i = 0; i < 2; ++i) d[i] = take(with_d && i < both ? delta_bytes(M, N) : 0);
        part[0] = take(part0 ? part_bytes(M, N) : 0);
        part[1] = take(part1 ? part_bytes(M, N) : 0);
        shares = take(shares_bytes(M, N, K, both, split.dx, split.dw));
    }
};

BackwardLayout layout_of(const wz_linear_backward_args &a) {
    BackwardLayout at(a.M, a.N, a.K, 1, a.dx, a.dw);
    at.beside = a.act == WZ_ACT_NONE && sums_beside(a.M, a.N, a.K, at.split, a.dx, a.dw);
    at.of_dy = at.beside || (a.act == WZ_ACT_NONE && a.M <= kFewSumRows);
    at.place(a.M, a.N, a.K, 1, a.act != WZ_ACT_NONE, a.db && !at.of_dy, false);
    return at;
}

BackwardLayout layout_of(const wz_gated_backward_args &a) {
    BackwardLayout at(a.M, a.N, a.K, 2, a.dx, a.dw_gate);
    at.place(a.M, a.N, a.K, 2, true, a.db_gate, a.db_up);
    return at;
}

// The most that a call of these sizes needs, whichever gradients it asks for.
size_t most_bytes(int64_t M, int N, int K, int both) {
    const int least = least_shares(M);
    return both * (delta_bytes(M, N) + part_bytes(M, N)) +
           std::max(std::min(kMostSharesBytes, shares_bytes(M, N, K, both, 8, std::max(8, least))),
                    shares_bytes(M, N, K, both, 1, least));
}

}  // namespace

size_t linear_backward_bytes(int64_t M, int N, int K) { return most_bytes(M, N, K, 1); }
size_t gated_backward_bytes(int64_t M, int N, int K) { return most_bytes(M, N, K, 2); }
size_t linear_backward_need(const wz_linear_backward_args &a) { return a.M > 0 ? layout_of(a).total : 0; }
size_t gated_backward_need(const wz_gated_backward_args &a) { return a.M > 0 ? layout_of(a).total : 0; }

#define MM_TRY(call)                              \
    do {                                          \
        const cudaError_t mm_e = (call);          \
        if (mm_e != cudaSuccess) return mm_e;     \
    } while (0)

cudaError_t launch_linear_backward(const wz_linear_backward_args &a, char *ws, cudaStream_t s) {
    if (a.M == 0) {
        MM_TRY(zero_rows(a.dw, a.dw_stride, a.N, a.K, s));
        JoinArgs join = join_args(nullptr, nullptr, a.db, nullptr, 0, a.N, a.device_status);
        return launch_join(join, s);
    }
    const int sms = sm_count();
    if (sms < 2) return cudaErrorInvalidDevice;
    const int64_t d_stride = delta_stride(a.N);
    const BackwardLayout at = layout_of(a);
    __nv_bfloat16 *d = half((void *)(ws + at.d[0]));
    float *part = a.db && !at.of_dy ? reinterpret_cast<float *>(ws + at.part[0]) : nullptr;
    int64_t part_rows = (a.M + kDeltaRows - 1) / kDeltaRows;
    if (a.act != WZ_ACT_NONE && !a.pre) {
        MmArgs p = mm_args(a.act, a.device_status);
        forward_product(p, a.M, a.N, a.K, a.x, a.x_stride, a.w, a.w_stride, nullptr, 0);
        p.prob[0].out = d, p.prob[0].out_stride = d_stride;
        p.bias[0] = a.bias;
        p.dy = half(a.dy), p.dy_stride = a.dy_stride;
        p.part[0] = part, p.room_part = room_part(part_bytes(a.M, a.N), a.N);
        MM_TRY(launch_mm(kMmSlope, p, sms, s, &part_rows));
    } else if (a.act != WZ_ACT_NONE || part) {
        DeltaArgs p;
        memset(&p, 0, sizeof(p));
        p.dy = half(a.dy), p.dy_stride = a.dy_stride;
        p.pre[0] = half(a.pre), p.pre_stride[0] = a.pre_stride;
        p.d[0] = d, p.d_stride = d_stride;
        p.part[0] = part;
        p.M = a.M, p.N = a.N, p.act = a.act, p.status = a.device_status;
        p.room_rows = room_rows(a.M), p.room_part = room_part(part_bytes(a.M, a.N), a.N);
        MM_TRY(launch_delta(a.act == WZ_ACT_NONE ? kDeltaSums : kDeltaSlope, p, s));
    }
    Gradients g;
    memset(&g, 0, sizeof(g));
    g.both = 1;
    g.d[0] = a.act == WZ_ACT_NONE ? a.dy : (const void *)d;
    g.d_stride = a.act == WZ_ACT_NONE ? a.dy_stride : d_stride;
    g.w[0] = a.w, g.w_stride[0] = a.w_stride;
    g.x = a.x, g.x_stride = a.x_stride;
    g.dx = a.dx, g.dx_stride = a.dx_stride;
    g.dw[0] = a.dw, g.dw_stride[0] = a.dw_stride;
    g.M = a.M, g.N = a.N, g.K = a.K;
    JoinArgs join = join_args(part, nullptr, a.db, nullptr, part_rows, a.N, a.device_status);
    if (at.of_dy) {
        join.sums.part_rows = 0;
        join.sums.dy = half(a.dy), join.sums.dy_stride = a.dy_stride, join.sums.dy_rows = a.M;
    }
    MM_TRY(launch_gradients(g, at.split, at.beside, ws + at.shares, ws + at.total, join, a.device_status, sms, s));
    return launch_join(join, s);
}

cudaError_t launch_gated_backward(const wz_gated_backward_args &a, char *ws, cudaStream_t s) {
    float *db[2] = {a.db_gate, a.db_up};
    if (a.M == 0) {
        MM_TRY(zero_rows(a.dw_gate, a.dw_gate_stride, a.N, a.K, s));
        MM_TRY(zero_rows(a.dw_up, a.dw_up_stride, a.N, a.K, s));
        JoinArgs join = join_args(nullptr, nullptr, db[0], db[1], 0, a.N, a.device_status);
        return launch_join(join, s);
    }
    const int sms = sm_count();
    if (sms < 2) return cudaErrorInvalidDevice;
    const int64_t d_stride = delta_stride(a.N);
    const BackwardLayout at = layout_of(a);
    __nv_bfloat16 *d[2];
    float *part[2];
    for (int i = 0; i < 2; ++i) {
        d[i] = half((void *)(ws + at.d[i]));
        part[i] = db[i] ? reinterpret_cast<float *>(ws + at.part[i]) : nullptr;
    }
    int64_t part_rows = (a.M + kDeltaRows - 1) / kDeltaRows;
    if (a.gate) {
        DeltaArgs p;
        memset(&p, 0, sizeof(p));
        p.dy = half(a.dout), p.dy_stride = a.dout_stride;
        p.pre[0] = half(a.gate), p.pre_stride[0] = a.gate_stride;
        p.pre[1] = half(a.up), p.pre_stride[1] = a.up_stride;
        p.d[0] = d[0], p.d[1] = d[1], p.d_stride = d_stride;
        p.part[0] = part[0], p.part[1] = part[1];
        p.M = a.M, p.N = a.N, p.act = a.act, p.status = a.device_status;
        p.room_rows = room_rows(a.M), p.room_part = room_part(part_bytes(a.M, a.N), a.N);
        MM_TRY(launch_delta(kDeltaGated, p, s));
    } else {
        MmArgs p = mm_args(a.act, a.device_status);
        forward_product(p, a.M, a.N, a.K, a.x, a.x_stride, a.w_gate, a.w_gate_stride, a.w_up, a.w_up_stride);
        p.prob[0].out = d[0], p.prob[0].out_stride = d_stride;
        p.out2 = d[1], p.out2_stride = d_stride;
        p.bias[0] = a.b_gate, p.bias[1] = a.b_up;
        p.dy = half(a.dout), p.dy_stride = a.dout_stride;
        p.part[0] = part[0], p.part[1] = part[1], p.room_part = room_part(part_bytes(a.M, a.N), a.N);
        MM_TRY(launch_mm(kMmGatedSlope, p, sms, s, &part_rows));
    }
    Gradients g;
    memset(&g, 0, sizeof(g));
    g.both = 2;
    g.d[0] = d[0], g.d[1] = d[1], g.d_stride = d_stride;
    g.w[0] = a.w_gate, g.w[1] = a.w_up, g.w_stride[0] = a.w_gate_stride, g.w_stride[1] = a.w_up_stride;
    g.x = a.x, g.x_stride = a.x_stride;
    g.dx = a.dx, g.dx_stride = a.dx_stride;
    g.dw[0] = a.dw_gate, g.dw[1] = a.dw_up;
    g.dw_stride[0] = a.dw_gate_stride, g.dw_stride[1] = a.dw_up_stride;
    g.M = a.M, g.N = a.N, g.K = a.K;
    JoinArgs join = join_args(part[0], part[1], db[0], db[1], part_rows, a.N, a.device_status);
    MM_TRY(launch_gradients(g, at.split, at.beside, ws + at.shares, ws + at.total, join, a.device_status, sms, s));
    return launch_join(join, s);
}

}  // namespace wz

#ifdef WZ_CHECKED
// Test hook: the limit of the waits that the matrix products give up on; 0: the ordinary one.
extern "C" __attribute__((visibility("default"))) void wz_check_mm_wait(uint64_t ns) {
    wz::check_mm_wait_ns = ns ? ns : wz::kMmTimeoutNs;
}

// Test hook: what the kernels take for out of range although it is not (see check_room).
extern "C" __attribute__((visibility("default"))) void wz_check_mm_room(int what) { wz::check_room = what; }
#endif
