// Matrix products on pairs of SMs: tiles of 256 rows x 256 columns of
//
//   D[i][j] = sum_k A[i][k] B[j][k]
//
// with what follows a layer's product (bias, activation, residual, the gated product,
// the slopes of the backward pass) applied to the fp32 sums.
//
// cta_group::2: a cluster of two CTAs holds 128 rows of A and 128 of B each, in six
// stages of 64 along K (32 KB a CTA), and 128 rows of D (256 columns of tensor memory,
// twice, so that a tile's epilogue overlaps the next one's main loop).  An operand
// tile is two boxes of 64 x 64 with 128-byte swizzle, K-major (64 rows of 64 k) or
// MN-major (64 k of 64 rows); what lies outside an operand arrives as zeros, so any
// size works.  In a gated product the even CTA's B is the gate's weights and the odd
// one's the up projection's: columns 0 .. 127 of D are g and 128 .. 255 are u of the
// same 128 outputs, and a thread has both.
//   Persistent pairs walk the tiles of up to three products.
// Warps: 0 copies, 1 products (the even CTA's), 2-9 epilogue (two a TMEM lane
// quadrant, half of the columns each).
#include <cstring>
#include <type_traits>

#include "wz_mm.cuh"

namespace wz {

namespace {

constexpr int kRows = 128, kStepK = 64;              // rows of an operand tile of a CTA, K of a stage
constexpr int kOperandBytes = kRows * kStepK * 2;    // 16 KB
constexpr int kBoxBytes = kOperandBytes / 2;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;
constexpr int kEpiWarps = 8;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr int kAccCols = 256;
constexpr int kGroupRows = 8;                        // row tiles that are walked together

struct Shared {
    uint64_t full[kStages];
    uint64_t empty[kStages];
    uint64_t tfull[2];
    uint64_t tempty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};

constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + sizeof(Shared);
static_assert(kSmemBytes <= 227 * 1024, "shared memory of the pair CTA");

struct Tile {
    int prob, m, n;
};

// The tiles of pair `pair` of `pairs`, in order: the first product's dealt in turn,
// then the others'.
struct Walk {
    const MmArgs &p;
    int pair, pairs, t;
    __device__ Walk(const MmArgs &args, int pair_, int pairs_) : p(args), pair(pair_), pairs(pairs_), t(pair_) {}
    __device__ bool next(Tile &tile) {
        int x = t, i = 0;
        for (; i < p.problems; ++i) {
            const int tiles = p.prob[i].mt * p.prob[i].nt;
            if (x < tiles) break;
            x -= tiles;
        }
        if (i == p.problems) return false;
        t += pairs;
        // kGroupRows row tiles at a time, column by column: pairs that run side by
        // side share both operands' tiles in L2
        const MmProblem &q = p.prob[i];
        const int group = x / (kGroupRows * q.nt), left = q.mt - group * kGroupRows;
        const int rows = left < kGroupRows ? left : kGroupRows;
        x -= group * kGroupRows * q.nt;
        tile.prob = i;
        tile.n = x / rows;
        tile.m = group * kGroupRows + x - tile.n * rows;
        return true;
    }
};

__device__ __forceinline__ void give_up(const MmArgs &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

// 128 rows r0 .. and 64 k of an operand.
__device__ __forceinline__ void load_operand(uint8_t *dst, const CUtensorMap *m, uint32_t bar, int mn, int r0, int k0,
                                             uint64_t policy) {
    if (mn) {
        ptx::tma_load_2d_pair(dst, m, bar, r0, k0, policy);
        ptx::tma_load_2d_pair(dst + kBoxBytes, m, bar, r0 + 64, k0, policy);
    } else {
        ptx::tma_load_2d_pair(dst, m, bar, k0, r0, policy);
        ptx::tma_load_2d_pair(dst + kBoxBytes, m, bar, k0, r0 + 64, policy);
    }
}

// 32 columns of the warp's rows.
__device__ __forceinline__ void read_columns(uint32_t tcol, float (&x)[32]) {
    uint32_t v[32];
    ptx::tmem_ld_32x32b_x32(tcol, v);
    ptx::tmem_ld_wait();
    ptx::reg_fence32(v);
#pragma unroll
    for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(v[j]);
}

// Columns n .. n + 31 of a row of a product, at tcol in tensor memory.
template <int ACT>
__device__ __forceinline__ void store_columns(const MmArgs &p, const MmProblem &q, uint32_t tcol, int row, int n) {
    float x[32];
    read_columns(tcol, x);
    const int left = q.N - n;
    mm_add_bias(p.bias[0] ? p.bias[0] + n : nullptr, x, left);
    if (row >= q.M) return;
    if (p.pre[0]) mm_store(p.pre[0] + row * p.pre_stride[0] + n, x, left);
#pragma unroll
    for (int j = 0; j < 32; ++j) x[j] = mm_act1<ACT>(x[j]);
    if (p.residual) {
        float r[32];
        mm_load(p.residual + row * p.residual_stride + n, r, left);
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] += r[j];
    }
    mm_store(q.out + row * q.out_stride + n, x, left);
}

template <int ACT>
__device__ __forceinline__ void gated_columns(const MmArgs &p, const MmProblem &q, uint32_t tcol, int row, int n) {
    float g[32], u[32];
    read_columns(tcol, g);
    read_columns(tcol + kAccCols / 2, u);
    const int left = q.N - n;
    mm_add_bias(p.bias[0] ? p.bias[0] + n : nullptr, g, left);
    mm_add_bias(p.bias[1] ? p.bias[1] + n : nullptr, u, left);
    if (row >= q.M) return;
    if (p.pre[0]) {
        mm_store(p.pre[0] + row * p.pre_stride[0] + n, g, left);
        mm_store(p.pre[1] + row * p.pre_stride[1] + n, u, left);
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) g[j] = mm_act1<ACT>(g[j]) * u[j];
    mm_store(q.out + row * q.out_stride + n, g, left);
}

// The sums over the warp's 32 rows, of which those behind M count nothing.
__device__ __forceinline__ void store_sums(float *part, const MmProblem &q, float (&d)[32], int row, int n) {
    if (row >= q.M) {
#pragma unroll
        for (int j = 0; j < 32; ++j) d[j] = 0.f;
    }
    const float sum = mm_column_sum(d);
    const int lane = threadIdx.x & 31, first = row - lane;
    if (first < q.M && lane < q.N - n) part[(size_t)(first >> 5) * q.N + n + lane] = sum;
}

template <int ACT>
__device__ __forceinline__ void slope_columns(const MmArgs &p, const MmProblem &q, uint32_t tcol, int row, int n) {
    float x[32], dy[32];
    read_columns(tcol, x);
    const int left = q.N - n;
    mm_add_bias(p.bias[0] ? p.bias[0] + n : nullptr, x, left);
    if (row < q.M) {
        mm_load(p.dy + row * p.dy_stride + n, dy, left);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float value, slope;
            mm_slope1<ACT>(x[j], value, slope);
            x[j] = dy[j] * slope;
        }
        mm_store(q.out + row * q.out_stride + n, x, left);
    }
    if (p.part[0]) store_sums(p.part[0], q, x, row, n);
}

template <int ACT>
__device__ __forceinline__ void gated_slope_columns(const MmArgs &p, const MmProblem &q, uint32_t tcol, int row, int n) {
    float g[32], u[32];
    read_columns(tcol, g);
    read_columns(tcol + kAccCols / 2, u);
    const int left = q.N - n;
    mm_add_bias(p.bias[0] ? p.bias[0] + n : nullptr, g, left);
    mm_add_bias(p.bias[1] ? p.bias[1] + n : nullptr, u, left);
    if (row < q.M) {
        float dy[32];
        mm_load(p.dy + row * p.dy_stride + n, dy, left);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float value, slope;
            mm_slope1<ACT>(g[j], value, slope);
            g[j] = dy[j] * u[j] * slope;
            u[j] = dy[j] * value;
        }
        mm_store(q.out + row * q.out_stride + n, g, left);
        mm_store(p.out2 + row * p.out2_stride + n, u, left);
    }
    if (p.part[0]) store_sums(p.part[0], q, g, row, n);
    if (p.part[1]) store_sums(p.part[1], q, u, row, n);
}

}  // namespace

template <int EPI>
__global__ void __launch_bounds__(kThreads, 1) mm_pair_kernel(const __grid_constant__ MmMaps maps,
                                                              const __grid_constant__ MmArgs p) {
    constexpr bool kBoth = mm_both(EPI);
    constexpr int kTileN = kBoth ? kAccCols / 2 : kAccCols;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Shared *S = reinterpret_cast<Shared *>(ring + (size_t)kStages * kStageBytes);
    volatile int *abort_flag = &S->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(&S->full[s], 1);
            ptx::mbar_init(&S->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(&S->tfull[b], 1);
            ptx::mbar_init(&S->tempty[b], 2 * kEpiWarps);
        }
        ptx::mbar_init(&S->drain, 1);
        S->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == 1) {
        ptx::tmem_alloc_pair(&S->tmem_base, 2 * kAccCols);
        ptx::tmem_relinquish_pair();
    }
    pdl_wait();   // an operand may be the previous grid's output
    pdl_trigger();
    __syncthreads();
    ptx::cluster_sync();   // both CTAs' barriers are ready
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;
    Walk walk(p, (int)blockIdx.x >> 1, (int)gridDim.x >> 1);
    Tile t;

    if (warp == 0 && ptx::elect_one()) {
        // ---------------- copies: this CTA's halves ----------------
        const uint64_t policy = ptx::policy_evict_last();
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && !*abort_flag && walk.next(t)) {
            const MmProblem &q = p.prob[t.prob];
            const int m0 = t.m * 2 * kRows + (int)rank * kRows;
            const int n0 = kBoth ? t.n * kTileN : t.n * kTileN + (int)rank * kRows;
            for (int seg = 0; ok && seg < q.segments; ++seg) {
                const CUtensorMap *a = &maps.m[q.a[seg]], *b = &maps.m[q.b[kBoth ? (int)rank : seg]];
                for (int ks = 0; ks < q.steps; ++ks) {
                    if (!ptx::mbar_wait(&S->empty[stage], phase ^ 1u, p.wait_ns)) {
                        give_up(p, abort_flag);
                        ok = false;
                        break;
                    }
                    uint8_t *st = ring + (size_t)stage * kStageBytes;
                    const uint32_t full = ptx::map_cluster(&S->full[stage], 0);
                    if (rank == 0) ptx::mbar_arrive_expect_tx(&S->full[stage], 2u * kStageBytes);
                    load_operand(st, a, full, q.a_mn, m0, ks * kStepK, policy);
                    load_operand(st + kOperandBytes, b, full, q.b_mn, n0, ks * kStepK, policy);
                    if (++stage == kStages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else if (warp == 1 && rank == 0 && ptx::elect_one()) {
        // ---------------- products of the pair ----------------
        const uint32_t ring32 = ptx::smem_u32(ring);
        int stage = 0, it = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && !*abort_flag && walk.next(t)) {
            const MmProblem &q = p.prob[t.prob];
            // K-major: rows of 128 bytes, 8 to a kilobyte; 16 k are 32 bytes.
            // MN-major: a kilobyte is 8 k of 64 rows, 64 rows on is the next box; 16 k are 2 KB.
            const uint32_t idesc = ptx::idesc_bf16(2 * kRows, kAccCols, q.a_mn, q.b_mn);
            const uint64_t a_base = ptx::smem_desc(ring32, q.a_mn ? kBoxBytes : 16, 1024, 2);
            const uint64_t b_base = ptx::smem_desc(ring32 + kOperandBytes, q.b_mn ? kBoxBytes : 16, 1024, 2);
            const uint64_t a_step = q.a_mn ? 128 : 2, b_step = q.b_mn ? 128 : 2;
            const int b = it & 1;
            if (!ptx::mbar_wait(&S->tempty[b], ((uint32_t)(it >> 1) & 1u) ^ 1u, p.wait_ns)) {
                give_up(p, abort_flag);
                break;
            }
            ptx::tc_fence_after();
            const uint32_t d = tmem + (uint32_t)(b * kAccCols);
            const int steps = q.segments * q.steps;
            for (int ks = 0; ks < steps; ++ks) {
                if (!ptx::mbar_wait(&S->full[stage], phase, p.wait_ns)) {
                    give_up(p, abort_flag);
                    ok = false;
                    break;
                }
                ptx::tc_fence_after();
                const uint64_t so = (uint64_t)stage * (uint64_t)(kStageBytes >> 4);
#pragma unroll
                for (int k = 0; k < kStepK / 16; ++k)
                    ptx::mma_bf16_pair(d, a_base + so + k * a_step, b_base + so + k * b_step, idesc, (ks | k) ? 1u : 0u);
                ptx::mma_commit_pair(&S->empty[stage]);
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (ok) ptx::mma_commit_pair(&S->tfull[b]);
            ++it;
        }
        ptx::mma_commit_pair(&S->drain);
        ptx::mbar_wait(&S->drain, 0, kMmTimeoutNs);
    } else if (warp == 1 && rank == 1 && ptx::elect_one()) {
        ptx::mbar_wait(&S->drain, 0, 2 * kMmTimeoutNs);   // the even CTA's last arrivals here
    } else if (warp >= 2) {
        // ---------------- epilogue of this CTA's 128 rows ----------------
        const int quadrant = warp & 3;   // TMEM lanes 32 quadrant ..
        const uint32_t tempty[2] = {ptx::map_cluster(&S->tempty[0], 0), ptx::map_cluster(&S->tempty[1], 0)};
        int it = 0;
        while (!*abort_flag && walk.next(t)) {
            const MmProblem &q = p.prob[t.prob];
            const int b = it & 1;
            if (!ptx::mbar_wait(&S->tfull[b], (uint32_t)(it >> 1) & 1u, p.wait_ns)) {
                give_up(p, abort_flag);
                break;
            }
            __syncwarp();
            ptx::tc_fence_after();
            const int row = t.m * 2 * kRows + (int)rank * kRows + quadrant * 32 + lane, n0 = t.n * kTileN;
            const uint32_t tbase = tmem + ((uint32_t)(quadrant * 32) << 16) + (uint32_t)(b * kAccCols);
            mm_with_act(p.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                for (int c = 32 * ((warp - 2) >> 2); c < kTileN && n0 + c < q.N; c += 64) {
                    if constexpr (EPI == kMmStore) store_columns<ACT>(p, q, tbase + c, row, n0 + c);
                    if constexpr (EPI == kMmGated) gated_columns<ACT>(p, q, tbase + c, row, n0 + c);
                    if constexpr (EPI == kMmSlope) slope_columns<ACT>(p, q, tbase + c, row, n0 + c);
                    if constexpr (EPI == kMmGatedSlope) gated_slope_columns<ACT>(p, q, tbase + c, row, n0 + c);
                }
            });
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster(b ? tempty[1] : tempty[0]);
            ++it;
        }
    }
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {
        // copies that were issued before the wait ran out land within microseconds
        const uint64_t t0 = ptx::globaltimer();
        while (ptx::globaltimer() - t0 < 2000000) {
        }
    }
    __syncthreads();
    ptx::cluster_sync();   // no commit or arrival is under way to either CTA
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem, 2 * kAccCols);
    }
}

MmMapList::MmMapList() { memset(&maps, 0, sizeof(maps)); }

int MmMapList::add(const MmOperand &o, int box_rows) {
    auto enc = tmap_encode_fn();
    cuuint64_t dims[2] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows};
    cuuint64_t strides[1] = {(cuuint64_t)o.stride * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t es[2] = {1, 1};
    ok = ok && enc && count < kMmMaps &&
         enc(&maps.m[count], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(o.base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    return count++;
}

cudaError_t launch_mm_pair(MmEpilogue epi, MmArgs &p, int sms, bool pdl, cudaStream_t s, int64_t *part_rows) {
    const int tile_n = mm_both(epi) ? kAccCols / 2 : kAccCols;
    int64_t tiles = 0;
    MmMapList list;
    for (int i = 0; i < p.problems; ++i) {
        MmProblem &q = p.prob[i];
        q.mt = (int)(((int64_t)q.M + 2 * kRows - 1) / (2 * kRows));
        q.nt = (q.N + tile_n - 1) / tile_n;
        tiles += (int64_t)q.mt * q.nt;
        for (int j = 0; j < q.segments; ++j) q.a[j] = list.add(q.from_a[j], 64);
        for (int j = 0; j < (mm_both(epi) ? 2 : q.segments); ++j) q.b[j] = list.add(q.from_b[j], 64);
    }
    if (!list.ok) return cudaErrorInvalidValue;
    if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
    if (part_rows) *part_rows = ((int64_t)p.prob[0].M + 31) / 32;
    const void *fn = epi == kMmStore   ? (const void *)mm_pair_kernel<kMmStore>
                     : epi == kMmGated ? (const void *)mm_pair_kernel<kMmGated>
                     : epi == kMmSlope ? (const void *)mm_pair_kernel<kMmSlope>
                                       : (const void *)mm_pair_kernel<kMmGatedSlope>;
    cudaError_t e = allow_smem(fn, kSmemBytes);
    if (e != cudaSuccess) return e;
    const int pairs = (int)(tiles < sms / 2 ? tiles : sms / 2);
    void *args[] = {&list.maps, &p};
    return launch_kernel(fn, dim3(2 * pairs), dim3(kThreads), kSmemBytes, s, args, pdl, 2);
}

}  // namespace wz
