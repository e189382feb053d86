// Matrix products on pairs of SMs: tiles of 256 outputs x up to 256 rows of
//
//   D^T[i][j] = sum_k B[i][k] A[j][k]     i: outputs (lanes of tensor memory), j: rows
//
// cta_group::2: a cluster of two CTAs holds 128 outputs' weights and half of the rows
// each, in six stages of 64 along K (32 KB a CTA), and the sums of its 128 outputs (256
// columns of tensor memory, twice, so that a tile's epilogue overlaps the next one's main
// loop).  With the rows in the columns a tile's row count is a multiple of 32 and not of
// 256: 333 rows are tiles of 192 and 160.  An operand tile is K-major, one box of
// 64 k of its rows, or MN-major, a box of 64 rows of its 64 k each, both with 128-byte
// swizzle; what lies outside an operand arrives as zeros, so any size works.  (A thread
// issues a copy every 55 cycles: with boxes of 64 x 64 and 32 x 64 a step of 192 rows took 0.32 us.)  In a gated product a CTA's 128 lanes are the
// gate's weights of 64 outputs and the up projection's of the same 64.
//   Persistent pairs walk the tiles of up to three products.
// Warps: 0 copies, 1 products (the even CTA's), 2-9 epilogue: 32 rows' sums at a time go
// through one of two buffers in shared memory and are finished row by row.
#include <cstring>
#include <type_traits>

#include "wz_mm.cuh"

namespace wz {

namespace {

constexpr int kOutputs = 128, kStepK = 64;               // outputs of a CTA, K of a stage
constexpr int kOperandBytes = kOutputs * kStepK * 2;     // 16 KB
constexpr int kBoxBytes = kOperandBytes / 2;             // 64 x 64
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;
constexpr int kEpiWarps = 8;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr int kAccCols = 256;                            // the most rows of a tile
constexpr int kChunk = 32;                               // rows of sums in shared memory at a time
constexpr int kChunkFloats = kChunk * kOutputs;
constexpr int kGroupRows = 8;                            // row tiles that are walked together

struct Shared {
    uint64_t full[kStages];
    uint64_t empty[kStages];
    uint64_t tfull[2];
    uint64_t tempty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
};

constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + 2 * kChunkFloats * 4 + sizeof(Shared);
static_assert(kSmemBytes <= 227 * 1024, "shared memory of the pair CTA");

struct Tile {
    int prob, row0, rows, n;   // rows: a multiple of 32, those behind the last one among them
};

// The tiles of pair `pair` of `pairs`, in order: the first product's dealt in turn,
// then the others'.
struct Walk {
    const MmArgs &p;
    int pairs, t;
    __device__ Walk(const MmArgs &args, int pair, int pairs_) : p(args), pairs(pairs_), t(pair) {}
    __device__ bool next(Tile &tile) {
        int x = t, i = 0;
        for (; i < p.problems; ++i) {
            const int tiles = p.prob[i].mt * p.prob[i].nt;
            if (x < tiles) break;
            x -= tiles;
        }
        if (i == p.problems) return false;
        t += pairs;
        // kGroupRows row tiles at a time, output tile by output tile: pairs that run
        // side by side share both operands' tiles in L2
        const MmProblem &q = p.prob[i];
        const int group = x / (kGroupRows * q.nt), left = q.mt - group * kGroupRows;
        const int rows = left < kGroupRows ? left : kGroupRows;
        x -= group * kGroupRows * q.nt;
        tile.prob = i;
        tile.n = x / rows;
        tile.row0 = (group * kGroupRows + x - tile.n * rows) * q.tile_m;
        const int r = q.M - tile.row0;
        tile.rows = r < q.tile_m ? (r + 31) / 32 * 32 : q.tile_m;
        return true;
    }
};

__device__ __forceinline__ void give_up(const MmArgs &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

// Barriers of the epilogue warps; the second says, to all alike, whether all came with `ok`.
__device__ __forceinline__ void epilogue_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool epilogue_all(bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "bar.red.and.pred q, 1, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(ok ? 1u : 0u)
        : "memory");
    return r != 0;
}

}  // namespace

template <int EPI>
__global__ void __launch_bounds__(kThreads, 1) mm_pair_kernel(const __grid_constant__ MmMaps maps,
                                                              const __grid_constant__ MmArgs p) {
    constexpr bool kBoth = mm_both(EPI);
    constexpr int kOwn = kBoth ? kOutputs / 2 : kOutputs;   // outputs of a CTA
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float *sums = reinterpret_cast<float *>(ring + (size_t)kStages * kStageBytes);
    Shared *S = reinterpret_cast<Shared *>(sums + 2 * kChunkFloats);
    volatile int *abort_flag = &S->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();

    if (warp == 2 && lane < p.maps) ptx::prefetch_tmap(&maps.m[lane]);
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
    __syncthreads();
    pdl_trigger();
    ptx::cluster_sync();   // both CTAs' barriers are ready
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;
    Walk walk(p, (int)blockIdx.x >> 1, (int)gridDim.x >> 1);
    Tile t;

    if (warp == 0) {
        if (ptx::elect_one()) {
            // ---------------- copies: this CTA's halves ----------------
            const uint64_t policy = ptx::policy_evict_last();
            const uint32_t full0 = ptx::map_cluster(&S->full[0], 0);   // the even CTA's barriers count both's
            int stage = 0;
            uint32_t phase = 1;
            bool ok = true;
            while (ok && walk.next(t)) {
                const MmProblem &q = p.prob[t.prob];
                const bool a_mn = q.a_mn, b_mn = q.b_mn;
                const int i0 = (t.n * 2 + (int)rank) * kOwn, r0 = t.row0 + (int)rank * (t.rows / 2);
                // an operand K-major is one box (a gated product's weights two), MN-major one for each 64 rows
                const int boxes = a_mn ? (t.rows / 2 + 63) / 64 : 1, ends = q.steps * kStepK;
                const uint32_t bytes = 2u * (uint32_t)(kOperandBytes + (a_mn ? boxes * kBoxBytes : q.box_rows * kStepK * 2));
                for (int seg = 0; ok && seg < q.segments; ++seg) {
                    const CUtensorMap *a = &maps.m[q.a[seg]], *b = &maps.m[q.b[kBoth ? 0 : seg]];
                    const CUtensorMap *b2 = &maps.m[q.b[1]];
                    for (int k = 0; k < ends; k += kStepK) {
                        if (!ptx::mbar_wait(&S->empty[stage], phase, p.wait_ns)) {
                            give_up(p, abort_flag);
                            ok = false;
                            break;
                        }
                        uint8_t *st = ring + stage * kStageBytes;
                        const uint32_t full = full0 + (uint32_t)stage * 8;
                        if (rank == 0) ptx::mbar_arrive_expect_tx(&S->full[stage], bytes);
                        if constexpr (kBoth) {
                            ptx::tma_load_2d_pair(st, b, full, k, i0, policy);
                            ptx::tma_load_2d_pair(st + kBoxBytes, b2, full, k, i0, policy);
                        } else if (b_mn) {
                            ptx::tma_load_2d_pair(st, b, full, i0, k, policy);
                            ptx::tma_load_2d_pair(st + kBoxBytes, b, full, i0 + 64, k, policy);
                        } else {
                            ptx::tma_load_2d_pair(st, b, full, k, i0, policy);
                        }
                        st += kOperandBytes;
                        if (a_mn)
                            for (int h = 0; h < boxes; ++h)
                                ptx::tma_load_2d_pair(st + h * kBoxBytes, a, full, r0 + 64 * h, k, policy);
                        else
                            ptx::tma_load_2d_pair(st, a, full, k, r0, policy);
                        if (++stage == kStages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                }
            }
        }
    } else if (warp == 1 && rank == 0) {
        if (ptx::elect_one()) {
            // ---------------- products of the pair ----------------
            const uint32_t ring32 = ptx::smem_u32(ring);
            int stage = 0, it = 0;
            uint32_t phase = 0;
            bool ok = true;
            while (ok && walk.next(t)) {
                const MmProblem &q = p.prob[t.prob];
                // K-major: rows of 128 bytes, 8 to a kilobyte; 16 k are 32 bytes.
                // MN-major: a kilobyte is 8 k of 64 rows, 64 rows on is the next box; 16 k are 2 KB.
                const uint32_t idesc = ptx::idesc_bf16(2 * kOutputs, t.rows, q.b_mn, q.a_mn);
                const uint64_t w_base = ptx::smem_desc(ring32, q.b_mn ? kBoxBytes : 16, 1024, 2);
                const uint64_t x_base = ptx::smem_desc(ring32 + kOperandBytes, q.a_mn ? kBoxBytes : 16, 1024, 2);
                const uint64_t w_step = q.b_mn ? 128 : 2, x_step = q.a_mn ? 128 : 2;
                const int b = it & 1;
                if (!ptx::mbar_wait(&S->tempty[b], ((uint32_t)(it >> 1) & 1u) ^ 1u, p.wait_ns)) {
                    give_up(p, abort_flag);
                    break;
                }
                ptx::tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(b * kAccCols);
                uint32_t more = 0;
                for (int left = q.segments * q.steps; left > 0; --left) {
                    if (!ptx::mbar_wait(&S->full[stage], phase, p.wait_ns)) {
                        give_up(p, abort_flag);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after();
                    const uint64_t so = (uint64_t)(stage * (kStageBytes >> 4));
#pragma unroll
                    for (int k = 0; k < kStepK / 16; ++k)
                        ptx::mma_bf16_pair(d, w_base + so + k * w_step, x_base + so + k * x_step, idesc, k ? 1u : more);
                    more = 1;
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
        }
    } else if (warp == 1 && rank == 1 && ptx::elect_one()) {
        ptx::mbar_wait(&S->drain, 0, 2 * kMmTimeoutNs);   // the even CTA's last arrivals here
    } else if (warp >= 2) {
        // ---------------- epilogue of this CTA's outputs ----------------
        constexpr int U = kBoth ? 2 : 4;          // rows of a lane in a chunk
        const int quadrant = warp & 3, side = (warp - 2) >> 2, w8 = warp - 2;
        const int own = kBoth ? lane & 15 : lane;
        // the lane's rows of a chunk: first, first + every, ..
        const int first = kBoth ? 4 * w8 + (lane >> 4) : 4 * w8, every = kBoth ? 2 : 1;
        const uint32_t tempty[2] = {ptx::map_cluster(&S->tempty[0], 0), ptx::map_cluster(&S->tempty[1], 0)};
        int it = 0, buffer = 0;
        while (walk.next(t)) {
            const MmProblem &q = p.prob[t.prob];
            const int b = it & 1;
            const int64_t end = t.row0 + t.rows < q.M ? t.row0 + t.rows : q.M;
            MmOutputs o;
            mm_outputs<kBoth>(p, q, o, (t.n * 2 + (int)rank) * kOwn + 4 * own);
            const bool mine = o.left > 0;
            float other[U][4];
            if (mine) mm_fetch<EPI, U>(p, o, other, (int64_t)t.row0 + first, every, end);
            // the warps leave together, on one verdict: their barriers count all of them
            const bool full = ptx::mbar_wait(&S->tfull[b], (uint32_t)(it >> 1) & 1u, p.wait_ns);
            if (!full) give_up(p, abort_flag);
            if (!epilogue_all(full)) break;
            ptx::tc_fence_after();
            const uint32_t tbase = tmem + ((uint32_t)(quadrant * 32) << 16) + (uint32_t)(b * kAccCols);
            mm_with_act(p.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                for (int c0 = 0; t.row0 + c0 < end; c0 += kChunk, buffer ^= 1) {
                    float *at = sums + buffer * kChunkFloats;
                    {
                        float v[16];
                        mm_read16(tbase + (uint32_t)(c0 + 16 * side), v);
                        float *to = at + 16 * side * kOutputs + quadrant * 32 + lane;
#pragma unroll
                        for (int j = 0; j < 16; ++j) to[j * kOutputs] = v[j];
                    }
                    if (t.row0 + c0 + kChunk >= end) {   // the last of the tile's sums are read
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive_cluster(b ? tempty[1] : tempty[0]);
                    }
                    epilogue_barrier();
                    if (mine) {
                        float v[U][4], u[U][4];
#pragma unroll
                        for (int k = 0; k < U; ++k) {
                            const float *row = at + (first + k * every) * kOutputs + 4 * own;
                            const float4 x = *reinterpret_cast<const float4 *>(row);
                            v[k][0] = x.x, v[k][1] = x.y, v[k][2] = x.z, v[k][3] = x.w;
                            if constexpr (kBoth) {
                                const float4 y = *reinterpret_cast<const float4 *>(row + kOutputs / 2);
                                u[k][0] = y.x, u[k][1] = y.y, u[k][2] = y.z, u[k][3] = y.w;
                            }
                        }
                        const int64_t r = (int64_t)t.row0 + c0 + first;
                        mm_finish<EPI, ACT, U>(p, q, o, v, u, other, r, every, end);
                        mm_fetch<EPI, U>(p, o, other, r + kChunk, every, end);
                    }
                }
            });
            if constexpr (EPI == kMmSlope || EPI == kMmGatedSlope) {
                // the warps' sums over their rows, in order; a buffer holds eight warps' of one kind,
                // and in a gated product those of a warp's even and odd rows
                constexpr int kHalves = kBoth ? 2 : 1;
#pragma unroll
                for (int w = 0; w < (kBoth ? 2 : 1); ++w) {
                    float *at = sums + buffer * kChunkFloats;
                    *reinterpret_cast<float4 *>(at + (w8 * kHalves + (kBoth ? lane >> 4 : 0)) * kOwn + 4 * own) =
                        make_float4(o.sum[w][0], o.sum[w][1], o.sum[w][2], o.sum[w][3]);
                    epilogue_barrier();
                    const int i = (int)threadIdx.x - 64, out = (t.n * 2 + (int)rank) * kOwn + i;
                    if (i < kOwn && out < q.N && p.part[w]) {
                        float s = 0.f;
                        for (int k = 0; k < kEpiWarps * kHalves; ++k) s += at[k * kOwn + i];
                        p.part[w][(size_t)(t.row0 / q.tile_m) * q.N + out] = s;
                    }
                    buffer ^= 1;
                }
            }
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

namespace {

// Rows of a tile: 256, or the rows dealt evenly to as few tiles.
int even_tile(int M) {
    const int64_t tiles = ((int64_t)M + kAccCols - 1) / kAccCols;
    return (int)(((int64_t)M + tiles * 32 - 1) / (tiles * 32) * 32);
}

}  // namespace

cudaError_t launch_mm_pair(MmEpilogue epi, MmArgs &p, int sms, bool pdl, cudaStream_t s, int64_t *part_rows) {
    const int tile_n = mm_both(epi) ? kOutputs : 2 * kOutputs;
    int64_t tiles = 0;
    MmMapList list;
    for (int i = 0; i < p.problems; ++i) {
        MmProblem &q = p.prob[i];
        q.tile_m = even_tile(q.M);
        q.box_rows = q.tile_m / 2;   // a CTA's
        q.mt = (int)(((int64_t)q.M + q.tile_m - 1) / q.tile_m);
        q.nt = (q.N + tile_n - 1) / tile_n;
        tiles += (int64_t)q.mt * q.nt;
        for (int j = 0; j < q.segments; ++j) q.a[j] = list.add(q.from_a[j], q.a_mn ? 64 : q.box_rows);
        for (int j = 0; j < (mm_both(epi) ? 2 : q.segments); ++j) q.b[j] = list.add(q.from_b[j], q.b_mn || mm_both(epi) ? 64 : kOutputs);
    }
    if (!list.ok) return cudaErrorInvalidValue;
    p.maps = list.count;
    if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
    if (part_rows) *part_rows = p.prob[0].mt;
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
