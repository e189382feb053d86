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
// issues a copy every 55 cycles: with boxes of 64 x 64 and 32 x 64 a step of 192 rows took
// 0.32 us.)  In a gated product a CTA's 128 lanes are the gate's weights of 64 outputs and
// the up projection's of the same 64.
//   Persistent pairs walk the tiles of up to three products: both gradients of a layer are
// one launch, whose rounds of tiles even out together.
//   What bounds it: a step of 64 along K is max(2 rows, 256 + rows) cycles, products against
// the 64 bytes a cycle that come into an SM, so tiles of 256 rows are bound by the tensor
// cores: 18,662 x 3584 x 3584 253 us (1,892 TFLOP/s), 18,699 x 14336 x 3584 1,138 to 1,196 under
// the power limit; the pipe is busy in 96 % of the active cycles of 6,151 x 3584 x 2 x 14336.  An epilogue takes 4,900 cycles, 64-byte stores at
// 4.8 cycles, which fewer than ten steps do not hide; staging them in shared memory, by rows or for
// TMA stores, was not faster, and TMA writes a whole word where a row ends inside one.
// Warps: 0 copies, 1 products (the even CTA's), 2-17 epilogue, four a TMEM lane quadrant.  A
// lane of the epilogue has an output and takes 16 of its rows at a time: a warp reads and
// writes 64 contiguous bytes of a row, and waits for no other one (in a gated product the
// two that have the gate's and the up projection's sums of the same outputs exchange
// halves of 32 rows, and each finishes one).
#include <algorithm>
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
constexpr int kEpiWarps = 16;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr int kAccCols = 256;                            // the most rows of a tile
constexpr int kUnitRows = 16;                            // rows that an epilogue warp takes at a time
constexpr int kGiveFloats = kUnitRows * 32;              // sums that a warp of a gated product gives away
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

static_assert(kEpiWarps == kSumRows && kGiveFloats >= 33, "mm_column_sums");

constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + kEpiWarps * kGiveFloats * 4 + sizeof(Shared);
static_assert(kSmemBytes <= 227 * 1024, "shared memory of the pair CTA");

struct Tile {
    int prob, row0, rows, n;   // rows: a multiple of 32, those behind the last one among them
    int part, step, steps;     // share of K: the first step and their number
};

// The tiles of a pair, product by product.  A product's first `head` tiles go to the pairs from
// `from` on, in turn: those that had one of the longer tiles before it less than the
// others.  The rest is dealt to all pairs.
struct Walk {
    const MmArgs &p;
    int pair, pairs, i, x, end, stride;
    bool rest;
    __device__ Walk(const MmArgs &args, int pair_, int pairs_) : p(args), pair(pair_), pairs(pairs_), i(0) { begin(); }
    __device__ void begin() {
        const MmProblem &q = p.prob[i];
        rest = pair < q.from || !q.head;
        x = pair - q.from - q.skip;
        if (rest) x = q.head + pair;
        else if (x < 0) x += pairs - q.from;
        end = rest ? q.tiles : q.head;
        stride = rest ? pairs : pairs - q.from;
    }
    __device__ bool next(Tile &tile) {
        while (x >= end) {
            if (!rest) {
                rest = true;
                x = p.prob[i].head + pair;
                end = p.prob[i].tiles;
                stride = pairs;
            } else {
                if (++i == p.problems) {
                    --i;
                    return false;
                }
                begin();
            }
        }
        // kGroupRows row tiles at a time, output tile by output tile: pairs that run
        // side by side share both operands' tiles in L2
        const MmProblem &q = p.prob[i];
        int x = this->x;
        this->x += stride;
        tile.part = 0;
        for (const int each = q.mt * q.nt; x >= each; x -= each) ++tile.part;
        tile.step = tile.part * q.share + min(tile.part, q.more);
        tile.steps = q.share + (tile.part < q.more ? 1 : 0);
        const int group = q.by_group.divide(x), m0 = group * kGroupRows, y = x - m0 * q.nt;
        const bool last = q.mt - m0 < kGroupRows;
        tile.prob = i;
        tile.n = last ? q.by_last.divide(y) : y / kGroupRows;
        tile.row0 = (m0 + y - tile.n * (last ? q.mt - m0 : kGroupRows)) * q.tile_m;
        const int r = q.M - tile.row0;
        tile.rows = r < q.tile_m ? (r + 31) / 32 * 32 : q.tile_m;
        return true;
    }
};

__device__ __forceinline__ void give_up(const MmArgs &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

// Barriers of two warps; the second says, to both alike, whether both came with `ok`.
__device__ __forceinline__ void pair_barrier(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool pair_all(int id, bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %2, 0;\n\t"
        "bar.red.and.pred q, %1, 64, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(id), "r"(ok ? 1u : 0u)
        : "memory");
    return r != 0;
}

// 16 values, `stride` apart, of which the first `count` are there; zeros for the others.
__device__ __forceinline__ void fetch(const __nv_bfloat16 *p, int64_t stride, int count, float (&x)[kUnitRows]) {
    if (count >= kUnitRows) {
#pragma unroll
        for (int j = 0; j < kUnitRows; ++j) x[j] = __bfloat162float(p[j * stride]);
    } else {
#pragma unroll
        for (int j = 0; j < kUnitRows; ++j) x[j] = j < count ? __bfloat162float(p[j * stride]) : 0.f;
    }
}

__device__ __forceinline__ void put(__nv_bfloat16 *p, int64_t stride, int count, const float (&x)[kUnitRows]) {
    if (count >= kUnitRows) {
#pragma unroll
        for (int j = 0; j < kUnitRows; ++j) p[j * stride] = __float2bfloat16_rn(x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kUnitRows; ++j)
            if (j < count) p[j * stride] = __float2bfloat16_rn(x[j]);
    }
}

}  // namespace

template <int EPI>
__global__ void __launch_bounds__(kThreads, 1) mm_pair_kernel(const __grid_constant__ MmMaps maps,
                                                              const __grid_constant__ MmArgs p) {
    constexpr bool kBoth = mm_both(EPI);
    constexpr int kOwn = kBoth ? kOutputs / 2 : kOutputs;   // outputs of a CTA
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float *gives = reinterpret_cast<float *>(ring + (size_t)kStages * kStageBytes);
    Shared *S = reinterpret_cast<Shared *>(gives + kEpiWarps * kGiveFloats);
    volatile int *abort_flag = &S->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_rank();

    if (warp == 2 && lane < p.maps) ptx::prefetch_tmap(&maps.m[lane]);
    if (warp == 0) {
        if (lane < kStages) {
            ptx::mbar_init(&S->full[lane], 1);
            ptx::mbar_init(&S->empty[lane], 1);
        } else if (lane < kStages + 2) {
            ptx::mbar_init(&S->tfull[lane - kStages], 1);
            ptx::mbar_init(&S->tempty[lane - kStages], 2 * kEpiWarps);
        } else if (lane == 31) {
            ptx::mbar_init(&S->drain, 1);
            S->abort = 0;
        }
        ptx::fence_barrier_init();
        __syncwarp();
    }
    pdl_wait();   // an operand may be the previous grid's output
    ptx::cluster_sync();   // both CTAs' barriers are ready
    pdl_trigger();
    if (warp == 1) {
        // (tensor memory is taken while the first copies are under way)
        ptx::tmem_alloc_pair(&S->tmem_base, 2 * kAccCols);
        ptx::tmem_relinquish_pair();
    }
    if (warp != 0) asm volatile("bar.sync 15, %0;" ::"n"(kThreads - 32) : "memory");   // all but the copies' warp
    ptx::tc_fence_after();
    const uint32_t tmem = warp != 0 ? *(volatile uint32_t *)&S->tmem_base : 0;
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
                int left = t.steps, k = t.step * kStepK;
                for (int seg = 0; ok && left > 0; ++seg, k -= ends) {
                    if (k >= ends) continue;   // the share begins in a later segment
                    const CUtensorMap *a = &maps.m[q.a[seg]], *b = &maps.m[q.b[kBoth ? 0 : seg]];
                    const CUtensorMap *b2 = &maps.m[q.b[1]];
                    for (; k < ends && left > 0; k += kStepK, --left) {
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
            // the products' last arrivals here: all stages are free again
            for (int i = 0; ok && i < kStages; ++i) {
                ok = ptx::mbar_wait(&S->empty[stage], phase, p.wait_ns);
                if (!ok) give_up(p, abort_flag);
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1u;
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
                    ok = false;
                    break;
                }
                ptx::tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(b * kAccCols);
                uint32_t more = 0;
                // (two sums, of the even and of the odd steps: see kLongSteps)
                const int second = EPI == kMmSlope || EPI == kMmGatedSlope ? p.second : 0;
                for (int left = t.steps, odd = 0; left > 0; --left, odd ^= 1) {
                    if (!ptx::mbar_wait(&S->full[stage], phase, p.wait_ns)) {
                        give_up(p, abort_flag);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after();
                    const uint64_t so = (uint64_t)(stage * (kStageBytes >> 4));
#pragma unroll
                    for (int k = 0; k < kStepK / 16; ++k)
                        ptx::mma_bf16_pair(odd ? d + (uint32_t)second : d, w_base + so + k * w_step,
                                           x_base + so + k * x_step, idesc, k ? 1u : more);
                    if (!second || odd) more = 1;
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
            // both epilogues' last arrivals here: the sums of all tiles are read
            for (int b = 0; ok && b < 2; ++b) {
                const int uses = (it + 1 - b) >> 1;
                ok = uses == 0 || ptx::mbar_wait(&S->tempty[b], (uint32_t)(uses - 1) & 1u, p.wait_ns);
                if (!ok) give_up(p, abort_flag);
            }
        }
    } else if (warp == 1 && rank == 1 && ptx::elect_one()) {
        ptx::mbar_wait(&S->drain, 0, 2 * kMmTimeoutNs);   // the even CTA's last arrivals here
    } else if (warp >= 2) {
        // ---------------- epilogue of this CTA's outputs ----------------
        constexpr int kSides = kEpiWarps / 4;                   // warps of a quadrant
        constexpr int kStride = kSides * kUnitRows * (kBoth ? 2 : 1);
        const int quadrant = warp & 3, side = (warp - 2) >> 2;
        const int kind = kBoth ? quadrant >> 1 : 0;             // 1: the up projection's sums
        const int barrier = 1 + 2 * side + (quadrant & 1);      // of the two warps with the same outputs
        float *give = gives + (4 * side + quadrant) * kGiveFloats + lane;
        const float *take = gives + (4 * side + (quadrant ^ 2)) * kGiveFloats + lane;
        const uint32_t tempty[2] = {ptx::map_cluster(&S->tempty[0], 0), ptx::map_cluster(&S->tempty[1], 0)};
        if constexpr (EPI == kMmStore) {
            // bias gradients, while the first products are on their way
            const auto barrier = [] { asm volatile("bar.sync 14, %0;" ::"n"(kEpiWarps * 32) : "memory"); };
            for (int x = (int)blockIdx.x; x < p.sums.blocks; x += (int)gridDim.x) {
                mm_column_sums(p.sums, x, (int)threadIdx.x - 64, reinterpret_cast<float (*)[33]>(gives), barrier);
                barrier();
            }
        }
        int it = 0;
        while (walk.next(t)) {
            const MmProblem &q = p.prob[t.prob];
            const int b = it & 1;
            const int rows = q.M - t.row0 < t.rows ? q.M - t.row0 : t.rows;
            const int i = (t.n * 2 + (int)rank) * kOwn + 32 * (kBoth ? quadrant & 1 : quadrant) + lane;
            const bool inside = i < q.N && wz_in_range(p.status, t.row0 >= 0 && i >= 0 && t.row0 + (int64_t)rows <= q.room_rows);
            const int there = inside ? rows : 0;                // of the lane's rows
            const float bias = p.bias[kind] && i < q.N ? __ldg(p.bias[kind] + i) : 0.f;
            // from this warp's first row on, which it is in a gated product when it has finished the exchange
            const int first = side * (kStride / kSides), mine = first + kUnitRows * kind;
            const int64_t row = t.row0 + mine;
            const int64_t s_from = EPI == kMmStore ? p.residual_stride : p.dy_stride, s_out = q.out_stride;
            const __nv_bfloat16 *from = EPI == kMmStore ? p.residual : EPI == kMmGated ? nullptr : p.dy;
            if (from) from += row * s_from + i;
            __nv_bfloat16 *out = q.out + row * s_out + i, *out2 = p.out2 + row * p.out2_stride + i;
            __nv_bfloat16 *pre = p.pre[kind] ? p.pre[kind] + (t.row0 + first) * p.pre_stride[kind] + i : nullptr;
            const int64_t s_pre = p.pre_stride[kind];
            float other[kUnitRows];                             // the residual, or dy
            if (from) fetch(from, s_from, there - mine, other);
            float sum0 = 0.f, sum1 = 0.f;
            const bool full = ptx::mbar_wait(&S->tfull[b], (uint32_t)(it >> 1) & 1u, p.wait_ns);
            if (!full) give_up(p, abort_flag);
            // (two warps that exchange sums leave on one verdict)
            if (kBoth ? !pair_all(barrier, full) : !__all_sync(0xffffffffu, full)) break;
            ptx::tc_fence_after();
            const uint32_t tcol = tmem + ((uint32_t)(quadrant * 32) << 16) + (uint32_t)(b * kAccCols);
            const auto sums = [&](int c, float (&x)[kUnitRows]) {
                mm_read16(tcol + (uint32_t)c, x);
                if ((EPI == kMmSlope || EPI == kMmGatedSlope) && p.second) {
                    float y[kUnitRows];
                    mm_read16(tcol + (uint32_t)(p.second + c), y);
#pragma unroll
                    for (int j = 0; j < kUnitRows; ++j) x[j] += y[j];
                }
            };
            const auto read = [&](bool last) {   // the warp's sums of the tile are read
                if (!last) return;
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive_cluster_local(b ? tempty[1] : tempty[0]);
            };
            read(first >= rows);
            mm_with_act(p.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                for (int c = first; c < rows; c += kStride) {
                    if constexpr (!kBoth) {
                        float x[kUnitRows];
                        sums(c, x);
                        read(c + kStride >= rows);
                        if (EPI == kMmStore && q.sums) {   // a share of K: the sums as they are
                            const int64_t first_sum = ((int64_t)t.part * q.M + t.row0 + c) * q.N + i;
                            float *to = q.sums + first_sum;
                            int count = there - c;
                            if (count > 0 && !wz_in_range(p.status, first_sum + (int64_t)(min(count, kUnitRows) - 1) * q.N < q.room_sums))
                                count = 0;
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j)
                                if (j < count) to[(int64_t)j * q.N] = x[j];
                            continue;
                        }
#pragma unroll
                        for (int j = 0; j < kUnitRows; ++j) x[j] += bias;
                        if (EPI == kMmStore && pre) {
                            put(pre, s_pre, there - c, x);
                            pre += kStride * s_pre;
                        }
                        if constexpr (EPI == kMmStore) {
                            float far_there[kUnitRows];
                            const bool far = mm_far<ACT>(x, far_there);
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j) x[j] = mm_act1<ACT>(x[j]);
                            mm_put_far<false>(far, far_there, x);
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j)
                                if (from) x[j] += other[j];
                        } else {
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j) {
                                float value, slope;
                                mm_slope1<ACT>(x[j], value, slope);
                                x[j] = other[j] * slope;
                                // (rows behind the last have no finite product where a weight has none)
                                sum0 += c + j < there ? x[j] : 0.f;
                            }
                        }
                        if (from) {   // the next rows'
                            from += kStride * s_from;
                            fetch(from, s_from, there - c - kStride, other);
                        }
                        put(out, s_out, there - c, x);
                        out += kStride * s_out;
                    } else {
                        // the gate's warp finishes the first 16 rows, the up projection's the others
                        float x[kUnitRows], y[kUnitRows];   // g and u
                        sums(c, x);
                        sums(c + kUnitRows, y);
                        read(c + kStride >= rows);
#pragma unroll
                        for (int j = 0; j < kUnitRows; ++j) {
                            x[j] += bias;
                            y[j] += bias;
                            give[j * 32] = kind ? x[j] : y[j];
                        }
                        if (EPI == kMmGated && pre) {
                            put(pre, s_pre, there - c, x);
                            put(pre + kUnitRows * s_pre, s_pre, there - c - kUnitRows, y);
                            pre += kStride * s_pre;
                        }
                        pair_barrier(barrier);
#pragma unroll
                        for (int j = 0; j < kUnitRows; ++j) {
                            const float partner = take[j * 32];
                            if (kind) x[j] = partner;   // y: this warp's u of the second half
                            else y[j] = partner;
                        }
                        pair_barrier(barrier);          // both have read
                        const int count = there - c - kUnitRows * kind;
                        float far_there[kUnitRows];
                        if constexpr (EPI == kMmGated) {
                            const bool far = mm_far<ACT>(x, far_there);
                            mm_far_times(far, far_there, y);
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j) x[j] = mm_act1<ACT>(x[j]) * y[j];
                            mm_put_far<true>(far, far_there, x);
                        } else {
                            const bool far = mm_far<ACT>(x, far_there);
                            mm_far_times(far, far_there, other);
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j) {
                                float value, slope;
                                mm_slope1<ACT>(x[j], value, slope);
                                x[j] = other[j] * y[j] * slope;
                                y[j] = other[j] * value;
                                sum0 += j < count ? x[j] : 0.f;
                            }
                            mm_put_far<true>(far, far_there, y);
#pragma unroll
                            for (int j = 0; j < kUnitRows; ++j) sum1 += j < count ? y[j] : 0.f;
                            from += kStride * s_from;
                            fetch(from, s_from, count - kStride, other);
                            put(out2, p.out2_stride, count, y);
                            out2 += kStride * p.out2_stride;
                        }
                        put(out, s_out, count, x);
                        out += kStride * s_out;
                    }
                }
            });
            if constexpr (EPI == kMmSlope || EPI == kMmGatedSlope) {
                // each warp's sums over its rows are a row of their own
                const size_t at = (size_t)((t.row0 / q.tile_m) * kSides * (kBoth ? 2 : 1) + (kBoth ? 2 * side + kind : side)) * q.N + i;
                if (i < q.N && (p.part[0] || p.part[1]) && wz_in_range(p.status, at < (size_t)p.room_part)) {
                    if (p.part[0]) p.part[0][at] = sum0;
                    if (kBoth && p.part[1]) p.part[1][at] = sum1;
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
    // No commit or arrival is under way to either CTA: each barrier's last phase has been waited for in the CTA that has
    // it, full and tfull by the products and the epilogue, empty, tempty and drain above (a wait that ran out instead
    // has been followed by the two milliseconds).  So the barrier has nothing to order, and waits for no store.
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
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
    cuuint32_t box[2] = {(cuuint32_t)kStepK, (cuuint32_t)box_rows};
    cuuint32_t es[2] = {1, 1};
    ok = ok && enc && count < kMmMaps &&
         enc(&maps.m[count], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(o.base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    return count++;
}

namespace {

// What a tile takes: a step is bound by its products, two cycles a row, or by what a CTA's
// 128 outputs and half of the rows bring in, 64 bytes a cycle; the epilogue takes 5,000 cycles.
int64_t tile_cost(const MmProblem &q) {
    return std::max<int64_t>((int64_t)(q.share + 1) * std::max(2 * q.tile_m, 256 + q.tile_m), 5000);
}

}  // namespace

// The rows dealt evenly to as few tiles of at most `most` rows as hold them.
static int even_tile(int64_t M, int most) {
    const int64_t k = (M + most - 1) / most;
    return (int)((M + k * 32 - 1) / (k * 32) * 32);
}

// Cycles of the rounds of a product's tiles on the pairs, for each step of K.
static int64_t rounds_cost(int64_t M, int64_t tile, int64_t output_tiles) {
    const int64_t tiles = (std::max<int64_t>(M, 1) + tile - 1) / tile * output_tiles;
    return (tiles + kPlanPairs - 1) / kPlanPairs * std::max<int64_t>(2 * tile, 256 + tile);
}

// Rows of a tile: dealt evenly to as few tiles as hold them, or to one or two more where that makes the
// rounds of tiles on the pairs cheaper (741 rows x 37 output tiles: 148 tiles of 192 rows are two rounds as
// 111 of 256 are).
int mm_pair_tile(int64_t M, int64_t output_tiles) {
    const int64_t least = M > 0 ? (M + kAccCols - 1) / kAccCols : 1;
    int best = 0;
    int64_t cost = 0;
    for (int64_t k = least; k <= least + (least <= 8 ? 2 : 0); ++k) {
        const int64_t tile = (std::max<int64_t>(M, 1) + k * 32 - 1) / (k * 32) * 32;
        const int64_t t = rounds_cost(M, tile, output_tiles);
        if (!best || t < cost) {
            best = (int)tile;
            cost = t;
        }
    }
    return best;
}

cudaError_t launch_mm_pair(MmEpilogue epi, MmArgs &p, int sms, cudaStream_t s, int64_t *part_rows) {
    const int tile_n = mm_both(epi) ? kOutputs : 2 * kOutputs;
    int64_t tiles = 0;
    MmMapList list;
    for (int i = 0; i < p.problems; ++i) {
        MmProblem &q = p.prob[i];
        q.nt = (q.N + tile_n - 1) / tile_n;
        if (!q.tile_m) q.tile_m = mm_pair_tile(q.M, q.nt);
        if (i == 0) {
            // Two sums where they are needed, and where tiles of half the rows have little more to do: their
            // epilogues are shorter too.  Gated slopes of 741 x 1152 x 4616 take 24.5 us with and without (1.29
            // times the rounds), of 4,103 rows 88 with and 77 without (1.33).
            const int half = std::min(q.tile_m, even_tile(q.M, kAccCols / 2));
            const bool two = (epi == kMmSlope || epi == kMmGatedSlope) && q.steps > 1 &&
                             (q.steps > kLongSteps ||
                              10 * rounds_cost(q.M, half, q.nt) <= 13 * rounds_cost(q.M, q.tile_m, q.nt));
            p.second = two ? kAccCols / 2 : 0;
            if (two) q.tile_m = half;
        }
        q.box_rows = q.tile_m / 2;   // a CTA's
        q.mt = (int)(((int64_t)q.M + q.tile_m - 1) / q.tile_m);
        q.split = q.sums ? q.split : 1;
        if ((int64_t)q.mt * q.nt > INT32_MAX / 32 || (int64_t)q.mt * q.nt * q.split > INT32_MAX / 2) return cudaErrorInvalidValue;
        q.share = q.segments * q.steps / q.split;
        q.more = q.segments * q.steps % q.split;
        q.tiles = q.mt * q.nt * q.split;
        tiles += q.tiles;
        q.by_group.set((uint32_t)(kGroupRows * q.nt));
        q.by_last.set((uint32_t)(q.mt % kGroupRows ? q.mt % kGroupRows : kGroupRows));
        for (int j = 0; j < q.segments; ++j) q.a[j] = list.add(q.from_a[j], q.a_mn ? 64 : q.box_rows);
        for (int j = 0; j < (mm_both(epi) ? 2 : q.segments); ++j) q.b[j] = list.add(q.from_b[j], q.b_mn || mm_both(epi) ? 64 : kOutputs);
    }
    if (!list.ok) return cudaErrorInvalidValue;
    p.maps = list.count;
    if (part_rows) *part_rows = (int64_t)p.prob[0].mt * (kEpiWarps / 4) * (mm_both(epi) ? 2 : 1);
    const void *fn = epi == kMmStore   ? (const void *)mm_pair_kernel<kMmStore>
                     : epi == kMmGated ? (const void *)mm_pair_kernel<kMmGated>
                     : epi == kMmSlope ? (const void *)mm_pair_kernel<kMmSlope>
                                       : (const void *)mm_pair_kernel<kMmGatedSlope>;
    cudaError_t e = allow_smem(fn, kSmemBytes);
    if (e != cudaSuccess) return e;
    const int pairs = (int)(tiles < sms / 2 ? tiles : sms / 2);
    // after a product that does not come out even, the pairs that had a tile less take as many
    // tiles of the next ones first as make up for it
    int behind = 0, skip = 0;   // the first of these pairs (0: none), and whose turn it is among them
    int64_t lag = 0;            // what they have to make up for
    for (int i = 0; i < p.problems; ++i) {
        MmProblem &q = p.prob[i];
        const int64_t cost = tile_cost(q), each = behind ? (lag + cost / 2) / cost : 0;
        const int few = pairs - behind;
        q.head = (int)std::min<int64_t>(q.tiles, each * few);
        q.from = q.head ? behind : 0;
        q.skip = q.head ? skip : 0;
        if (q.head && q.head == q.tiles) {
            lag -= (skip + q.head) / few * cost;
            skip = (skip + q.head) % few;
            continue;
        }
        behind = (q.tiles - q.head) % pairs;
        lag = cost;
        skip = 0;
    }
    void *args[] = {&list.maps, &p};
    return launch_kernel(fn, dim3(2 * pairs), dim3(kThreads), kSmemBytes, s, args, true, 2);
}

}  // namespace wz
