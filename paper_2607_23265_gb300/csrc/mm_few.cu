// Matrix products with few rows, or few tiles: tiles of 128 outputs x 16 .. 256 rows on one SM,
//
//   D^T[i][j] = sum_k B[i][k] A[j][k]     i: outputs (128 lanes of tensor memory), j: rows
//
// so that the number of rows is padded to 16 only.  Weights of few
// rows are a stream that has to come from HBM as fast as it can: K is shared by the CTAs
// of a cluster, each with a ring of up to twelve stages in flight, and their sums are
// joined through distributed shared memory, in the order of their ranks, each CTA
// finishing its share of the rows.  No workspace, no second kernel, equal bits each time.
//
// A stage is 64 along K: 128 outputs' weights (16 KB; a gated product both projections',
// whose sums lie beside one another in tensor memory) and the tile's rows, each K-major,
// one box of 64 k of its rows, or MN-major, a box of 64 rows of its 64 k each, with
// 128-byte swizzle.  What lies outside an operand arrives as zeros.
// Warps: 0 copies, 1 products, then all eight the epilogue.
//
// Tensor memory is taken by every CTA and held while it waits for its cluster.  So no two
// such CTAs may share an SM unless both find room, or clusters could wait for one
// another: a CTA of up to 256 columns asks for more than a third of an SM's shared
// memory, one of 512 for more than two thirds, and the pairs of mm_pair.cu leave too little for either.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "wz_mm.cuh"

namespace wz {

namespace {

constexpr int kOutputs = 128, kStepK = 64;
constexpr int kWeightBytes = kOutputs * kStepK * 2;   // 16 KB
constexpr int kBoxBytes = kWeightBytes / 2;           // 64 x 64
constexpr int kMaxStages = 12;
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCluster = 8;

struct Shared {
    uint64_t full[kMaxStages];
    uint64_t empty[kMaxStages];
    uint64_t done;
    uint32_t tmem_base;
    int abort;
};

constexpr size_t kExtra = 1024 + sizeof(Shared);
// an SM has 228 KB, of which a CTA's first kilobyte is the system's
constexpr size_t kSmHas = 228 * 1024;
constexpr size_t kSmemTwo = kSmHas / 2 - 1024;         // two CTAs an SM
constexpr size_t kSmemOne = 227 * 1024;
constexpr size_t kSmemLeastTwo = kSmHas / 3;           // not three
constexpr size_t kSmemLeastOne = kSmHas * 2 / 3;       // not beside one of the others

__device__ __forceinline__ void give_up(const MmArgs &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

// Four floats of another CTA's shared memory (or of this one's).
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

__device__ __forceinline__ uint32_t tmem_columns(int n) { return n <= 32 ? 32u : 1u << (32 - __clz(n - 1)); }

}  // namespace

template <int EPI>
__global__ void __launch_bounds__(kThreads, 2) mm_few_kernel(const __grid_constant__ MmMaps maps,
                                                             const __grid_constant__ MmArgs p) {
    constexpr bool kBoth = mm_both(EPI);
    constexpr int kSums = kBoth ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Shared *S = reinterpret_cast<Shared *>(ring + p.ring_bytes);
    volatile int *abort_flag = &S->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // this CTA's tile, and its share of K
    const int cluster = p.cluster, id = (int)blockIdx.x / cluster, rank = (int)blockIdx.x - id * cluster;
    int which = 0;
    while (which + 1 < p.problems && id >= p.prob[which + 1].first) ++which;
    const MmProblem &q = p.prob[which];
    const bool shared_k = q.split > 1;
    const int tile = shared_k ? id - q.first : (id - q.first) * cluster + rank;
    const int part = shared_k ? rank : 0;
    const bool active = tile < q.mt * q.nt;
    const int tn = tile / q.mt, tm = tile - tn * q.mt;
    const int row0 = tm * q.tile_m, out0 = tn * kOutputs;
    const int total = q.segments * q.steps;
    const int step0 = (int)((int64_t)total * part / q.split), step1 = (int)((int64_t)total * (part + 1) / q.split);
    const uint32_t columns = tmem_columns(kSums * q.tile_m);

    if (warp == 2 && lane < p.maps) ptx::prefetch_tmap(&maps.m[lane]);
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(&S->full[s], 1);
            ptx::mbar_init(&S->empty[s], 1);
        }
        ptx::mbar_init(&S->done, 1);
        S->abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == 1) {
        ptx::tmem_alloc(&S->tmem_base, columns);
        ptx::tmem_relinquish();
    }
    pdl_wait();   // an operand may be the previous grid's output
    __syncthreads();
    pdl_trigger();
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;

    if (active && warp == 0) {
        if (ptx::elect_one()) {
            // ---------------- copies ----------------
            // (a step's issue has to be short: a division for its segment and a look at the abort
            // word made it 390 cycles, more than its products take)
            const uint64_t once = ptx::policy_evict_first(), again = ptx::policy_evict_last();
            const uint64_t weights = q.mt > 1 ? again : once;   // row tiles share them in L2
            // an operand K-major is one box, MN-major one for each 64 rows
            const bool a_mn = q.a_mn, b_mn = q.b_mn;
            const int boxes = a_mn ? (q.tile_m + 63) / 64 : 1, steps = q.steps, stages = p.stages;
            const uint32_t bytes = (uint32_t)(kSums * kWeightBytes + (a_mn ? boxes * kBoxBytes : q.tile_m * kStepK * 2));
            int seg = step0 / steps, k = (step0 - seg * steps) * kStepK, stage = 0;
            const CUtensorMap *a = &maps.m[q.a[seg]], *b = &maps.m[q.b[seg]], *b2 = &maps.m[q.b[1]];
            uint32_t phase = 1;
            for (int left = step1 - step0; left > 0; --left) {
                if (!ptx::mbar_wait(&S->empty[stage], phase, p.wait_ns)) {
                    give_up(p, abort_flag);
                    break;
                }
                uint8_t *st = ring + stage * p.stage_bytes;
                uint64_t *full = &S->full[stage];
                ptx::mbar_arrive_expect_tx(full, bytes);
                if (b_mn) {
                    ptx::tma_load_2d(st, b, full, out0, k, weights);
                    ptx::tma_load_2d(st + kBoxBytes, b, full, out0 + 64, k, weights);
                } else {
                    ptx::tma_load_2d(st, b, full, k, out0, weights);
                }
                if constexpr (kBoth) ptx::tma_load_2d(st + kWeightBytes, b2, full, k, out0, weights);
                st += kSums * kWeightBytes;
                if (a_mn)
                    for (int h = 0; h < boxes; ++h)
                        ptx::tma_load_2d(st + h * kBoxBytes, a, full, row0 + 64 * h, k, again);
                else
                    ptx::tma_load_2d(st, a, full, k, row0, again);
                k += kStepK;
                if (k == steps * kStepK && seg + 1 < q.segments) {
                    k = 0;
                    ++seg;
                    a = &maps.m[q.a[seg]];
                    b = &maps.m[q.b[seg]];
                }
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (active && warp == 1) {
        if (ptx::elect_one()) {
            // ---------------- products ----------------
            // K-major: rows of 128 bytes, 8 to a kilobyte; 16 k are 32 bytes.
            // MN-major: a kilobyte is 8 k of 64 rows, 64 rows on is the next box; 16 k are 2 KB.
            const uint32_t ring32 = ptx::smem_u32(ring);
            const uint32_t idesc = ptx::idesc_bf16(kOutputs, q.tile_m, q.b_mn, q.a_mn);
            const uint64_t w_base = ptx::smem_desc(ring32, q.b_mn ? kBoxBytes : 16, 1024, 2);
            const uint64_t x_base = ptx::smem_desc(ring32 + kSums * kWeightBytes, q.a_mn ? kBoxBytes : 16, 1024, 2);
            const uint64_t w_step = q.b_mn ? 128 : 2, x_step = q.a_mn ? 128 : 2;
            const int stages = p.stages, second = q.tile_m;
            int stage = 0;
            uint32_t phase = 0, more = 0;
            for (int left = step1 - step0; left > 0; --left) {
                if (!ptx::mbar_wait(&S->full[stage], phase, p.wait_ns)) {
                    give_up(p, abort_flag);
                    break;
                }
                ptx::tc_fence_after();
                const uint64_t so = (uint64_t)(stage * (p.stage_bytes >> 4));
#pragma unroll
                for (int w = 0; w < kSums; ++w)
#pragma unroll
                    for (int k = 0; k < kStepK / 16; ++k)
                        ptx::mma_bf16(tmem + (uint32_t)(w * second),
                                      w_base + so + (uint64_t)(w * (kWeightBytes >> 4)) + k * w_step,
                                      x_base + so + k * x_step, idesc, k ? 1u : more);
                more = 1;
                ptx::mma_commit(&S->empty[stage]);
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            ptx::mma_commit(&S->done);
        }
    }
    __syncwarp();
    // ---------------- epilogue ----------------
    // The sums go through shared memory, a warp writing 32 outputs of 16 rows, and then
    // takes one row's 128 outputs after the other, four to a lane: 256 contiguous bytes.
    const int quadrant = warp & 3, side = warp >> 2;
    const int rows = q.M - row0 < q.tile_m ? q.M - row0 : q.tile_m;
    MmOutputs o;
    mm_outputs<kBoth>(p, q, o, out0 + 4 * lane);
    // (a wait that gives up says so; the products under way are waited for all the same)
    if (active && !ptx::mbar_wait(&S->done, 0, p.wait_ns)) {
        give_up(p, abort_flag);
        ptx::mbar_wait(&S->done, 0, kMmTimeoutNs);
    }
    __syncthreads();
    const bool ok = active && !*abort_flag;
    ptx::tc_fence_after();
    // the ring is free: every copy has been used, and every product is complete
    float *sums = reinterpret_cast<float *>(ring);
    const uint32_t tbase = tmem + ((uint32_t)(quadrant * 32) << 16);
    const int chunk = shared_k ? q.tile_m : p.chunk;   // rows that are in shared memory at a time
    for (int c0 = 0; c0 < rows; c0 += chunk) {
        const int c1 = c0 + chunk < rows ? c0 + chunk : rows;
        if (ok)
            for (int c = c0 + 16 * side; c < c1; c += 32)
#pragma unroll
                for (int w = 0; w < kSums; ++w) {
                    float v[16];
                    mm_read16(tbase + (uint32_t)(w * q.tile_m + c), v);
                    float *to = sums + (size_t)(w * chunk + c - c0) * kOutputs + quadrant * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j) to[j * kOutputs] = v[j];
                }
        if (shared_k) ptx::cluster_sync();
        else __syncthreads();
        if (ok && o.left > 0)
            mm_with_act(p.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                constexpr int U = kBoth ? 1 : 2;   // rows in flight
                // this CTA's share of the rows
                const int share = shared_k ? (rows + q.split - 1) / q.split : c1 - c0;
                const int lo = shared_k ? part * share : c0, hi = lo + share < c1 ? lo + share : c1;
                MmAt<EPI> rows_at(p, q, (int64_t)row0 + lo + warp, o.i);
                for (int c = lo + warp; c < hi; c += U * kWarps) {
                    const int count = (hi - c + kWarps - 1) / kWarps;
                    float v[U][4] = {}, u[U][4] = {}, other[U][4];
                    mm_fetch<EPI, U, false>(rows_at, o.left, other, kWarps, count);
                    const float *at = sums + (size_t)(c - c0) * kOutputs + 4 * lane;
                    if (!shared_k) {
#pragma unroll
                        for (int k = 0; k < U; ++k)
                            if (c + k * kWarps < hi)
#pragma unroll
                                for (int w = 0; w < kSums; ++w) {
                                    const float4 t = *reinterpret_cast<const float4 *>(
                                        at + (size_t)(w * chunk + k * kWarps) * kOutputs);
                                    float(&d)[4] = w ? u[k] : v[k];
                                    d[0] = t.x, d[1] = t.y, d[2] = t.z, d[3] = t.w;
                                }
                    } else {
                        for (int r0 = 0; r0 < q.split; r0 += 4) {
                            float4 t[4][U * kSums];
#pragma unroll
                            for (int r = 0; r < 4; ++r)
#pragma unroll
                                for (int x = 0; x < U * kSums; ++x) {
                                    const int k = x / kSums, w = x % kSums;
                                    t[r][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                                    if (r0 + r < q.split && c + k * kWarps < hi)
                                        t[r][x] = ld_cluster4(ptx::map_cluster(
                                            at + (size_t)(w * chunk + k * kWarps) * kOutputs, (uint32_t)(r0 + r)));
                                }
#pragma unroll
                            for (int r = 0; r < 4; ++r)
#pragma unroll
                                for (int x = 0; x < U * kSums; ++x) {
                                    float(&d)[4] = x % kSums ? u[x / kSums] : v[x / kSums];
                                    d[0] += t[r][x].x, d[1] += t[r][x].y, d[2] += t[r][x].z, d[3] += t[r][x].w;
                                }
                        }
                    }
                    mm_finish<EPI, ACT, U, false>(rows_at, o, v, u, other, kWarps, count);
                    rows_at.advance(U * kWarps);
                }
            });
        if (c1 < rows) __syncthreads();
    }
    ptx::tc_fence_before();
    if (*abort_flag && threadIdx.x == 0) {
        // copies that were issued before the wait ran out land within microseconds
        const uint64_t t0 = ptx::globaltimer();
        while (ptx::globaltimer() - t0 < 2000000) {
        }
    }
    __syncthreads();
    if (shared_k) ptx::cluster_sync();   // nobody reads this CTA's sums any more
    if constexpr (EPI == kMmSlope || EPI == kMmGatedSlope) {
        // the warps' sums over their rows, in order
#pragma unroll
        for (int w = 0; w < kSums; ++w)
            *reinterpret_cast<float4 *>(sums + (w * kWarps + warp) * kOutputs + 4 * lane) =
                make_float4(o.sum[w][0], o.sum[w][1], o.sum[w][2], o.sum[w][3]);
        __syncthreads();
        const int w = (int)threadIdx.x / kOutputs, i = (int)threadIdx.x % kOutputs;
        if (ok && w < kSums && out0 + i < q.N && p.part[w]) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) s += sums[(w * kWarps + k) * kOutputs + i];
            p.part[w][(size_t)(tm * q.split + part) * q.N + out0 + i] = s;
        }
    }
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, columns);
    }
}

namespace {

int round_up(int x, int to) { return (x + to - 1) / to * to; }

// A row tile's bytes of a stage.
int row_bytes(const MmProblem &q, int tile_m) {
    return (q.a_mn ? round_up(tile_m, 64) : tile_m) * kStepK * 2;
}

// Whether a product can take tiles of tile_m rows and `split` CTAs a tile: the sums fit
// into tensor memory and, where they are joined, into shared memory, no CTA is without
// a step, and the sums over rows have a place.
bool fits(MmEpilogue epi, const MmProblem &q, int tile_m, int split) {
    const int sums = mm_both(epi) ? 2 : 1;
    if (tile_m % 16 != 0 || tile_m < 16 || tile_m > 256 || sums * tile_m > 512) return false;
    if (split > 1 && sums * tile_m * kOutputs * 4 + kExtra > kSmemOne) return false;
    if (split > q.segments * q.steps) return false;
    const int64_t tiles = ((int64_t)q.M + tile_m - 1) / tile_m;
    return (epi != kMmSlope && epi != kMmGatedSlope) || tiles * split <= mm_part_rows(q.M);
}

#ifdef WZ_CHECKED
int check_kind = 0, check_cluster = 1, check_tile = 64;
#endif

}  // namespace

bool plan_mm_few(MmEpilogue epi, const MmArgs &p, int sms, MmFewPlan *plan) {
#ifdef WZ_CHECKED
    if (check_kind) {
        if (check_kind == 1) return false;
        plan->cluster = check_cluster;
        for (int i = 0; i < p.problems; ++i) {
            const MmProblem &q = p.prob[i];
            plan->tile_m[i] = std::min(check_tile, round_up(q.M, 16));
            plan->split[i] = fits(epi, q, plan->tile_m[i], check_cluster) ? check_cluster : 1;
            if (!fits(epi, q, plan->tile_m[i], plan->split[i])) return false;
        }
        return true;
    }
#endif
    int cluster = 1;
    for (int i = 0; i < p.problems; ++i) {
        const MmProblem &q = p.prob[i];
        plan->tile_m[i] = round_up(std::min(q.M, 64), 16);
        plan->split[i] = 1;
        if (q.M > 64 || !fits(epi, q, plan->tile_m[i], 1)) return false;
        const int tiles = (q.N + kOutputs - 1) / kOutputs;
        cluster = std::max(1, std::min({kMaxCluster, sms / tiles, q.segments * q.steps}));
    }
    if (p.problems > 1) return false;
    while (!fits(epi, p.prob[0], plan->tile_m[0], cluster)) --cluster;
    plan->cluster = cluster;
    plan->split[0] = cluster;
    return true;
}

cudaError_t launch_mm_few(MmEpilogue epi, MmArgs &p, const MmFewPlan &plan, bool pdl, cudaStream_t s,
                          int64_t *part_rows) {
    const int sums = mm_both(epi) ? 2 : 1;
    MmMapList list;
    int64_t clusters = 0;
    int columns = 0, dump = 0, most_steps = 1;
    p.cluster = plan.cluster;
    p.stage_bytes = 0;
    for (int i = 0; i < p.problems; ++i) {
        MmProblem &q = p.prob[i];
        q.tile_m = plan.tile_m[i];
        q.split = plan.split[i];
        q.mt = (int)(((int64_t)q.M + q.tile_m - 1) / q.tile_m);
        q.nt = (q.N + kOutputs - 1) / kOutputs;
        if ((int64_t)q.mt * q.nt > INT32_MAX / kMaxCluster) return cudaErrorInvalidValue;
        q.first = (int)clusters;
        clusters += q.split > 1 ? q.mt * q.nt : (q.mt * q.nt + plan.cluster - 1) / plan.cluster;
        p.stage_bytes = std::max(p.stage_bytes, sums * kWeightBytes + row_bytes(q, q.tile_m));
        columns = std::max(columns, sums * q.tile_m);
        if (q.split > 1) dump = std::max(dump, sums * q.tile_m * kOutputs * 4);
        most_steps = std::max(most_steps, (q.segments * q.steps + q.split - 1) / q.split);
        for (int j = 0; j < q.segments; ++j) q.a[j] = list.add(q.from_a[j], q.a_mn ? 64 : q.tile_m);
        for (int j = 0; j < (mm_both(epi) ? 2 : q.segments); ++j) q.b[j] = list.add(q.from_b[j], q.b_mn ? 64 : kOutputs);
    }
    if (!list.ok || clusters * plan.cluster > INT32_MAX) return cudaErrorInvalidValue;
    p.stage_bytes = round_up(p.stage_bytes, 1024);
    p.maps = list.count;
    // two CTAs an SM where their tensor memory, and joining sums, allow it
    const bool two = columns <= 256 && dump + kExtra <= kSmemTwo && clusters * plan.cluster > sm_count();
    const size_t most = (two ? kSmemTwo : kSmemOne) - kExtra;
    p.stages = (int)std::min<size_t>({(size_t)kMaxStages, most / p.stage_bytes, (size_t)std::max(most_steps, 1)});
    p.ring_bytes = std::max(p.stages * p.stage_bytes, dump);
    if (p.stages < 1 || (size_t)p.ring_bytes > most) return cudaErrorInvalidValue;
    p.chunk = std::min(256, p.ring_bytes / (sums * kOutputs * 4) / 16 * 16);
    const size_t smem = std::max(kExtra + (size_t)p.ring_bytes,
                                 (columns <= 256 ? kSmemLeastTwo : kSmemLeastOne) + 1);
    if (part_rows) *part_rows = (int64_t)p.prob[0].mt * p.prob[0].split;
    const void *fn = epi == kMmStore   ? (const void *)mm_few_kernel<kMmStore>
                     : epi == kMmGated ? (const void *)mm_few_kernel<kMmGated>
                     : epi == kMmSlope ? (const void *)mm_few_kernel<kMmSlope>
                                       : (const void *)mm_few_kernel<kMmGatedSlope>;
    const cudaError_t e = allow_smem(fn, smem);
    if (e != cudaSuccess) return e;
    void *args[] = {&list.maps, &p};
    return launch_kernel(fn, dim3((unsigned)(clusters * plan.cluster)), dim3(kThreads), smem, s, args, pdl,
                         (unsigned)plan.cluster);
}

}  // namespace wz

#ifdef WZ_CHECKED
// Test hook: the kernel that products take. kind 0: by their sizes, 1: mm_pair.cu's, 2: this file's where it
// can, with clusters and row tiles of these sizes.
extern "C" __attribute__((visibility("default"))) void wz_check_mm_plan(int kind, int cluster, int tile_m) {
    wz::check_kind = kind;
    wz::check_cluster = cluster;
    wz::check_tile = tile_m;
}
#endif
