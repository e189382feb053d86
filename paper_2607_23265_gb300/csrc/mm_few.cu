// Matrix products of few tiles: 128 outputs of a CTA x 16 .. 256 rows,
//
//   D^T[i][j] = sum_k B[i][k] A[j][k]     i: outputs (lanes of tensor memory), j: rows
//
// on one SM each (row tiles in sixteens, for few rows) or on a pair of SMs (in thirty-twos; half
// of the rows' tile a CTA).  What few rows need is a stream of weights that comes from HBM as
// fast as it can, and what few tiles need is to be spread over all SMs: so K is shared by the
// CTAs of a cluster, each with a ring of up to twelve stages in flight, and their sums
// are joined through distributed shared memory, in the order of their ranks, each CTA
// finishing its share of the rows.  No workspace, no second kernel, equal bits each time.
//
// A stage is 64 along K: 128 weight rows (16 KB; in a gated product the gate's and the up
// projection's of the same 64 outputs), K-major, one box of 64 k, or, for the gradient of x,
// MN-major, a box of 64 rows of its 64 k each; and the rows' tile, K-major.  128-byte
// swizzle; what lies outside an operand arrives as zeros.
// Warps: 0 copies, 1 products, then all eight the epilogue.
//
// Measured: 1 x 3584 x 2 x 14336 (rows x K x outputs) 31.0 us (6.6 TB/s; HBM bounds it), 64 x 14336 x 3584
// 19.8 (5.3 TB/s), 333 x 3584 x 4608 15.4, of which 2.1 us are the start, 6.7 the products, at 64
// bytes a cycle into an SM, 3.2 the wait for the cluster's other CTAs and the way of the sums (16-byte
// stores took as long, bulk copies between the CTAs 0.8 us longer) and 1.8 the finish.
//
// Two CTAs share an SM where there are enough of them, so that one's start and epilogue
// overlap the other's products.  Tensor memory is taken by every CTA and held while it waits
// for its cluster, so no CTA may be left without: all take 256 columns at most, and more than
// a third of an SM's shared memory, and the pairs of mm_pair.cu leave too little for one.  Nor
// may the next grid's CTAs come before: some kernels take tensor memory before they wait for
// the grid in front of them.
#include <algorithm>
#include <atomic>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "wz_mm.cuh"

namespace wz {

namespace {

constexpr int kLanes = 128, kStepK = 64;
constexpr int kWeightBytes = kLanes * kStepK * 2;     // 16 KB
constexpr int kBoxBytes = kWeightBytes / 2;           // 64 x 64
constexpr int kRowBytes = kLanes * 4;                 // sums of a row
constexpr int kMaxStages = 12;
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCluster = 8;
// Steps whose weights are sent for before the grid in front has ended: 1 x 3584 x 2 x 14336 (rows x K x outputs) 32.2 us
// without, 30.8 with; 64 x 14336 x 3584 20.0 and 19.5; 32 steps: 36.7 and 20.6.  (Nothing gained in mm_pair.cu.)
constexpr int kAhead = 12;

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
constexpr size_t kSmemTwo = kSmHas / 2 - 2048;        // two CTAs an SM
constexpr size_t kSmemOne = 227 * 1024;
constexpr size_t kSmemLeast = kSmHas / 3;             // not three

__device__ __forceinline__ void give_up(const MmArgs &p, volatile int *abort_flag) {
    *abort_flag = 1;
    if (p.status) atomicOr(p.status, WZ_STATUS_WAIT_TIMEOUT);
}

__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// The two halves of a cluster's barrier; the relaxed arrival does not wait for the thread's stores.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_relaxed() {
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t tmem_columns(int n) { return n <= 32 ? 32u : 1u << (32 - __clz(n - 1)); }

}  // namespace

template <int EPI, bool PAIR>
__global__ void __launch_bounds__(kThreads, 2) mm_few_kernel(const __grid_constant__ MmMaps maps,
                                                             const __grid_constant__ MmArgs p) {
    constexpr bool kBoth = mm_both(EPI);
    constexpr int kOwn = kBoth ? kLanes / 2 : kLanes;     // outputs of a CTA
    constexpr int kGroup = PAIR ? 2 : 1;                  // CTAs of a tile's K share
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Shared *S = reinterpret_cast<Shared *>(ring + p.ring_bytes);
    volatile int *abort_flag = &S->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // this CTA's tile, and its share of K
    const MmProblem &q = p.prob[0];
    const int tile = p.by_cluster.divide((int)blockIdx.x), rank = (int)blockIdx.x - tile * p.cluster;
    const int side = rank % kGroup, part = rank / kGroup;
    const bool shared_k = q.split > 1;
    const int tn = q.by_mt.divide(tile), row0 = (tile - tn * q.mt) * q.tile_m;
    const int out0 = (tn * kGroup + side) * kOwn;
    const int rows = q.M - row0 < q.tile_m ? q.M - row0 : q.tile_m;
    const int columns = (rows + 16 * kGroup - 1) / (16 * kGroup) * (16 * kGroup);   // of the products
    const int step0 = part * q.share + min(part, q.more), step1 = step0 + q.share + (part < q.more ? 1 : 0);
    const uint32_t allocated = tmem_columns(q.tile_m);

    if (warp == 0) {
        if (lane < p.stages) {
            ptx::mbar_init(&S->full[lane], 1);
            ptx::mbar_init(&S->empty[lane], 1);
        }
        if (lane == 31) {
            ptx::mbar_init(&S->done, 1);
            S->abort = 0;
        }
        ptx::fence_barrier_init();
        __syncwarp();
    }
    if (warp == 2 && lane < p.maps) ptx::prefetch_tmap(&maps.m[lane]);
    // the first weights come to L2 while the grid before this one ends
    if (warp == 3 && row0 == 0 && lane < kAhead && step0 + lane < step1) {
        const int seg = (step0 + lane) / q.steps, k = (step0 + lane - seg * q.steps) * kStepK;
        if (kBoth || !q.b_mn) {
            ptx::tma_prefetch_2d(&maps.m[q.b[seg]], k, out0);
            if constexpr (kBoth) ptx::tma_prefetch_2d(&maps.m[q.b[1]], k, out0);
        } else {
            ptx::tma_prefetch_2d(&maps.m[q.b[seg]], out0, k);
            ptx::tma_prefetch_2d(&maps.m[q.b[seg]], out0 + 64, k);
        }
    }
    pdl_wait();   // an operand may be the previous grid's output
    if constexpr (PAIR) ptx::cluster_sync();   // both CTAs' barriers are ready
    else __syncthreads();
    // sums may come here from now on, unless the ring is in their place
    if (shared_k && p.apart) cluster_arrive();

    if (warp == 0) {
        if (ptx::elect_one()) {
            // ---------------- copies: this CTA's weights, and its half of the rows ----------------
            // (a step's issue has to be short: a division for its segment and a look at the abort
            // word made it 390 cycles, more than its products take)
            const uint64_t once = ptx::policy_evict_first(), again = ptx::policy_evict_last();
            const uint64_t weights = q.mt > 1 ? again : once;   // row tiles share them in L2
            const bool b_mn = q.b_mn;
            const int r0 = row0 + side * (columns / 2), steps = q.steps, stages = p.stages;
            const uint32_t bytes = (uint32_t)kGroup * (uint32_t)(kWeightBytes + q.box_rows * kStepK * 2);
            const uint32_t full0 = PAIR ? ptx::map_cluster(&S->full[0], (uint32_t)(rank & ~1)) : 0;
            int seg = step0 / steps, k = (step0 - seg * steps) * kStepK, stage = 0;
            const CUtensorMap *a = &maps.m[q.a[seg]], *b = &maps.m[q.b[seg]], *b2 = &maps.m[q.b[1]];
            uint32_t phase = 1;
            for (int left = step1 - step0; left > 0; --left) {
                if (!ptx::mbar_wait(&S->empty[stage], phase, p.wait_ns)) {
                    give_up(p, abort_flag);
                    break;
                }
                uint8_t *st = ring + stage * p.stage_bytes;
                const auto copy = [&](uint8_t *to, const CUtensorMap *m, int x, int y, uint64_t policy) {
                    if constexpr (PAIR) ptx::tma_load_2d_pair(to, m, full0 + (uint32_t)stage * 8, x, y, policy);
                    else ptx::tma_load_2d(to, m, &S->full[stage], x, y, policy);
                };
                if (side == 0) ptx::mbar_arrive_expect_tx(&S->full[stage], bytes);
                if constexpr (kBoth) {
                    copy(st, b, k, out0, weights);
                    copy(st + kBoxBytes, b2, k, out0, weights);
                } else if (b_mn) {
                    copy(st, b, out0, k, weights);
                    copy(st + kBoxBytes, b, out0 + 64, k, weights);
                } else {
                    copy(st, b, k, out0, weights);
                }
                copy(st + kWeightBytes, a, k, r0, again);
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
    } else if (warp == 1) {
        // (tensor memory is taken while the first copies are under way)
        if constexpr (PAIR) {
            ptx::tmem_alloc_pair(&S->tmem_base, allocated);
            ptx::tmem_relinquish_pair();
        } else {
            ptx::tmem_alloc(&S->tmem_base, allocated);
            ptx::tmem_relinquish();
        }
        __syncwarp();
        pdl_trigger();   // not before: see the top
        if (side == 0 && ptx::elect_one()) {
            // ---------------- products ----------------
            // (layouts: mm_pair.cu)
            const uint32_t d = *(volatile uint32_t *)&S->tmem_base, ring32 = ptx::smem_u32(ring);
            const uint32_t idesc = ptx::idesc_bf16(kGroup * kLanes, columns, q.b_mn, 0);
            const uint64_t w_base = ptx::smem_desc(ring32, q.b_mn ? kBoxBytes : 16, 1024, 2);
            const uint64_t x_base = ptx::smem_desc(ring32 + kWeightBytes, 16, 1024, 2);
            const uint64_t w_step = q.b_mn ? 128 : 2, x_step = 2;
            const int stages = p.stages;
            const uint16_t both = (uint16_t)(3u << (rank & ~1));
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
                for (int k = 0; k < kStepK / 16; ++k) {
                    if constexpr (PAIR)
                        ptx::mma_bf16_pair(d, w_base + so + k * w_step, x_base + so + k * x_step, idesc, k ? 1u : more);
                    else
                        ptx::mma_bf16(d, w_base + so + k * w_step, x_base + so + k * x_step, idesc, k ? 1u : more);
                }
                more = 1;
                if constexpr (PAIR) ptx::mma_commit_pair(&S->empty[stage], both);
                else ptx::mma_commit(&S->empty[stage]);
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if constexpr (PAIR) ptx::mma_commit_pair(&S->done, both);
            else ptx::mma_commit(&S->done);
        }
    }
    __syncwarp();
    // ---------------- epilogue ----------------
    // The sums go through shared memory, a warp writing 32 outputs of 32 rows (those of a shared K
    // to the CTA that finishes the row), and then takes one row's outputs after the other (two
    // rows' in a gated product), four to a lane.
    constexpr int kLanesRow = kOwn / 4, kRowsWarp = 32 / kLanesRow, kRowsAll = kRowsWarp * kWarps;
    const int quadrant = warp & 3, half = warp >> 2, own = lane % kLanesRow, sub = lane / kLanesRow;
    MmOutputs o;
    mm_outputs<kBoth>(p, q, o, out0 + 4 * own);
    // rows that are in shared memory at a time, of each share of K; a multiple of four
    const int chunk = shared_k ? (rows + 4 * q.split - 1) / (4 * q.split) * 4 : p.chunk;
    // times that the lane's stage of the ring is used (here, while the products are under way)
    const int uses = PAIR && warp == 0 && lane < p.stages ? (step1 - step0 + p.stages - 1 - lane) / p.stages : 0;
    // (a wait that gives up says so; the products under way are waited for all the same)
    if (!ptx::mbar_wait(&S->done, 0, p.wait_ns)) {
        give_up(p, abort_flag);
        ptx::mbar_wait(&S->done, 0, 2 * kMmTimeoutNs);
    }
    __syncthreads();
    const bool ok = !*abort_flag;
    ptx::tc_fence_after();
    const uint32_t tmem = S->tmem_base;
    // (the ring is free now: every copy has been used, and every product is complete)
    float *sums = reinterpret_cast<float *>(ring + (shared_k && p.apart ? p.ring_bytes - p.sums_bytes : 0));
    const uint32_t tbase = tmem + ((uint32_t)(quadrant * 32) << 16);
    if (shared_k) {
        if (!p.apart) cluster_arrive();
        cluster_wait();
    }
    for (int c0 = 0; c0 < rows; c0 += chunk) {
        // to shared memory: all of this CTA's sums, or a chunk of them
        const int end = shared_k || c0 + chunk > rows ? rows : c0 + chunk;
        if (ok)
            for (int c = c0 + 32 * half; c < end; c += 64) {
                uint32_t raw[32];
                ptx::tmem_ld_32x32b_x32(tbase + (uint32_t)c, raw);
                int owner = shared_k ? c / chunk : 0, at = c - c0 - owner * chunk;
                ptx::tmem_ld_wait();
                ptx::reg_fence32(raw);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    if (c + j < end) {
                        float *to = sums + (size_t)(part * chunk + at) * kLanes + quadrant * 32 + lane;
                        if (shared_k && owner != part) {
                            const uint32_t there = ptx::map_cluster(to, (uint32_t)(owner * kGroup + side));
#pragma unroll
                            for (int i = 0; i < 4; ++i) st_cluster(there + (uint32_t)(i * kRowBytes), __uint_as_float(raw[j + i]));
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) to[i * kLanes] = __uint_as_float(raw[j + i]);
                        }
                    }
                    at += 4;
                    if (at >= chunk) at -= chunk, ++owner;
                }
            }
        // this CTA's rows
        const int lo = shared_k ? part * chunk : c0, hi = lo + chunk < rows ? lo + chunk : rows;
        const int first = lo + warp * kRowsWarp + sub;   // the lane's first row
        const bool mine = ok && o.left > 0 &&
                          wz_in_range(p.status, o.i >= 0 && row0 >= 0 && lo >= 0 && (int64_t)row0 + hi <= q.room_rows);
        constexpr int U = 2;                              // rows in flight
        MmAt<EPI> at(p, q, (int64_t)row0 + first, o.i);
        float other[U][4];
        if (mine) mm_fetch<EPI, U>(at, o.left, other, kRowsAll, (hi - first + kRowsAll - 1) / kRowsAll);
        // (the last arrivals that free the stages came with the one on done, but nothing orders them before it; 333 x 3584 x
        // 4608 took 0.2 us longer with this right behind that wait, 0.3 at the kernel's end)
        if (c0 == 0 && uses > 0 && !ptx::mbar_wait(&S->empty[lane], (uint32_t)(uses - 1) & 1u, p.wait_ns)) give_up(p, abort_flag);
        __syncwarp();
        if (shared_k) ptx::cluster_sync();
        else __syncthreads();
        if (mine)
            mm_with_act(p.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                for (int c = first; c < hi; c += U * kRowsAll) {
                    const int count = (hi - c + kRowsAll - 1) / kRowsAll;
                    float v[U][4] = {}, u[U][4] = {};
                    const float *from = sums + (size_t)(c - lo) * kLanes + 4 * own;
                    for (int r = 0; r < q.split; ++r, from += (size_t)chunk * kLanes) {
#pragma unroll
                        for (int k = 0; k < U; ++k)
                            if (k < count) {
                                const float4 x = *reinterpret_cast<const float4 *>(from + k * kRowsAll * kLanes);
                                v[k][0] += x.x, v[k][1] += x.y, v[k][2] += x.z, v[k][3] += x.w;
                                if constexpr (kBoth) {
                                    const float4 y = *reinterpret_cast<const float4 *>(from + k * kRowsAll * kLanes + kOwn);
                                    u[k][0] += y.x, u[k][1] += y.y, u[k][2] += y.z, u[k][3] += y.w;
                                }
                            }
                    }
                    mm_finish<EPI, ACT, U>(at, o, v, u, other, kRowsAll, count);
                    at.advance(U * kRowsAll);
                    mm_fetch<EPI, U>(at, o.left, other, kRowsAll, count - U);
                }
            });
        if (end == rows) break;
        __syncthreads();
    }
    ptx::tc_fence_before();
    if (*abort_flag && threadIdx.x == 0) {
        // copies that were issued before the wait ran out land within microseconds
        const uint64_t t0 = ptx::globaltimer();
        while (ptx::globaltimer() - t0 < 2000000) {
        }
    }
    __syncthreads();
    if constexpr (EPI == kMmSlope || EPI == kMmGatedSlope) {
        // the lanes' sums over their rows, in order
        constexpr int kSums = kBoth ? 2 : 1, kEach = kWarps * kRowsWarp;
#pragma unroll
        for (int w = 0; w < kSums; ++w)
            *reinterpret_cast<float4 *>(sums + (w * kEach + warp * kRowsWarp + sub) * kOwn + 4 * own) =
                make_float4(o.sum[w][0], o.sum[w][1], o.sum[w][2], o.sum[w][3]);
        __syncthreads();
        const int w = (int)threadIdx.x / kOwn, i = (int)threadIdx.x % kOwn;
        if (ok && w < kSums && out0 + i < q.N && p.part[w]) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kEach; ++k) s += sums[(w * kEach + k) * kOwn + i];
            const size_t at = (size_t)((row0 / q.tile_m) * q.split + part) * q.N + out0 + i;
            if (wz_in_range(p.status, at < (size_t)p.room_part)) p.part[w][at] = s;
        }
    }
    // a pair's arrivals have all come, to the CTA that has the barrier: full is waited for by the products, empty and done by
    // the epilogue (a wait that ran out has been followed by the two milliseconds)
    if (PAIR) {
        cluster_arrive_relaxed();
        cluster_wait();
    }
    if (warp == 1) {
        ptx::tc_fence_after();
        if constexpr (PAIR) ptx::tmem_dealloc_pair(tmem, allocated);
        else ptx::tmem_dealloc(tmem, allocated);
    }
}

namespace {

int round_up(int x, int to) { return (x + to - 1) / to * to; }

// The most rows of sums that come to a CTA of a shared K: a chunk from each share.
int sums_rows(int tile_m, int split) { return (tile_m + 4 * split - 1) / (4 * split) * 4 * split; }

// Whether a product can take tiles of tile_m rows and `split` shares of K a tile: its sums
// fit into tensor memory and, where they are joined, into shared memory, no share is
// empty, and the sums over rows have a place and a short enough share (kLongSteps).
bool fits(MmEpilogue epi, const MmProblem &q, bool pair, int tile_m, int split) {
    const int even = pair ? 32 : 16;
    if (tile_m % even != 0 || tile_m < even || tile_m > 256) return false;
    if (split > q.segments * q.steps || split * (pair ? 2 : 1) > kMaxCluster) return false;
    const int64_t tiles = ((int64_t)q.M + tile_m - 1) / tile_m;
    return (epi != kMmSlope && epi != kMmGatedSlope) ||
           (tiles * split <= mm_part_rows(q.M) && q.steps <= kLongSteps * split);
}

// Clusters of each size that the current device has room for with one CTA an SM (a property of the device,
// asked for once); null on an error.  With two CTAs an SM there is room for about twice as many; the
// runtime's answer for such sizes is that of one.
struct Places {
    int n[kMaxCluster + 1];
};

const Places *cluster_places() {
    constexpr int kDevices = 64;
    static std::mutex mu;
    static Places places[kDevices];
    static std::atomic<int> known[kDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return nullptr;
    if (known[dev].load(std::memory_order_acquire)) return &places[dev];
    std::lock_guard<std::mutex> lock(mu);
    if (known[dev].load(std::memory_order_relaxed)) return &places[dev];
    const void *fn = (const void *)mm_few_kernel<kMmStore, false>;
    if (allow_smem(fn, kSmemOne) != cudaSuccess) return nullptr;
    for (int size = 1; size <= kMaxCluster; ++size) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)size);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kSmemOne;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)size;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&places[dev].n[size], fn, &cfg) != cudaSuccess || places[dev].n[size] < 1)
            return nullptr;
    }
    known[dev].store(1, std::memory_order_release);
    return &places[dev];
}

#ifdef WZ_CHECKED
int check_kind = 0, check_split = 1, check_tile = 64;
#endif

}  // namespace

bool plan_mm_few(MmEpilogue epi, const MmArgs &p, int sms, MmFewPlan *plan) {
#ifdef WZ_CHECKED
    if (check_kind) {
        if (check_kind == 1) return false;
        plan->pair = check_kind == 3;
        const int even = plan->pair ? 32 : 16;
        plan->tile_m = std::min(round_up(check_tile, even), round_up(p.prob[0].M, even));
        plan->split = fits(epi, p.prob[0], plan->pair, plan->tile_m, check_split) ? check_split : 1;
        return fits(epi, p.prob[0], plan->pair, plan->tile_m, plan->split);
    }
#endif
    // What a call takes, in cycles, fitted to 9 weights (512 x 512 to 14336 x 3584) of 1 to 2,048 rows, plain
    // and gated, with up to 60 plans each: the plan that it chooses is 1.9 % slower than the fastest on
    // average, 19 % at most (48 x 3584 x 4608).  A step of K is bound by what comes into an SM or by its issue, a pair's wide
    // ones by the products; all of them together by HBM (the weights once, up to 3,700 bytes a cycle
    // from two CTAs an SM, 3,200 from 84); clusters that find no place share SMs.  Examples, us, this
    // file's best / mm_pair.cu's: 80 x 14336 x 3584 (rows x K x outputs) 21 / 49, 512 x 14336 x 3584 41 / 66,
    // 333 x 3584 x 4608 15.5 / 17.7, 128 x 1152 x 1152 4.9 / 7.2, but 1100 x 3584 x 3584 30 / 20 and
    // 333 x 1152 x 4608 9.6 / 9.4.
    const MmProblem &q = p.prob[0];
    const int both = mm_both(epi) ? 1 : 0, total = q.segments * q.steps;
    const auto ceil_div = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    const int64_t weights = (int64_t)q.N * total * kStepK * 2 * (both + 1);
    const bool slopes = epi == kMmSlope || epi == kMmGatedSlope;
    // rows that do not begin on 128 bytes come in as two lines each
    const int lines = (q.from_a[0].stride | q.from_b[0].stride) % 64 ? 2 : 1;
    const int64_t outputs = ceil_div((int64_t)q.N << both, 2 * kLanes);
    const int wide = mm_pair_tile(q.M, outputs);
    const int64_t rounds = ceil_div(ceil_div(q.M, wide) * outputs, sms / 2);
    if (rounds > 3) return false;
    const Places *places = cluster_places();
    if (!places) return false;
    int64_t best = 6900 + wide * (both ? 18 : 11) +
                   std::max(rounds * total * std::max(2 * wide, (295 + wide) * lines), weights / 3250);
    bool few = false;
    for (int pair = 0; pair < 2; ++pair) {
        const int even = pair ? 32 : 16, group = pair + 1;
        int last = 0;
        for (int k = 1; k <= 8; ++k) {
            const int64_t tile = ceil_div(ceil_div(q.M, k), even) * even;
            if (tile > 256 || tile == last) continue;
            last = (int)tile;
            const int64_t tiles = ceil_div(q.M, tile) * ceil_div((int64_t)q.N << both, kLanes * group);
            const int64_t step = pair ? std::max<int64_t>({2 * tile, (190 + tile * 11 / 8) * lines, 338})
                                      : std::max<int64_t>((190 + 2 * tile) * lines, 362);
            for (int split = 1; split * group <= kMaxCluster; ++split) {
                const int size = split * group;
                // (clusters of five that fill their places: a row of 3584 x 3584 10.4 us, four 7.8)
                if (size == 5 || size == 7 || !fits(epi, q, pair, (int)tile, split)) continue;
                const int64_t waves = tiles <= places->n[size] ? 1 : 2 * ceil_div(tiles, 2 * places->n[size]);
                if (waves > 6) break;
                // joined: through the cluster's shared memory; else through the CTA's own
                const int64_t end = (split > 1 ? 48 * tile + 173 * size : 200 + 38 * tile) + (slopes ? 25 * tile : 0);
                const int64_t streamed = weights / (3900 - 60000 / std::max<int64_t>(tiles * size, 40));
                const int64_t t = 5100 + std::max(waves * ceil_div(total, split) * step, streamed) + end * (6 * waves + 1) / 7;
                if (t < best) {
                    best = t;
                    few = true;
                    plan->pair = pair;
                    plan->split = split;
                    plan->tile_m = (int)tile;
                }
            }
        }
    }
    return few;
}

cudaError_t launch_mm_few(MmEpilogue epi, MmArgs &p, const MmFewPlan &plan, cudaStream_t s,
                          int64_t *part_rows) {
    const int group = plan.pair ? 2 : 1, own = (mm_both(epi) ? kLanes / 2 : kLanes) * group;
    MmMapList list;
    MmProblem &q = p.prob[0];
    p.cluster = plan.split * group;
    p.by_cluster.set((uint32_t)p.cluster);
    q.tile_m = plan.tile_m;
    q.box_rows = q.tile_m / group;
    q.split = plan.split;
    q.mt = (int)(((int64_t)q.M + q.tile_m - 1) / q.tile_m);
    q.nt = (q.N + own - 1) / own;
    if ((int64_t)q.mt * q.nt > INT32_MAX / kMaxCluster) return cudaErrorInvalidValue;
    q.tiles = q.mt * q.nt;
    q.by_mt.set((uint32_t)q.mt);
    q.share = q.segments * q.steps / q.split;
    q.more = q.segments * q.steps % q.split;
    const int64_t clusters = q.tiles;
    const int dump = q.split > 1 ? std::max(sums_rows(q.tile_m, q.split) * kRowBytes, kWarps * 1024) : 0;
    const int most_steps = q.share + (q.more ? 1 : 0);
    p.stage_bytes = round_up(kWeightBytes + q.box_rows * kStepK * 2, 1024);
    for (int j = 0; j < q.segments; ++j) q.a[j] = list.add(q.from_a[j], q.box_rows);
    for (int j = 0; j < (mm_both(epi) ? 2 : q.segments); ++j)
        q.b[j] = list.add(q.from_b[j], q.b_mn || mm_both(epi) ? 64 : kLanes);
    if (!list.ok || clusters * p.cluster > INT32_MAX) return cudaErrorInvalidValue;
    p.maps = list.count;
    const Places *places = cluster_places();
    if (!places) return cudaErrorInvalidDevice;
    const bool two = dump + kExtra <= kSmemTwo && clusters > places->n[p.cluster];
    const size_t most = (two ? kSmemTwo : kSmemOne) - kExtra;
    // joined sums have a place of their own where six stages are left, or as many as there are steps
    p.apart = dump > 0 && (size_t)(std::min(most_steps, 6) * p.stage_bytes + dump) <= most;
    p.sums_bytes = dump;
    const size_t ring = most - (p.apart ? dump : 0);
    p.stages = (int)std::min<size_t>({(size_t)kMaxStages, ring / p.stage_bytes, (size_t)most_steps});
    // (the slopes' sums over rows take 8 KB at the end)
    p.ring_bytes = p.apart ? p.stages * p.stage_bytes + dump : std::max({p.stages * p.stage_bytes, dump, kWarps * 1024});
    if (p.stages < 1 || (size_t)p.ring_bytes > most) return cudaErrorInvalidValue;
    p.chunk = std::min(256, p.ring_bytes / kRowBytes / 32 * 32);   // (a warp reads 32 rows at a time)
    const size_t smem = std::max(kExtra + (size_t)p.ring_bytes, kSmemLeast + 1);
    if (part_rows) *part_rows = (int64_t)q.mt * q.split;
    const void *fns[4][2] = {
        {(const void *)mm_few_kernel<kMmStore, false>, (const void *)mm_few_kernel<kMmStore, true>},
        {(const void *)mm_few_kernel<kMmGated, false>, (const void *)mm_few_kernel<kMmGated, true>},
        {(const void *)mm_few_kernel<kMmSlope, false>, (const void *)mm_few_kernel<kMmSlope, true>},
        {(const void *)mm_few_kernel<kMmGatedSlope, false>, (const void *)mm_few_kernel<kMmGatedSlope, true>}};
    const void *fn = fns[epi][plan.pair];
    const cudaError_t e = allow_smem(fn, smem);
    if (e != cudaSuccess) return e;
    void *args[] = {&list.maps, &p};
    return launch_kernel(fn, dim3((unsigned)(clusters * p.cluster)), dim3(kThreads), smem, s, args, true,
                         (unsigned)p.cluster);
}

}  // namespace wz

#ifdef WZ_CHECKED
// Test hook: the kernel that products take. kind 0: by their sizes, 1: mm_pair.cu's, 2 and 3: this file's on one SM
// and on pairs, where it can, with K in `split` shares and row tiles of this size.
extern "C" __attribute__((visibility("default"))) void wz_check_mm_plan(int kind, int split, int tile_m) {
    wz::check_kind = kind;
    wz::check_split = split;
    wz::check_tile = tile_m;
}
#endif
