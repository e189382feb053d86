// Attention over the paged 8-bit cache (wz_attend): which kernel a call takes, its
// workspace, its tensor maps.
//   attend_few.cu   at most 16 query rows (new tokens x heads of a group): decoding
//   attend_many.cu  more: questions and prompts
#include <algorithm>
#include <cstring>

#include "wz_attend.cuh"

namespace wz {

namespace {

bool encode_cache(PFN_cuTensorMapEncodeTiled_v12000 enc, CUtensorMap *m, const wz_kv_cache &c, const void *codes) {
    cuuint64_t dims[3] = {(cuuint64_t)c.D, (cuuint64_t)c.page_tokens, (cuuint64_t)c.pages * c.heads};
    cuuint64_t strides[2] = {(cuuint64_t)c.D, (cuuint64_t)c.D * c.page_tokens};
    cuuint32_t box[3] = {128, (cuuint32_t)c.page_tokens, 1};   // channels past D are filled with zeros
    cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(codes), dims, strides, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct AttendPlan {
    bool few;
    int max_new;
    int splits;              // attend_many: CTAs that share the slots of a row tile
    int paired;              // .. and whose two tiles share them too
    size_t rows;             // rows of pieces in the workspace
    size_t workspace;
};

#ifdef WZ_CHECKED
uint64_t check_wait_ns = kATimeoutNs;
#endif

constexpr size_t kPieceRow = 128 * sizeof(float) + sizeof(float2);

AttendPlan attend_plan(const wz_attend_args &a, int sms) {
    AttendPlan pl;
    pl.max_new = (int)(a.max_new ? std::min<int64_t>(a.max_new, a.T) : a.T);
    const int64_t rows = (int64_t)pl.max_new * (a.Hq / a.cache.heads);
    pl.few = rows <= 16;
    pl.splits = 1;
    pl.paired = 0;
    if (pl.few) {
        pl.rows = (size_t)kFewSlots * 16;
        pl.workspace = pl.rows * kPieceRow + (size_t)a.T * a.cache.heads * sizeof(int2);
        return pl;
    }
    // Few row tiles leave SMs idle: their slots are cut into pieces.  A split costs a
    // CTA's start and end and the pieces' way through memory, about kSplitTiles tiles.
    const int64_t items = (rows + kManyRows - 1) / kManyRows * a.cache.heads * a.B;
    const int64_t tiles = ((int64_t)a.max_pages * a.cache.page_tokens + kATile - 1) / kATile;
    // Up to 128 rows fill one of a CTA's two tiles.  Paired, both work on them, which takes
    // 0.62 to 0.75 of the time a tile, but twice the pieces: 10 tokens of 28/4 heads x 96 on 2 x
    // 328,032 slots 193 us for 237, 32 of 32/8 x 128 on 8 x 4,097 44 for 48; 16 of 28/4 x 128
    // on 18,699, where a CTA has five tiles, 37 for 29.
    double best = 0;
    for (int paired = 0; paired <= (rows <= 128 && items <= kManySlots ? 1 : 0); ++paired)
        for (int s = 1; s <= 32 && (s == 1 || (items * s <= kManySlots && s <= tiles)); ++s) {
            const int64_t waves = (items * s + sms - 1) / sms;
            const double cost = (double)waves * ((double)tiles / s * (paired ? 0.62 : 1.) +
                                                 (paired ? 3 : s > 1 ? 2 : 1) * kSplitTiles);
            if ((s == 1 && !paired) || cost < best) {
                best = cost;
                pl.splits = s;
                pl.paired = paired;
            }
        }
    pl.rows = pl.splits > 1 || pl.paired ? (size_t)(items * pl.splits) * kManyRows : 0;
    pl.workspace = pl.rows * kPieceRow;
    return pl;
}

}  // namespace

size_t attend_workspace_bytes(int64_t T, int Hq) {
    const size_t few = (size_t)kFewSlots * 16 * kPieceRow + (size_t)T * Hq * sizeof(int2);
    const size_t many = (size_t)kManySlots * kManyRows * kPieceRow;
    return T * Hq <= 16 ? few : std::max(few, many);
}

size_t attend_workspace_need(const wz_attend_args &a) { return attend_plan(a, std::max(sm_count(), 1)).workspace; }

cudaError_t launch_attend(const wz_attend_args &a, void *workspace, cudaStream_t s) {
    auto enc = tmap_encode_fn();
    if (!enc) return cudaErrorNotSupported;
    const int sms = sm_count();
    if (sms < 1) return cudaErrorInvalidDevice;
    AttendMaps maps;
    memset(&maps, 0, sizeof(maps));
    if (!encode_cache(enc, &maps.k, a.cache, a.cache.k) || !encode_cache(enc, &maps.v, a.cache, a.cache.v))
        return cudaErrorInvalidValue;
    const AttendPlan pl = attend_plan(a, sms);
    AttendParams p;
    memset(&p, 0, sizeof(p));
    p.q = static_cast<const __nv_bfloat16 *>(a.q);
    p.out = static_cast<__nv_bfloat16 *>(a.out);
    p.q_stride = a.q_stride; p.out_stride = a.out_stride; p.lse = a.lse;
    p.cu = a.cu; p.kv_len = a.kv_len; p.table = a.page_table;
    p.k_scale = a.cache.k_scale; p.v_scale = a.cache.v_scale;
    p.part = static_cast<float *>(workspace);
    p.ml = reinterpret_cast<float2 *>(p.part + pl.rows * 128);
    p.spans = reinterpret_cast<int2 *>(p.ml + pl.rows);
    p.pages = a.cache.pages;
    p.T = (int)a.T; p.B = a.B; p.Hq = a.Hq; p.heads = a.cache.heads; p.G = a.Hq / a.cache.heads;
    p.D = a.cache.D; p.P = a.cache.page_tokens; p.max_pages = a.max_pages; p.max_new = pl.max_new; p.causal = a.causal != 0;
    while (1 << p.shift < p.P) ++p.shift;
    p.scale2 = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)p.D)) * kLog2e;
    p.status = a.device_status;
#ifdef WZ_CHECKED
    p.wait_ns = check_wait_ns;
#endif
    return pl.few ? launch_attend_few(maps, p, pl.max_new, sms, s)
                  : launch_attend_many(maps, p, pl.max_new, pl.splits, pl.paired, s);
}

}  // namespace wz

#ifdef WZ_CHECKED
// Test hook: the limit of the waits that the attention kernels give up on; 0: the ordinary one.
extern "C" __attribute__((visibility("default"))) void wz_check_attend_wait(uint64_t ns) {
    wz::check_wait_ns = ns ? ns : wz::kATimeoutNs;
}
#endif
