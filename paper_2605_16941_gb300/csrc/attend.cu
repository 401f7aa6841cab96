// attend.cu -- wino_attend: the host side of the attention over a paged cache, and its launches (the kernel: attend_kernel.cuh).
#include "attend_kernel.cuh"

namespace wino {
namespace {

using namespace attend;

int32_t positions_per_tile(const wino_kv_batch &b) { return kTileM / (b.n_q_heads / b.n_kv_heads); }

struct Scratch {
    int32_t quarters, piece;
    size_t ml, o, total;
};

Scratch scratch_layout(const wino_kv_batch &b)
{
    const int32_t dp = b.head_dim <= 64 ? 64 : 128;
    const bool small = b.n_rows <= positions_per_tile(b);  // then no task has rows in its second tile
    Scratch s{};
    s.quarters = small ? (b.n_rows * (b.n_q_heads / b.n_kv_heads) + 31) / 32 : 4;
    s.piece = small ? dp / 2 : dp;
    const size_t warps = (size_t)kMaxCtas * 2 * 2 * (size_t)s.quarters;
    s.ml = (size_t)kMaxCtas * kLevels * 8 * sizeof(int32_t);
    s.o = s.ml + warps * 32 * sizeof(float2);
    s.total = s.o + warps * 32 * (size_t)s.piece * sizeof(float);
    return s;
}

// A tensor map over 16-bit elements in 128-byte swizzled boxes 64 elements wide; strides in elements.
int encode(CUtensorMap *m, int32_t dtype, const void *ptr, int rank, const int64_t *dims, const int64_t *strides,
           const int32_t *box)
{
    auto fn = encode_fn();
    if (!fn)
        return WINO_ERR_CUDA;
    cuuint64_t d[5], st[4];
    cuuint32_t bx[5], es[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        d[i] = (cuuint64_t)dims[i];
        bx[i] = (cuuint32_t)box[i];
        if (i > 0)  // the stride of a single entry is never used; the encoder wants a legal one
            st[i - 1] = (cuuint64_t)(dims[i] > 1 ? strides[i] : 64) * 2;
    }
    return fn(m, dtype == WINO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
              const_cast<void *>(ptr), d, st, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? WINO_OK
               : WINO_ERR_CUDA;
}

}  // namespace

// The units that a batch may have at most, whatever its lengths and however its sequences share rows.
double attend_units(const wino_kv_batch &b)
{
    return (double)b.n_seq * (b.n_rows / (2 * positions_per_tile(b)) + 1) * b.n_kv_heads *
           ((double)b.table_width * b.page_size / kTileN + 1 + kTaskCost);
}

size_t attend_scratch_bytes(const wino_kv_batch &b) { return scratch_layout(b).total; }

namespace attend {

int attend_args(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b, uint8_t *scratch,
                StatusWords *status, AttendArgs *args, CUtensorMap *tq)
{
    const Scratch L = scratch_layout(b);
    AttendArgs &a = *args;
    a = AttendArgs{};
    a.q = q;
    a.out = out;
    a.b = b;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.status = status;
    a.nodes = reinterpret_cast<int32_t *>(scratch);
    a.part_ml = reinterpret_cast<float2 *>(scratch + L.ml);
    a.part_o = reinterpret_cast<float4 *>(scratch + L.o);
    a.quarters = L.quarters;
    a.piece = L.piece;
    a.group = b.n_q_heads / b.n_kv_heads;
    a.positions = positions_per_tile(b);
    a.split = 1;
    a.box_rows = std::min(b.page_size, kTileN);
    a.boxes = kTileN / a.box_rows;
    for (int i = 0; i < 2; ++i) {
        const uint64_t w = (uint64_t)(i + 1) * a.positions;
        a.magic[i] = (uint32_t)(((uint64_t(1) << 32) + w - 1) / w);
    }
    // A part that is left for another CTA to join is written and read in 2 to 3 us where all warps have rows, and in less
    // than 1 us for a few rows, so that runs are longer there.  Runs of 6 / 8 / 12 at least: 18.3 / 16.8 / 16.9 us for a
    // block of 128 + 128 rows behind 1025 slots (32 heads), 26.4 / 26.1 / 29.1 for 16 of 32 + 32; a few rows, one token over
    // 300 / 4097 / 16385 slots, runs of 3: 9.7 / 22.3 / 28.7, of 8: 13.4 / 20.2 / 27.4.
    a.min_units = L.piece * L.quarters >= 256 ? 8 : 3;
    a.wide = attend_units(b) >= 2147483648.0;
    a.page_shift = -1;
    for (int i = 4; i <= 30; ++i)
        if (b.page_size == 1 << i)
            a.page_shift = i;
    a.wide_rows = aligned(out.data, 32) && (b.n_rows == 1 || out.row_stride % 16 == 0) &&
                  (b.n_q_heads == 1 || out.head_stride % 16 == 0);
    const int64_t q_dims[3] = {b.head_dim, b.n_q_heads, b.n_rows}, q_strides[3] = {1, q.head_stride, q.row_stride};
    const int32_t q_box[3] = {64, a.group, a.positions};
    return encode(tq, b.dtype & ~WINO_CACHE_E4M3, q.data, 3, q_dims, q_strides, q_box);
}

}  // namespace attend

int launch_attend(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b, uint8_t *scratch,
                  StatusWords *status, int sm_count, cudaStream_t stream)
{
    AttendArgs a;
    CUtensorMap tq, tk, tv;
    int rc = attend_args(q, out, scale, b, scratch, status, &a, &tq);
    if (rc != WINO_OK)
        return rc;
    // Heads and pages in one coordinate: pages a whole number of heads apart, every index below 2^31.  Only at 128 dims:
    // the map's inner extents are whole halves, and a narrower head's second half would run into its neighbour.
    int64_t per_page = 0, joint_stride = b.head_stride;
    if (b.n_kv_heads == 1) {
        per_page = 1;
        joint_stride = b.page_stride;
    } else if (b.n_pages == 1) {
        per_page = b.n_kv_heads;
    } else if (b.page_stride % b.head_stride == 0) {
        per_page = b.page_stride / b.head_stride;
    }
    const int64_t last = (b.n_pages - 1) * per_page + b.n_kv_heads;
    const bool joint = b.head_dim == 128 && per_page > 0 && last < (int64_t(1) << 31) - 1 && b.slot_stride < (int64_t(1) << 35);
    a.joint = joint ? (int32_t)per_page : 0;
    a.end = joint ? (int32_t)last : b.n_pages;
    a.tile = joint ? TileLayout{2048u, 1024u} : TileLayout{1024u, kHalfBytes};
    for (int i = 0; i < 2; ++i) {
        CUtensorMap *const m = i ? &tv : &tk;
        const uint16_t *const cache = i ? b.v_cache : b.k_cache;
        if (joint) {
            const int64_t dims[5] = {64, 8, 2, b.page_size / 8, last};
            const int64_t strides[5] = {1, b.slot_stride, 64, 8 * b.slot_stride,
                                        joint_stride};
            const int32_t box[5] = {64, 8, 2, a.box_rows / 8, 1};
            rc = encode(m, b.dtype, cache, 5, dims, strides, box);
        } else {
            const int64_t dims[4] = {b.head_dim, b.page_size, b.n_kv_heads, b.n_pages};
            const int64_t strides[4] = {1, b.slot_stride, b.head_stride, b.page_stride};
            const int32_t box[4] = {64, a.box_rows, 1, 1};
            rc = encode(m, b.dtype, cache, 4, dims, strides, box);
        }
        if (rc != WINO_OK)
            return rc;
    }
    const int ctas = std::min(sm_count, kMaxCtas);
    if (b.head_dim <= 64)
        return b.dtype == WINO_BF16 ? launch<64, true, false>(tq, tk, tv, a, ctas, stream)
                                    : launch<64, false, false>(tq, tk, tv, a, ctas, stream);
    return b.dtype == WINO_BF16 ? launch<128, true, false>(tq, tk, tv, a, ctas, stream)
                                : launch<128, false, false>(tq, tk, tv, a, ctas, stream);
}

}  // namespace wino
