// attend_scaled.cu -- wino_attend_scaled: wino_attend over a cache of e4m3 codes (the kernel: attend_kernel.cuh).
#include "attend_kernel.cuh"

namespace wino {
namespace attend {

int encode_codes(CUtensorMap *m, const void *cache, const wino_kv_batch &b, int32_t width, int32_t box_rows, bool swizzled)
{
    auto fn = encode_fn();
    if (!fn)
        return WINO_ERR_CUDA;
    const cuuint64_t dims[4] = {(cuuint64_t)b.head_dim, (cuuint64_t)b.page_size, (cuuint64_t)b.n_kv_heads, (cuuint64_t)b.n_pages};
    const int64_t strides[3] = {b.slot_stride, b.head_stride, b.page_stride};
    cuuint64_t st[3];
    for (int i = 0; i < 3; ++i)  // the stride of a single entry is never used; the encoder wants a legal one
        st[i] = (cuuint64_t)(dims[i + 1] > 1 ? strides[i] : 128);
    const cuuint32_t box[4] = {(cuuint32_t)width, (cuuint32_t)box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUtensorMapSwizzle swizzle = !swizzled ? CU_TENSOR_MAP_SWIZZLE_NONE
                                                 : (width == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B);
    // The L2 cache fetches what a head has of a slot and not its neighbour's beside it, which another CTA reads later: 64
    // tokens over up to 32767 slots, layout [slots][heads], 162 us; with 256 bytes 208.
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(cache), dims, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              swizzle, width == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_64B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? WINO_OK
               : WINO_ERR_CUDA;
}

}  // namespace attend

int launch_attend_scaled(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b,
                         const wino_kv_scales &scales, uint8_t *scratch, StatusWords *status, int sm_count, cudaStream_t stream)
{
    using namespace attend;
    AttendArgs a;
    CUtensorMap tq, tk, tv;
    int rc = attend_args(q, out, scale, b, scratch, status, &a, &tq);
    if (rc != WINO_OK)
        return rc;
    a.scales = scales;
    const int ctas = std::min(sm_count, kMaxCtas);
    if (few_rows(b))
        return launch_few(a, ctas, stream);
    a.end = b.n_pages;
    a.tile = TileLayout{1024u, kHalfBytes};
    const int32_t width = b.head_dim <= 64 ? 64 : 128, box_rows = a.box_rows;
    if ((rc = encode_codes(&tk, b.k_cache, b, width, box_rows, false)) != WINO_OK ||
        (rc = encode_codes(&tv, b.v_cache, b, width, box_rows, false)) != WINO_OK)
        return rc;
    const bool bf16 = (b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16;
    if (width == 64)
        return bf16 ? launch<64, true, true>(tq, tk, tv, a, ctas, stream) : launch<64, false, true>(tq, tk, tv, a, ctas, stream);
    return bf16 ? launch<128, true, true>(tq, tk, tv, a, ctas, stream) : launch<128, false, true>(tq, tk, tv, a, ctas, stream);
}

}  // namespace wino
