// cache_read.cu -- wino_cache_read: K and V of the batch's rows out of the cache's pages, codes as the values they stand for.
//
// Bound by HBM: each element is read and written once; a thread moves 8 elements of a head (16 bytes, from 8 codes or 16 bytes)
// for one row after the other, with the loads of four in flight.  Measured (us, replayed; floors from 6.7 TB/s): 2048 rows of 2 x 32
// heads of 128 from a 16-bit cache 12 (10), 13481 of 2 x 8 15.6 (16.4, in part from the L2 cache), 28931 of 2 x 8 from an 8-bit one 33 (26);
// a row and chunk at a time 23, 21 and 47.
#include "e4m3.cuh"
#include "ptx.cuh"
#include "rope_rows.cuh"

namespace wino {
namespace {

constexpr int kThreads = kRopeThreads;
constexpr int kAhead = 4;  // rows of which a thread has loads in flight

struct ReadArgs {
    wino_heads k, v;
    wino_kv_batch b;
    wino_kv_scales scales;
    StatusWords *status;
    int32_t rows_per_cta;
};

template <bool kScaled, bool kBf16>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ ReadArgs a)
{
    __shared__ Rows<1, kFewRowsPerCta, 0> sh;
    const wino_kv_batch &b = a.b;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    find_rows(b, wino_rope{}, nullptr, true, a.status, sh, row0, n_rows);
    const int chunks = b.head_dim / 8, units = 2 * b.n_kv_heads * chunks;
    for (int y = (int)threadIdx.x; y < units; y += kThreads) {
        const int h = y / chunks, c = y - h * chunks;
        const bool is_v = h >= b.n_kv_heads;
        const int hk = is_v ? h - b.n_kv_heads : h;
        const wino_heads &to = is_v ? a.v : a.k;
        if (!to.data)
            continue;
        const uint16_t *const cache = is_v ? b.v_cache : b.k_cache;
        const uint8_t *const scales = is_v ? a.scales.v_scale : a.scales.k_scale;
        const int64_t at = hk * b.head_stride + 8 * c;
        uint16_t *const dst = to.data + row0 * to.row_stride + hk * to.head_stride + 8 * c;
#pragma unroll 1
        for (int r0 = 0; r0 < n_rows; r0 += kAhead) {
            uint4 out[kAhead];
            uint32_t scale[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int r = min(r0 + k, n_rows - 1);
                if (sh.seq[r] < 0 || sh.page[r] < 0)
                    continue;
                const int64_t slot = at + (int64_t)sh.page[r] * b.page_stride + (int64_t)sh.in_page[r] * b.slot_stride;
                if (kScaled) {
                    const uint2 codes = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(cache) + slot);
                    out[k].x = codes.x;
                    out[k].y = codes.y;
                    scale[k] = scales[scale_at(b, sh.page[r], sh.in_page[r], hk)];
                } else {
                    out[k] = *reinterpret_cast<const uint4 *>(cache + slot);
                }
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int r = r0 + k;
                if (r >= n_rows || sh.seq[r] < 0 || sh.page[r] < 0)
                    continue;
                if (kScaled) {
                    const uint2 codes = make_uint2(out[k].x, out[k].y);
                    const uint32_t f = read_factor<kBf16>(scale[k]);
                    decode4<kBf16>(codes.x, f, out[k].x, out[k].y);
                    decode4<kBf16>(codes.y, f, out[k].z, out[k].w);
                }
                *reinterpret_cast<uint4 *>(dst + r * to.row_stride) = out[k];
            }
        }
    }
}

}  // namespace

cudaError_t launch_cache_read(const wino_heads *k, const wino_heads *v, const wino_kv_batch &b, const wino_kv_scales *scales,
                              StatusWords *status, cudaStream_t stream)
{
    ReadArgs a{};
    if (k)
        a.k = *k;
    if (v)
        a.v = *v;
    a.b = b;
    if (scales)
        a.scales = *scales;
    a.status = status;
    a.rows_per_cta = rope_rows_per_cta(b.n_rows);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((b.n_rows + a.rows_per_cta - 1) / a.rows_per_cta));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (!scales)
        return cudaLaunchKernelEx(&cfg, cache_read_kernel<false, true>, a);
    return (b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16 ? cudaLaunchKernelEx(&cfg, cache_read_kernel<true, true>, a)
                                                     : cudaLaunchKernelEx(&cfg, cache_read_kernel<true, false>, a);
}

}  // namespace wino
