// attend_scaled.cu -- wino_attend_scaled: attention of a step's rows over a paged cache of e4m3 codes.
//
// out = softmax(scale Q K^T) V with the running maximum m, sum l and unnormalised product O of an online softmax; a warp per row
// and query head, one slot at a time, 4 dims per lane.
#include "e4m3.cuh"
#include "ptx.cuh"
#include "rope_rows.cuh"

namespace wino {
namespace {

constexpr int kThreads = kRopeThreads;

struct ScaledArgs {
    wino_heads q, out;
    float scale_log2;
    wino_kv_batch b;
    wino_kv_scales scales;
    StatusWords *status;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) attend_scaled_kernel(const __grid_constant__ ScaledArgs a)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    __shared__ Rows<1> sh;
    const wino_kv_batch &b = a.b;
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    const int32_t row = (int32_t)blockIdx.x;
    find_rows(b, wino_rope{}, nullptr, false, a.status, sh, row, 1);
    const int head = (int)(blockIdx.y * (kThreads / 32) + (threadIdx.x >> 5)), lane = (int)threadIdx.x & 31;
    bool ok = true;
    if (sh.seq[0] >= 0 && head < b.n_q_heads) {
        const RowSees sees = row_sees(b, sh.q[0], row - sh.q[0].start);
        const int hk = head / (b.n_q_heads / b.n_kv_heads), c = 4 * lane;
        const bool live = c < b.head_dim;
        float q[4] = {}, o[4] = {}, m = -INFINITY, l = 0.f;
        if (live)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                q[k] = to_f<T>(a.q.data[row * a.q.row_stride + head * a.q.head_stride + c + k]);
        auto values = [&](const uint16_t *cache, const uint8_t *scales, int32_t page, int32_t at, float (&x)[4]) {
            uint32_t lo = 0, hi = 0;
            if (live && page >= 0) {
                const uint8_t *const p = reinterpret_cast<const uint8_t *>(cache) + page * b.page_stride + at * b.slot_stride + hk * b.head_stride;
                decode4<kBf16>(*reinterpret_cast<const uint32_t *>(p + c), read_factor<kBf16>(scales[scale_at(b, page, at, hk)]), lo, hi);
            }
            x[0] = to_f<T>((uint16_t)lo);
            x[1] = to_f<T>((uint16_t)(lo >> 16));
            x[2] = to_f<T>((uint16_t)hi);
            x[3] = to_f<T>((uint16_t)(hi >> 16));
        };
        for (int32_t j = 0; j < sees.lim; ++j) {
            if (j == sees.hole)
                continue;
            const int32_t page = load_page(b, sh.seq[0], j / b.page_size, ok), at = j % b.page_size;
            float x[4];
            values(b.k_cache, a.scales.k_scale, page, at, x);
            float s = q[0] * x[0] + q[1] * x[1] + q[2] * x[2] + q[3] * x[3];
            for (int i = 16; i; i >>= 1)
                s += __shfl_xor_sync(0xffffffffu, s, i);
            const float big = fmaxf(m, s);
            const float f = m == -INFINITY ? 0.f : ptx::ex2((m - big) * a.scale_log2), p = ptx::ex2((s - big) * a.scale_log2);
            m = big;
            l = l * f + p;
            values(b.v_cache, a.scales.v_scale, page, at, x);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                o[k] = o[k] * f + p * x[k];
        }
        if (live)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                a.out.data[row * a.out.row_stride + head * a.out.head_stride + c + k] = from_f<T>(l == 0.f ? 0.f : o[k] / l);
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
    // The last CTA publishes a failure and clears it for the next call.
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.status->finished, 1u) + 1u == gridDim.x * gridDim.y) {
            __threadfence();
            const int32_t failed = -abs(atomicExch(&a.status->current, (int32_t)WINO_OK));
            if (failed && a.status->first == WINO_OK)
                a.status->first = failed;
            a.status->finished = 0;
        }
    }
}

}  // namespace

int launch_attend_scaled(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b,
                         const wino_kv_scales &scales, StatusWords *status, cudaStream_t stream)
{
    const ScaledArgs a{q, out, scale * 1.4426950408889634f, b, scales, status};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)b.n_rows, (unsigned)((b.n_q_heads + 7) / 8));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const bool bf16 = (b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16;
    return (bf16 ? cudaLaunchKernelEx(&cfg, attend_scaled_kernel<__nv_bfloat16>, a)
                 : cudaLaunchKernelEx(&cfg, attend_scaled_kernel<__half>, a)) == cudaSuccess
               ? WINO_OK
               : WINO_ERR_CUDA;
}

}  // namespace wino
