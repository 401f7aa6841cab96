// attend.cu -- wino_attend: attention of a step's rows over a paged cache.
//
// One warp per (row, query head): 32 slots at a time, a slot per lane for the scores, then the dims spread over the
// lanes for the sum over V, with the running maximum and sum of the softmax in fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_batch.cuh"
#include "ptx.cuh"

namespace wino {
namespace {

constexpr int kWarps = 8;

struct AttendArgs {
    wino_heads q, out;
    wino_kv_batch b;
    float scale_log2;  // scale * log2(e)
    StatusWords *status;
};

__device__ __forceinline__ float to_f(uint16_t x, int dtype)
{
    return dtype == WINO_BF16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}

__device__ __forceinline__ uint16_t from_f(float x, int dtype)
{
    return dtype == WINO_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}

__global__ void __launch_bounds__(kWarps * 32) attend_kernel(const AttendArgs a)
{
    __shared__ int32_t seq;
    __shared__ float qs[kWarps][128];
    const wino_kv_batch &b = a.b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int32_t row = blockIdx.x;
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    if (threadIdx.x == 0)
        seq = -1;
    __syncthreads();
    bool ok = true;
    for (int32_t s = threadIdx.x; s < b.n_seq; s += kWarps * 32) {
        const SeqRows q = load_seq(b, s);
        ok = ok && q.ok;
        if (q.n > 0 && row >= q.start && row < q.start + q.n)
            seq = s;
    }
    __syncthreads();
    if (seq >= 0) {
        const SeqRows q = load_seq(b, seq);
        const RowSees sees = row_sees(b, q, row - q.start);
        for (int h = blockIdx.y * kWarps + warp; h < min(b.n_q_heads, (int)(blockIdx.y + 1) * kWarps); h += kWarps) {
            const int hk = h / (b.n_q_heads / b.n_kv_heads);
            for (int c = lane; c < b.head_dim; c += 32)
                qs[warp][c] = to_f(a.q.data[row * a.q.row_stride + h * a.q.head_stride + c], b.dtype);
            __syncwarp();
            float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
            for (int32_t j0 = 0; j0 < sees.lim; j0 += 32) {
                const int32_t j = j0 + lane;
                int64_t at = -1;
                float x = -INFINITY;
                if (j < sees.lim && j != sees.hole) {
                    const int32_t page = load_page(b, seq, j / b.page_size, ok);
                    if (page >= 0) {
                        at = page * b.page_stride + (j % b.page_size) * b.slot_stride + hk * b.head_stride;
                        float d = 0.f;
                        for (int c = 0; c < b.head_dim; ++c)
                            d = fmaf(qs[warp][c], to_f(b.k_cache[at + c], b.dtype), d);
                        x = d * a.scale_log2;
                    }
                }
                float mx = x;
                for (int i = 16; i; i >>= 1)
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, i));
                const float mn = fmaxf(m, mx);
                if (mn == -INFINITY)
                    continue;
                const float p = ptx::ex2(x - mn), f = ptx::ex2(m - mn);
                m = mn;
                l = l * f + p;
                for (int i = 0; i < 4; ++i)
                    o[i] *= f;
                for (int t = 0; t < 32; ++t) {
                    const int64_t av = __shfl_sync(0xffffffffu, at, t);
                    const float pt = __shfl_sync(0xffffffffu, p, t);
                    if (av >= 0)
                        for (int i = 0; i < 4; ++i)
                            if (lane + 32 * i < b.head_dim)
                                o[i] = fmaf(pt, to_f(b.v_cache[av + lane + 32 * i], b.dtype), o[i]);
                }
            }
            for (int i = 16; i; i >>= 1)
                l += __shfl_xor_sync(0xffffffffu, l, i);
            for (int i = 0; i < 4; ++i)
                if (lane + 32 * i < b.head_dim)
                    a.out.data[row * a.out.row_stride + h * a.out.head_stride + lane + 32 * i] =
                        from_f(l > 0.f ? o[i] / l : 0.f, b.dtype);
        }
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
}

__global__ void publish_kernel(StatusWords *status)
{
    ptx::grid_dep_wait();
    status->last = status->current;
    status->current = WINO_OK;
}

}  // namespace

size_t attend_scratch_bytes(const wino_kv_batch &) { return 0; }

int launch_attend(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b, uint8_t *,
                  StatusWords *status, int, cudaStream_t stream)
{
    AttendArgs a{q, out, b, scale * 1.4426950408889634f, status};
    attend_kernel<<<dim3((unsigned)b.n_rows, (unsigned)((b.n_q_heads + kWarps - 1) / kWarps)), kWarps * 32, 0, stream>>>(a);
    if (cudaGetLastError() != cudaSuccess)
        return WINO_ERR_CUDA;
    publish_kernel<<<1, 1, 0, stream>>>(status);
    return cudaGetLastError() == cudaSuccess ? WINO_OK : WINO_ERR_CUDA;
}

}  // namespace wino
