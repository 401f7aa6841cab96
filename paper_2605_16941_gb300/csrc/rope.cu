// rope.cu -- wino_rope_append: the new rows' queries and keys rotated, keys and values written into the cache's pages.
//
// Pair (a, b) of a head at position x, turned by t = x f:  a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t).
// Angles: t / 2 pi modulo 1 is what matters, and x f in 32 bits loses it for far positions (x = 10^6, f = 1: 0.06
// radians).  f / 2 pi is taken to a 64-bit fixed-point fraction of a turn once per CTA and pair; its product with the
// position, modulo 2^64, is then the fraction of the turn to 2^-63 |x|, by integer arithmetic.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_batch.cuh"
#include "ptx.cuh"

namespace wino {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRowsPerCta = 8;
constexpr int kMaxPairs = 64;  // head_dim / 2

struct RopeArgs {
    wino_heads q, q_out, k, v;
    wino_kv_batch b;
    wino_rope rope;
    StatusWords *status;
    int32_t rows_per_cta;
};

template <typename T>
__device__ __forceinline__ float to_f(uint16_t x);
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(uint16_t x)
{
    return __uint_as_float((uint32_t)x << 16);
}
template <>
__device__ __forceinline__ float to_f<__half>(uint16_t x)
{
    return __half2float(__ushort_as_half(x));
}
template <typename T>
__device__ __forceinline__ uint16_t from_f(float x);
template <>
__device__ __forceinline__ uint16_t from_f<__nv_bfloat16>(float x)
{
    return __bfloat16_as_ushort(__float2bfloat16_rn(x));
}
template <>
__device__ __forceinline__ uint16_t from_f<__half>(float x)
{
    return __half_as_ushort(__float2half_rn(x));
}

// The fraction of a turn per position, in units of 2^-64.
__device__ __forceinline__ uint64_t turn_fraction(double radians)
{
    const double x = radians * 0.15915494309189533577;  // 1 / (2 pi)
    return (uint64_t)((x - floor(x)) * 18446744073709551616.0);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const RopeArgs a)
{
    __shared__ float2 cs[kMaxRowsPerCta][kMaxPairs];
    __shared__ int32_t seq[kMaxRowsPerCta];
    __shared__ int32_t slot_page[kMaxRowsPerCta], slot_in[kMaxRowsPerCta], pos[kMaxRowsPerCta];
    __shared__ uint64_t turns[kMaxPairs];
    const wino_kv_batch &b = a.b;
    const int tid = (int)threadIdx.x;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    const int n_pairs = a.rope.rot_dim >> 1;
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    if (tid < kMaxRowsPerCta)
        seq[tid] = -1;
    for (int j = tid; j < n_pairs; j += kThreads)
        turns[j] = turn_fraction(a.rope.freq[j]);
    __syncthreads();
    bool ok = true;
    for (int32_t s = tid; s < b.n_seq; s += kThreads) {
        const SeqRows q = load_seq(b, s);
        ok = ok && q.ok;
        const int32_t r1 = min(n_rows, q.start + q.n - row0);
        if (q.n > 0)
            for (int32_t r = max(0, q.start - row0); r < r1; ++r)
                seq[r] = s;
    }
    __syncthreads();
    if (tid < n_rows && seq[tid] >= 0) {
        const int32_t s = seq[tid];
        const SeqRows q = load_seq(b, s);
        const int32_t i = row0 + tid - q.start, slot = row_slot(b, q, i), cap = b.table_width * b.page_size;
        int32_t page = -1;
        if (a.k.data && slot >= 0) {
            if (slot < cap)
                page = load_page(b, s, slot / b.page_size, ok);
            else
                ok = false;
        }
        slot_page[tid] = page;
        slot_in[tid] = page >= 0 ? slot % b.page_size : 0;
        pos[tid] = a.rope.positions ? a.rope.positions[row0 + tid]
                                    : q.base + (b.mask == WINO_MASK_SHADOW && i >= (q.n >> 1) ? i - (q.n >> 1) : i);
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
    __syncthreads();
    for (int x = tid; x < n_rows * n_pairs; x += kThreads) {
        const int r = x / n_pairs, j = x - r * n_pairs;
        if (seq[r] < 0)
            continue;
        const uint64_t t = turns[j] * (uint64_t)(int64_t)pos[r];
        float sn, cn;
        sincospif((float)(int32_t)(t >> 32) * (1.f / 2147483648.f), &sn, &cn);  // half-turns in [-1, 1)
        cs[r][j] = make_float2(cn * a.rope.factor, sn * a.rope.factor);
    }
    __syncthreads();
    // one (row, head, dim pair or plain dim) per thread and turn
    const int heads = (a.q.data ? b.n_q_heads : 0) + (a.k.data ? 2 * b.n_kv_heads : 0);
    const int D = b.head_dim, nq = a.q.data ? b.n_q_heads : 0;
    const int units = D - n_pairs;  // pairs, then the plain dims
    for (int64_t x = tid; x < (int64_t)n_rows * heads * units; x += kThreads) {
        const int u = (int)(x % units), h = (int)(x / units % heads), r = (int)(x / units / heads);
        if (seq[r] < 0)
            continue;
        const int64_t row = row0 + r;
        const uint16_t *src;
        uint16_t *dst;
        bool rotate = true;
        if (h < nq) {
            src = a.q.data + row * a.q.row_stride + h * a.q.head_stride;
            dst = a.q_out.data + row * a.q_out.row_stride + h * a.q_out.head_stride;
        } else {
            if (slot_page[r] < 0)
                continue;
            const bool is_k = h - nq < b.n_kv_heads;
            const int hk = is_k ? h - nq : h - nq - b.n_kv_heads;
            const wino_heads &w = is_k ? a.k : a.v;
            src = w.data + row * w.row_stride + hk * w.head_stride;
            dst = (is_k ? b.k_cache : b.v_cache) + (int64_t)slot_page[r] * b.page_stride +
                  (int64_t)slot_in[r] * b.slot_stride + hk * b.head_stride;
            rotate = is_k;
        }
        if (u < n_pairs) {
            const int i0 = a.rope.interleaved ? 2 * u : u, i1 = a.rope.interleaved ? 2 * u + 1 : u + n_pairs;
            if (rotate) {
                const float2 c = cs[r][u];
                const float p = to_f<T>(src[i0]), q = to_f<T>(src[i1]);
                dst[i0] = from_f<T>(p * c.x - q * c.y);
                dst[i1] = from_f<T>(q * c.x + p * c.y);
            } else {
                dst[i0] = src[i0];
                dst[i1] = src[i1];
            }
        } else {
            dst[u + n_pairs] = src[u + n_pairs];
        }
    }
}

}  // namespace

cudaError_t launch_rope_append(const wino_heads *q, const wino_heads *q_out, const wino_heads *k, const wino_heads *v,
                               const wino_kv_batch &b, const wino_rope &rope, StatusWords *status, cudaStream_t stream)
{
    RopeArgs a{};
    if (q) {
        a.q = *q;
        a.q_out = *q_out;
    }
    if (k) {
        a.k = *k;
        a.v = *v;
    }
    a.b = b;
    a.rope = rope;
    a.status = status;
    a.rows_per_cta = std::max(1, std::min(kMaxRowsPerCta, b.n_rows / 1024));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((b.n_rows + a.rows_per_cta - 1) / a.rows_per_cta));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return b.dtype == WINO_BF16 ? cudaLaunchKernelEx(&cfg, rope_append_kernel<__nv_bfloat16>, a)
                                : cudaLaunchKernelEx(&cfg, rope_append_kernel<__half>, a);
}

}  // namespace wino
