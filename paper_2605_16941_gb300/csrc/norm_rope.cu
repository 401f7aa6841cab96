// norm_rope.cu -- wino_norm_rope_append: per-head norms of the new rows' queries and keys, their rotation, and keys and values
// into the cache's pages, in the element type or as e4m3 codes.
//
// y = x (offset + w) / sqrt(mean(x^2) + eps) for a head x, then for each pair of its first rot_dim dims
// a' = m (a cos t - b sin t), b' = m (b cos t + a sin t), all in fp32; then one rounding.  Sums of squares beyond 2^100 are
// formed again of x 2^-100, so that no finite x overflows; eps >= 2^-60 covers what underflows.
#include <type_traits>

#include "e4m3.cuh"
#include "ptx.cuh"
#include "rope_rows.cuh"

namespace wino {
namespace {

constexpr int kThreads = kRopeThreads, kWarps = kThreads / 32;

struct NormRopeArgs {
    wino_heads q, q_out, k, v;
    wino_kv_batch b;
    wino_rope rope;
    wino_rope_axes axes;
    wino_head_norm norm;
    wino_kv_scales scales;
    StatusWords *status;
    int32_t rows_per_cta;
};

// The values x[0 .. n) of a head that `lanes` neighbouring lanes hold (others zero) become x / sqrt(mean(x^2) + eps).
template <int kN>
__device__ __forceinline__ void normalise(float (&x)[kN], int lanes, float dim, float eps)
{
    auto squares = [&]() {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kN; ++k)
            s = fmaf(x[k], x[k], s);
        for (int i = lanes >> 1; i; i >>= 1)
            s += __shfl_xor_sync(0xffffffffu, s, i);
        return s;
    };
    float s = squares();
    const bool large = !(s < 0x1p100f);
    if (__any_sync(0xffffffffu, large)) {
        if (large) {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                x[k] *= 0x1p-100f;
        }
        const float again = squares();
        if (large) {
            s = again;
            eps = 0.f;  // times 2^-200
        }
    }
    const float r = rsqrtf(s / dim + eps);
#pragma unroll
    for (int k = 0; k < kN; ++k)
        x[k] *= r;
}

// Any dims: a warp per head, whose lane l has the dims l, l + 32, l + 64 and l + 96.
template <typename T, bool kScaled, int kAxes>
__global__ void __launch_bounds__(kThreads) norm_append_any_kernel(const __grid_constant__ NormRopeArgs a)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    __shared__ Rows<kAxes> sh;
    __shared__ float head[kWarps][128];
    const wino_kv_batch &b = a.b;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, D = b.head_dim;
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    find_rows(b, a.rope, &a.axes, a.k.data != nullptr, a.status, sh, row0, n_rows);
    const int n_pairs = a.rope.rot_dim >> 1, nq = a.q.data ? b.n_q_heads : 0;
    const int heads = nq + (a.k.data ? 2 * b.n_kv_heads : 0);
    for (int u = warp; u < n_rows * heads; u += kWarps) {
        const int r = u / heads, h = u - r * heads;
        if (sh.seq[r] < 0 || (h >= nq && sh.page[r] < 0))
            continue;
        const bool is_q = h < nq, is_v = h >= nq + b.n_kv_heads;
        const int hk = is_q ? h : (is_v ? h - nq - b.n_kv_heads : h - nq);
        const wino_heads &from = is_q ? a.q : (is_v ? a.v : a.k);
        const uint16_t *const src = from.data + (int64_t)(row0 + r) * from.row_stride + hk * from.head_stride;
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = lane + 32 * k < D ? to_f<T>(src[lane + 32 * k]) : 0.f;
        const uint16_t *const weight = is_q ? a.norm.q_weight : a.norm.k_weight;
        if (!is_v && weight) {
            normalise(x, 32, (float)D, a.norm.eps);
            const uint16_t *const w = weight + hk * (is_q ? a.norm.q_head_stride : a.norm.k_head_stride);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (lane + 32 * k < D)
                    x[k] *= a.norm.offset + to_f<T>(w[lane + 32 * k]);
        }
        if (!is_v && n_pairs) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                head[warp][lane + 32 * k] = x[k];
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = lane + 32 * k;
                if (c < 2 * n_pairs) {
                    const bool second = a.rope.interleaved ? (c & 1) != 0 : c >= n_pairs;
                    const int j = a.rope.interleaved ? c >> 1 : (second ? c - n_pairs : c);
                    const int other = a.rope.interleaved ? c ^ 1 : (second ? j : c + n_pairs);
                    const float y = head[warp][other];
                    const float2 p = second ? turn(y, x[k], sh.cs[r][j]) : turn(x[k], y, sh.cs[r][j]);
                    x[k] = second ? p.y : p.x;
                }
            }
            __syncwarp();
        }
        if (is_q || !kScaled) {
            uint16_t *const dst = is_q ? a.q_out.data + (int64_t)(row0 + r) * a.q_out.row_stride + hk * a.q_out.head_stride
                                       : (is_v ? b.v_cache : b.k_cache) + (int64_t)sh.page[r] * b.page_stride +
                                             (int64_t)sh.in_page[r] * b.slot_stride + hk * b.head_stride;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (lane + 32 * k < D)
                    dst[lane + 32 * k] = from_f<T>(x[k]);
        } else {
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                most = max(most, __float_as_uint(x[k]) & 0x7fffffffu);
            most = __reduce_max_sync(0xffffffffu, most);
            const uint32_t s = scale_byte<kBf16>(most);
            const float f = code_factor(s);
            uint8_t *const dst = reinterpret_cast<uint8_t *>(is_v ? b.v_cache : b.k_cache) + (int64_t)sh.page[r] * b.page_stride +
                                 (int64_t)sh.in_page[r] * b.slot_stride + hk * b.head_stride;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (lane + 32 * k < D)
                    dst[lane + 32 * k] = s == kScaleNan ? (uint8_t)0 : (uint8_t)codes2(x[k] * f, 0.f);
            if (lane == 0)
                (is_v ? a.scales.v_scale : a.scales.k_scale)[scale_at(b, sh.page[r], sh.in_page[r], hk)] = (uint8_t)s;
        }
    }
}

}  // namespace

cudaError_t launch_norm_rope_append(const wino_heads *q, const wino_heads *q_out, const wino_heads *k, const wino_heads *v,
                                    const wino_kv_batch &b, const wino_rope &rope, const wino_rope_axes *axes,
                                    const wino_head_norm *norm, const wino_kv_scales *scales, StatusWords *status,
                                    cudaStream_t stream)
{
    NormRopeArgs a{};
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
    if (axes)
        a.axes = *axes;
    if (norm)
        a.norm = *norm;
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
    auto launch = [&](auto kernel) { return cudaLaunchKernelEx(&cfg, kernel, a); };
    auto of_type = [&](auto type, auto scaled) {
        using T = decltype(type);
        constexpr bool kScaled = decltype(scaled)::value;
        return axes ? launch(norm_append_any_kernel<T, kScaled, kMaxAxes>) : launch(norm_append_any_kernel<T, kScaled, 1>);
    };
    if ((b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16)
        return scales ? of_type(__nv_bfloat16(), std::true_type()) : of_type(__nv_bfloat16(), std::false_type());
    return scales ? of_type(__half(), std::true_type()) : of_type(__half(), std::false_type());
}

}  // namespace wino
