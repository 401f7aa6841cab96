// rope.cu -- wino_rope_append: the new rows' queries and keys rotated, keys and values written into the cache's pages.
//
// Pair (a, b) of a head at position x, turned by t = x f:  a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t).
// Bound by HBM: every element is read and written once, 16 bytes at a time (8 where head_dim or rot_dim is no multiple of
// 16).  A thread has one row and two such chunks of a head that hold 8 (4) whole pairs, keeps their cosines and sines in
// registers, and walks the heads with the loads of two of them in flight.  Measured (us): 2048 rows of 32 + 2 x 32 heads of
// 128 (100 MB) 21.3 with inputs that change from call to call, 16.6 replayed from a CUDA graph on one input, which the L2 cache
// holds in part; 20027 rows of 32 + 2 x 8 heads, half of each rotated (492 MB), 84 = 5.9 TB/s either way.  Replayed: four heads
// in flight 19.2 and 98, one 18.9 and 96; at most 3 / 5 / 6 CTAs of 256 threads per SM instead of 4: 22.1 / 18.9 / 26.3 and
// 88.8 / 83.2 / 96.4.  Rotations that are no multiple of 8 dims go pair by pair in 2-byte accesses: 20 dims of heads of 80 take 323
// where 40 take 74.  A CTA looks for its rows among all sequences: 16384 sequences of one row 97.
#include <algorithm>

#include "ptx.cuh"
#include "rope_rows.cuh"

namespace wino {
namespace {

constexpr int kThreads = kRopeThreads;
constexpr int kAhead = 2;  // heads of which a thread has loads in flight

struct RopeArgs {
    wino_heads q, q_out, k, v;
    wino_kv_batch b;
    wino_rope rope;
    StatusWords *status;
    int32_t rows_per_cta;
};

// Chunks of kWords 32-bit words; head_dim and rot_dim multiples of two chunks: two chunks of a head per thread and turn, which
// hold whole pairs, or plain dims.
template <int kWords>
struct Chunk;
template <>
struct Chunk<4> {
    using type = uint4;
};
template <>
struct Chunk<2> {
    using type = uint2;
};

template <typename T, int kWords>
__global__ void __launch_bounds__(kThreads, 4) rope_append_kernel(const RopeArgs a)
{
    __shared__ Rows<1, kFewRowsPerCta> sh;
    const wino_kv_batch &b = a.b;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    find_rows(a.b, a.rope, nullptr, a.k.data != nullptr, a.status, sh, row0, n_rows);
    using V = typename Chunk<kWords>::type;
    constexpr int kDims = 4 * kWords;  // of two chunks
    const int items = b.head_dim / kDims, turned = a.rope.rot_dim / kDims;  // of a head
    const int lanes = items * a.rows_per_cta;                         // (row, item) pairs of the CTA
    const int slots = kThreads / lanes;                               // heads at a time
    const int tid = (int)threadIdx.x, r = tid % lanes / items, j = tid % items, h0 = tid / lanes;
    if (h0 >= slots || r >= n_rows || sh.seq[r] < 0)
        return;
    // the item's chunks: halves j and j + turned, or neighbours
    const bool turns = j < turned;
    const int c0 = turns && !a.rope.interleaved ? j : 2 * j;
    const int c1 = turns && !a.rope.interleaved ? j + turned : 2 * j + 1;
    float2 cs[2 * kWords];
#pragma unroll
    for (int k = 0; k < 2 * kWords; ++k)
        cs[k] = turns ? sh.cs[r][2 * kWords * j + k] : make_float2(0.f, 0.f);
    const int64_t row = row0 + r;
    auto walk = [&](const uint16_t *src, int64_t src_stride, uint16_t *dst, int64_t dst_stride, int heads, bool rotate) {
        for (int h = h0; h < heads; h += kAhead * slots) {
            V x[kAhead], y[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (h + u * slots < heads) {
                    const V *p = reinterpret_cast<const V *>(src + (h + u * slots) * src_stride);
                    x[u] = p[c0];
                    y[u] = p[c1];
                }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (h + u * slots < heads) {
                    if (rotate) {
                        uint32_t *const v = &x[u].x, *const w = &y[u].x;
                        if (a.rope.interleaved) {
#pragma unroll
                            for (int k = 0; k < kWords; ++k) {
                                const float2 p = turn(to_f<T>((uint16_t)v[k]), to_f<T>((uint16_t)(v[k] >> 16)), cs[k]);
                                const float2 q = turn(to_f<T>((uint16_t)w[k]), to_f<T>((uint16_t)(w[k] >> 16)), cs[kWords + k]);
                                v[k] = pack2<T>(p.x, p.y);
                                w[k] = pack2<T>(q.x, q.y);
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < kWords; ++k) {
                                const float2 p = turn(to_f<T>((uint16_t)v[k]), to_f<T>((uint16_t)w[k]), cs[2 * k]);
                                const float2 q = turn(to_f<T>((uint16_t)(v[k] >> 16)), to_f<T>((uint16_t)(w[k] >> 16)), cs[2 * k + 1]);
                                v[k] = pack2<T>(p.x, q.x);
                                w[k] = pack2<T>(p.y, q.y);
                            }
                        }
                    }
                    V *const d = reinterpret_cast<V *>(dst + (h + u * slots) * dst_stride);
                    d[c0] = x[u];
                    d[c1] = y[u];
                }
        }
    };
    if (a.q.data)
        walk(a.q.data + row * a.q.row_stride, a.q.head_stride, a.q_out.data + row * a.q_out.row_stride, a.q_out.head_stride,
             b.n_q_heads, turns);
    if (sh.page[r] >= 0) {
        const int64_t at = (int64_t)sh.page[r] * b.page_stride + (int64_t)sh.in_page[r] * b.slot_stride;
        walk(a.k.data + row * a.k.row_stride, a.k.head_stride, b.k_cache + at, b.head_stride, b.n_kv_heads, turns);
        walk(a.v.data + row * a.v.row_stride, a.v.head_stride, b.v_cache + at, b.head_stride, b.n_kv_heads, false);
    }
}

// Any other dims: one pair or plain dim per thread and turn.
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_append_any_kernel(const RopeArgs a)
{
    __shared__ Rows<1, kFewRowsPerCta> sh;
    const wino_kv_batch &b = a.b;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    find_rows(a.b, a.rope, nullptr, a.k.data != nullptr, a.status, sh, row0, n_rows);
    const int n_pairs = a.rope.rot_dim >> 1, nq = a.q.data ? b.n_q_heads : 0;
    const int heads = nq + (a.k.data ? 2 * b.n_kv_heads : 0);
    const int units = b.head_dim - n_pairs;  // pairs, then the plain dims
    for (int64_t x = threadIdx.x; x < (int64_t)n_rows * heads * units; x += kThreads) {
        const int u = (int)(x % units), h = (int)(x / units % heads), r = (int)(x / units / heads);
        if (sh.seq[r] < 0)
            continue;
        const int64_t row = row0 + r;
        const uint16_t *src;
        uint16_t *dst;
        bool rotate = true;
        if (h < nq) {
            src = a.q.data + row * a.q.row_stride + h * a.q.head_stride;
            dst = a.q_out.data + row * a.q_out.row_stride + h * a.q_out.head_stride;
        } else {
            if (sh.page[r] < 0)
                continue;
            const bool is_k = h - nq < b.n_kv_heads;
            const int hk = is_k ? h - nq : h - nq - b.n_kv_heads;
            const wino_heads &w = is_k ? a.k : a.v;
            src = w.data + row * w.row_stride + hk * w.head_stride;
            dst = (is_k ? b.k_cache : b.v_cache) + (int64_t)sh.page[r] * b.page_stride +
                  (int64_t)sh.in_page[r] * b.slot_stride + hk * b.head_stride;
            rotate = is_k;
        }
        if (u < n_pairs) {
            const int i0 = a.rope.interleaved ? 2 * u : u, i1 = a.rope.interleaved ? 2 * u + 1 : u + n_pairs;
            if (rotate) {
                const float2 p = turn<__is_same(T, __nv_bfloat16)>(to_f<T>(src[i0]), to_f<T>(src[i1]), sh.cs[r][u]);
                dst[i0] = from_f<T>(p.x);
                dst[i1] = from_f<T>(p.y);
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
    const bool bf16 = b.dtype == WINO_BF16;
    if (b.head_dim % 16 == 0 && rope.rot_dim % 16 == 0)
        return bf16 ? cudaLaunchKernelEx(&cfg, rope_append_kernel<__nv_bfloat16, 4>, a)
                    : cudaLaunchKernelEx(&cfg, rope_append_kernel<__half, 4>, a);
    if (rope.rot_dim % 8 == 0)  // and so is head_dim
        return bf16 ? cudaLaunchKernelEx(&cfg, rope_append_kernel<__nv_bfloat16, 2>, a)
                    : cudaLaunchKernelEx(&cfg, rope_append_kernel<__half, 2>, a);
    return bf16 ? cudaLaunchKernelEx(&cfg, rope_append_any_kernel<__nv_bfloat16>, a)
                : cudaLaunchKernelEx(&cfg, rope_append_any_kernel<__half>, a);
}

}  // namespace wino
