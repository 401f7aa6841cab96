// norm_rope.cu -- wino_norm_rope_append: per-head norms of the new rows' queries and keys, their rotation, and keys and values
// into the cache's pages, in the element type or as e4m3 codes.
//
// y = x (offset + w) / sqrt(mean(x^2) + eps) for a head x, then for each pair of its first rot_dim dims
// a' = m (a cos t - b sin t), b' = m (b cos t + a sin t), all in fp32; then one rounding.  Sums of squares beyond 2^100 are
// formed again of x 2^-100, so that no finite x overflows; eps >= 2^-60 covers what underflows.  Subnormal numbers count as
// zeros.
//
// Bound by HBM where there are many rows, by latencies where there are few: every element is read and written once.  Measured
// (us, replayed; floors from 6.7 TB/s): 64 rows of 32 + 2 x 8 heads of 128 4.7 (one chain of loads: lengths, pages, rows); 2048 rows
// of 32 + 2 x 32 heads with three axes (101 MB) 21 (floor 15); 13481 rows of 32 + 2 x 8 heads with weights per head (331 MB) 65 (49);
// 28931 rows into an 8-bit cache (651 MB) 133 (97).  The rest is instructions, some 290 per 16 elements of a lane with the look-up, at 62 % of the
// issue slots.  What counted, as it was measured then: the rotation's two layouts as branches, not as selects of
// registers (2048 rows 56 and 31), shared weights in shared memory (28931 rows, read back, 198 and 220), cosines read where they are
// used instead of held in registers, some of which spilled (2048 rows 21 and 24, 28931 136 and 156).  3 CTAs an SM: with 4
// registers spill (27 instead of 21, 144 instead of 136, as it was with 16 rows of a CTA at most).  Rows of a CTA: the
// least that makes as few full waves of CTAs as there can be, up to 32 (2048 rows: 5 in one wave 20.7, 4 in one and an eighth
// 27.3; 13481 rows: 30 in one wave 64.8, 15 in two 67.2; up to 64 the same).
#include <type_traits>

#include "e4m3.cuh"
#include "ptx.cuh"
#include "rope_rows.cuh"

namespace wino {
namespace {

constexpr int kThreads = kRopeThreads, kWarps = kThreads / 32, kCtas = 3;  // CTAs of an SM

struct NormRopeArgs {
    wino_heads q, q_out, k, v;
    wino_kv_batch b;
    wino_rope rope;
    wino_rope_axes axes;
    wino_head_norm norm;
    wino_kv_scales scales;
    StatusWords *status;
    int32_t rows_per_cta;
    int32_t lanes;  // per head: the smallest power of two that covers it with 16 (kWhole) or 8 dims each
};

// 1 / sqrt(mean(x^2) + eps) of a head whose values `lanes` neighbouring lanes hold (others zero), by all lanes of the warp.  Where
// the squares come too close to fp32's limits they are formed of x 2^-100, and x becomes x 2^-30 and the result 2^30 times as
// large: both and their products with elements of any size are then normal numbers, if the quotient is.
template <int kN>
__device__ __forceinline__ float inverse_rms(float2 (&x)[kN], int lanes, float inv_dim, float eps)
{
    auto squares = [&](float by) {
        float2 p = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const float2 y = by == 1.f ? x[k] : ptx::mul2(x[k], make_float2(by, by));
            p = ptx::fma2(y, y, p);
        }
        float s = p.x + p.y;
        for (int i = lanes >> 1; i; i >>= 1)
            s += __shfl_xor_sync(0xffffffffu, s, i);
        return s;
    };
    float s = squares(1.f), back = 1.f;
    const bool large = !(s < 0x1p100f);
    if (__any_sync(0xffffffffu, large)) {
        const float again = squares(0x1p-100f);
        if (large) {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                x[k] = ptx::mul2(x[k], make_float2(0x1p-30f, 0x1p-30f));
            s = again;
            eps = 0.f;  // times 2^-200
            back = 0x1p-70f;
        }
    }
    // a Newton step: the root's own error, 2^-22, would move a code's border more than the rest of the arithmetic does
    const float x2 = s * inv_dim + eps, r = rsqrtf(x2);
    return (x2 < 0x1p127f ? r * fmaf(-0.5f * x2 * r, r, 1.5f) : r) * back;  // infinite elements leave 0 of the finite ones
}

enum class Kind { kQ, kK, kV };

template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi)
{
    uint32_t r;
    if (__is_same(T, __nv_bfloat16))
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// kWhole (head dims and rotations that are multiples of 16): a thread has two chunks of 8 dims of a head that hold whole pairs.
// Else it has one, whose partners it finds in shared memory where halves turn: 12000 rows of 32 + 2 x 8 heads of 80 dims, 40 of them
// turned (184 MB), 107 us, and 86 as neighbours; of 128 dims, 58 turned, into an 8-bit cache (270 MB), 113.  Whole, 13481 rows of 128
// dims (331 MB) take 64.
// The smallest power of two of lanes that covers a head works on it, so that sums and maxima take shuffles alone.  A unit is
// some neighbouring heads of one kind of one row, so that a warp never branches apart; the CTA's units, row by row, are cut into
// a run per warp, with the next unit's loads ahead, the first one's ahead of the look-up of pages and of the cosines.
// kPlain: no norms, no axes, no codes; the results are wino_rope_append's, bit for bit.
template <typename T, bool kScaled, int kAxes, bool kWhole, bool kPlain = false>
__global__ void __launch_bounds__(kThreads, kCtas) norm_append_kernel(const __grid_constant__ NormRopeArgs a)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    static_assert(!kPlain || (!kScaled && kAxes == 1 && !kWhole), "the others are wino_rope_append's own");
    constexpr int kPairs = kWhole ? 8 : 4;  // of neighbours, that a thread has
    __shared__ Rows<kAxes> sh;
    __shared__ float beside[kWhole ? 1 : kWarps][8][32];  // not kWhole: dims 8 j + e of a warp's heads, by e and lane
    const wino_kv_batch &b = a.b;
    const int32_t row0 = (int32_t)blockIdx.x * a.rows_per_cta;
    const int32_t n_rows = min(a.rows_per_cta, b.n_rows - row0);
    __shared__ __align__(16) float shared_weight[2][128];  // offset + weight where all heads share it; zeros behind the last dim
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    {
        const int k = (int)threadIdx.x >> 7, c = (int)threadIdx.x & 127;
        const uint16_t *const w = k ? a.norm.k_weight : a.norm.q_weight;
        shared_weight[k][c] = w && c < b.head_dim ? a.norm.offset + to_f<T>(w[c]) : 0.f;
    }
    const bool ok = find_sequences(b, a.rope, &a.axes, sh, row0, n_rows);
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int n_pairs = a.rope.rot_dim >> 1, turned = a.rope.rot_dim / 16, lanes = a.lanes, j = lane & (lanes - 1), of_unit = 32 / lanes, sub = lane / lanes;
    const bool live = j < b.head_dim / (2 * kPairs), turns = kWhole ? j < turned : n_pairs > 0;
    // the item's chunks: halves j and j + turned, or neighbours
    const int c0 = !kWhole || (turns && !a.rope.interleaved) ? j : 2 * j, c1 = turns && !a.rope.interleaved ? j + turned : 2 * j + 1;
    const float inv_dim = 1.f / (float)b.head_dim;
    auto unpack = [&](const uint4 &v, float2 *to) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            to[k] = make_float2(to_f<T>((uint16_t)w[k]), to_f<T>((uint16_t)(w[k] >> 16)));
    };
    const int nq = a.q.data ? b.n_q_heads : 0, nk = a.k.data ? b.n_kv_heads : 0;
    const int q_units = (nq + of_unit - 1) / of_unit, k_units = (nk + of_unit - 1) / of_unit, units = q_units + 2 * k_units;
    auto fetch = [&](int r, int u, uint4 &x, uint4 &y) {
        auto load = [&](const wino_heads &from, int first, int heads) {
            const int head = first * of_unit + sub;
            if (live && head < heads) {
                const uint4 *const p = reinterpret_cast<const uint4 *>(from.data + (row0 + r) * from.row_stride + head * from.head_stride);
                x = p[c0];
                if (kWhole)
                    y = p[c1];
            }
        };
        x = y = make_uint4(0, 0, 0, 0);
        if (sh.seq[r] < 0)
            return;
        if (u < q_units)
            load(a.q, u, nq);
        else if (u < q_units + k_units)
            load(a.k, u - q_units, nk);
        else
            load(a.v, u - q_units - k_units, nk);
    };
    int i = warp * (n_rows * units) / kWarps;
    const int end = (warp + 1) * (n_rows * units) / kWarps;
    int r = i / units, u = i - r * units;
    uint4 nx, ny;
    if (i < end)
        fetch(r, u, nx, ny);
    find_pages(b, a.rope, &a.axes, a.k.data != nullptr, a.status, sh, row0, n_rows, ok,
               [](float2 *row, int p, float c, float s) {
                   if (!kWhole) {
                       row[(p & 7) << 3 | p >> 3] = make_float2(c, s);  // neighbouring lanes' side by side
                       return;
                   }
                   // two of a lane's 8 pairs, cosines and then sines, of all lanes; then the next two
                   float *const two = reinterpret_cast<float *>(row + ((p & 6) << 3 | (p >> 3) << 1)) + (p & 1);
                   two[0] = c;
                   two[2] = s;
               });
    while (i < end) {
        const int64_t row = row0 + r, slot = (int64_t)sh.page[r] * b.page_stride + (int64_t)sh.in_page[r] * b.slot_stride;
        const bool used = sh.seq[r] >= 0, stored = used && sh.page[r] >= 0;
        auto unit = [&](auto kind, int head, int heads, uint4 x, uint4 y) {
            constexpr bool kQ = decltype(kind)::value == Kind::kQ, kV = decltype(kind)::value == Kind::kV;
            const bool mine = live && head < heads;
            float2 z[kPairs];  // the first chunk's pairs of neighbours, then the second's
            unpack(x, z);
            if constexpr (kWhole)
                unpack(y, z + 4);
            const uint16_t *const weight = kQ ? a.norm.q_weight : a.norm.k_weight;
            if (!kPlain && !kV && weight) {
                const float by = inverse_rms(z, lanes, inv_dim, a.norm.eps);
                const int64_t stride = kQ ? a.norm.q_head_stride : a.norm.k_head_stride;
                float2 w[kPairs];
                if (stride == 0) {
                    const float4 *const f = reinterpret_cast<const float4 *>(shared_weight[kQ ? 0 : 1]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float4 p = f[2 * c0 + k];
                        w[2 * k] = make_float2(p.x, p.y);
                        w[2 * k + 1] = make_float2(p.z, p.w);
                        if constexpr (kWhole) {
                            const float4 q = f[2 * c1 + k];
                            w[4 + 2 * k] = make_float2(q.x, q.y);
                            w[4 + 2 * k + 1] = make_float2(q.z, q.w);
                        }
                    }
                } else {
                    const uint4 *const p = reinterpret_cast<const uint4 *>(weight + min(head, heads - 1) * stride);
                    unpack(p[live ? c0 : 0], w);
                    if constexpr (kWhole)
                        unpack(p[live ? c1 : 0], w + 4);
#pragma unroll
                    for (int k = 0; k < kPairs; ++k)
                        w[k] = ptx::add2(w[k], make_float2(a.norm.offset, a.norm.offset));
                }
#pragma unroll
                for (int k = 0; k < kPairs; ++k)
                    z[k] = ptx::mul2(ptx::mul2(z[k], make_float2(by, by)), w[k]);
            }
            if constexpr (kWhole) {
                if (!kV && turns) {
                    float2 c[4], s[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4 p = reinterpret_cast<const float4 *>(sh.cs[r])[8 * k + j];
                        c[k] = make_float2(p.x, p.y);
                        s[k] = make_float2(p.z, p.w);
                    }
                    if (a.rope.interleaved) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            z[2 * k] = turn(z[2 * k].x, z[2 * k].y, make_float2(c[k].x, s[k].x));
                            z[2 * k + 1] = turn(z[2 * k + 1].x, z[2 * k + 1].y, make_float2(c[k].y, s[k].y));
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {  // as turn, two pairs at a time
                            const float2 p = z[k], q = z[4 + k];
                            z[k] = ptx::fma2(p, c[k], ptx::mul2(make_float2(-q.x, -q.y), s[k]));
                            z[4 + k] = ptx::fma2(q, c[k], ptx::mul2(p, s[k]));
                        }
                    }
                }
            } else if (!kV && turns) {
                const float2 *const cs = sh.cs[r];
                if (a.rope.interleaved) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int p = 4 * j + k;
                        if (p < n_pairs)
                            z[k] = turn<kPlain && kBf16>(z[k].x, z[k].y, cs[(p & 7) << 3 | p >> 3]);
                    }
                } else {
                    float(&mine_beside)[8][32] = beside[warp];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        mine_beside[2 * k][lane] = z[k].x;
                        mine_beside[2 * k + 1][lane] = z[k].y;
                    }
                    __syncwarp();
                    auto turned_dim = [&](int e, float x) {  // as turn
                        const int i = 8 * j + e;
                        const bool second = i >= n_pairs;
                        const int p = second ? i - n_pairs : i, other = second ? p : i + n_pairs;
                        if (p >= n_pairs)
                            return x;
                        const float2 c = cs[(p & 7) << 3 | p >> 3];
                        const float y = mine_beside[other & 7][lane - j + (other >> 3)];
                        if (kPlain && kBf16 && second)
                            return fmaf(y, c.y, x * c.x);
                        return fmaf(x, c.x, y * (second ? c.y : -c.y));
                    };
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        z[k] = make_float2(turned_dim(2 * k, z[k].x), turned_dim(2 * k + 1, z[k].y));
                    __syncwarp();
                }
            }
            if (kQ || !kScaled) {
                uint16_t *const dst = kQ ? a.q_out.data + row * a.q_out.row_stride + head * a.q_out.head_stride
                                         : (kV ? b.v_cache : b.k_cache) + slot + head * b.head_stride;
                auto pack = [&](const float2 *v) {
                    return make_uint4(pack_pair<T>(v[0].x, v[0].y), pack_pair<T>(v[1].x, v[1].y), pack_pair<T>(v[2].x, v[2].y),
                                      pack_pair<T>(v[3].x, v[3].y));
                };
                if constexpr (!kV) {  // V is stored as it came, NaNs and all
                    const uint4 as_was = x;
                    x = pack(z);
                    if constexpr (kWhole)
                        y = pack(z + 4);
                    if (kPlain) {  // and so are the dims that do not turn
                        const int turned_dims = a.rope.rot_dim - 8 * j;  // of the chunk
                        x = make_uint4(turned_dims > 0 ? x.x : as_was.x, turned_dims > 2 ? x.y : as_was.y,
                                       turned_dims > 4 ? x.z : as_was.z, turned_dims > 6 ? x.w : as_was.w);
                    }
                }
                if (mine) {
                    reinterpret_cast<uint4 *>(dst)[c0] = x;
                    if constexpr (kWhole)
                        reinterpret_cast<uint4 *>(dst)[c1] = y;
                }
            } else {
                uint32_t most = 0;
#pragma unroll
                for (int k = 0; k < kPairs; ++k)
                    most = max(most, max(__float_as_uint(z[k].x) & 0x7fffffffu, __float_as_uint(z[k].y) & 0x7fffffffu));
                for (int i = lanes >> 1; i; i >>= 1)
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, i));
                const uint32_t s = scale_byte<kBf16>(most);
                const float f = code_factor(s);
                auto codes = [&](const float2 *v) {
                    if (s == kScaleNan)
                        return make_uint2(0, 0);
                    return make_uint2(codes2(v[0].x * f, v[0].y * f) | codes2(v[1].x * f, v[1].y * f) << 16,
                                      codes2(v[2].x * f, v[2].y * f) | codes2(v[3].x * f, v[3].y * f) << 16);
                };
                if (mine) {
                    uint2 *const dst = reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(kV ? b.v_cache : b.k_cache) + slot +
                                                                 head * b.head_stride);
                    dst[c0] = codes(z);
                    if constexpr (kWhole)
                        dst[c1] = codes(z + 4);
                    if (j == 0)
                        (kV ? a.scales.v_scale : a.scales.k_scale)[scale_at(b, sh.page[r], sh.in_page[r], head)] = (uint8_t)s;
                }
            }
        };
        const int last = min(units, u + end - i);  // of this row
        for (; u < last; ++u, ++i) {
            const uint4 x = nx, y = ny;
            if (i + 1 < end)
                fetch(u + 1 < units ? r : r + 1, u + 1 < units ? u + 1 : 0, nx, ny);
            if (u < q_units) {
                if (used)
                    unit(std::integral_constant<Kind, Kind::kQ>(), u * of_unit + sub, nq, x, y);
            } else if (stored) {
                if (u < q_units + k_units)
                    unit(std::integral_constant<Kind, Kind::kK>(), (u - q_units) * of_unit + sub, nk, x, y);
                else
                    unit(std::integral_constant<Kind, Kind::kV>(), (u - q_units - k_units) * of_unit + sub, nk, x, y);
            }
        }
        u = 0;
        ++r;
    }
}

}  // namespace

cudaError_t launch_norm_rope_append(const wino_heads *q, const wino_heads *q_out, const wino_heads *k, const wino_heads *v,
                                    const wino_kv_batch &b, const wino_rope &rope, const wino_rope_axes *axes,
                                    const wino_head_norm *norm, const wino_kv_scales *scales, StatusWords *status,
                                    int sm_count, cudaStream_t stream)
{
    const bool plain = !axes && !scales && (!norm || (!norm->q_weight && !norm->k_weight));
    if (plain && rope.rot_dim % 8 == 0)  // 2048 rows of 32 + 2 x 32 heads 16.0 us, by the kernel here 19.0; of 80 dims, 40 turned, 44 and 108
        return launch_rope_append(q, q_out, k, v, b, rope, status, stream);
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
    // as few waves as kMaxRowsPerCta allows, and all of them full
    const int64_t at_once = (int64_t)sm_count * kCtas;
    a.rows_per_cta = (int32_t)((b.n_rows + at_once - 1) / at_once);
    if (a.rows_per_cta > kMaxRowsPerCta) {
        const int64_t waves = (b.n_rows + at_once * kMaxRowsPerCta - 1) / (at_once * kMaxRowsPerCta);
        a.rows_per_cta = (int32_t)((b.n_rows + at_once * waves - 1) / (at_once * waves));
    }
    const bool whole = b.head_dim % 16 == 0 && rope.rot_dim % 16 == 0;
    a.lanes = 1;
    while (a.lanes < b.head_dim / (whole ? 16 : 8))
        a.lanes *= 2;
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
        if constexpr (!kScaled)
            if (plain)  // pair by pair there: 12000 rows of 80 dims, 20 turned, 211
                return launch(norm_append_kernel<T, false, 1, false, true>);
        if (whole)
            return axes ? launch(norm_append_kernel<T, kScaled, kMaxAxes, true>) : launch(norm_append_kernel<T, kScaled, 1, true>);
        return axes ? launch(norm_append_kernel<T, kScaled, kMaxAxes, false>) : launch(norm_append_kernel<T, kScaled, 1, false>);
    };
    if ((b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16)
        return scales ? of_type(__nv_bfloat16(), std::true_type()) : of_type(__nv_bfloat16(), std::false_type());
    return scales ? of_type(__half(), std::true_type()) : of_type(__half(), std::false_type());
}

}  // namespace wino
