// rope_rows.cuh -- what the kernels that write new rows into a paged cache share: a CTA's rows with their sequences, pages
// and positions, and the cosines and sines of their pairs.
//
// Angles: t / 2 pi modulo 1 is what matters, and x f in 32 bits loses it for far positions (x = 10^6, f = 1: 0.06
// radians).  f / 2 pi is taken to a 64-bit fixed-point fraction of a turn once per CTA and pair; its product with the
// position, modulo 2^64, is then the fraction of the turn to 2^-63 |x|, by integer arithmetic.  The quotient is formed in two
// doubles, since one alone is off by 2^-54 of itself or more, which positions from 2^24 and frequencies above 1 make visible.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_batch.cuh"

namespace wino {

constexpr int kRopeThreads = 256;
constexpr int kMaxRowsPerCta = 32;  // of any kernel
constexpr int kFewRowsPerCta = 8;   // of those that go by rope_rows_per_cta
constexpr int kMaxPairs = 64;  // head_dim / 2
constexpr int kMaxAxes = 4;

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

// The fraction of a turn per position, in units of 2^-64, off by one at most for |radians| < 2^42: the product with 1 / (2 pi) as a
// sum of two doubles, hi + lo, its remainder by fma.
__device__ __forceinline__ uint64_t turn_fraction(double radians)
{
    constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;  // 1 / (2 pi) = kHigh + kLow to 2^-110
    const double hi = radians * kHigh;
    const double lo = fma(radians, kLow, fma(radians, kHigh, -hi));
    const int64_t turns = __double2ll_rn((hi - rint(hi)) * 18446744073709551616.0);  // the difference is exact
    return (uint64_t)turns + (uint64_t)__double2ll_rn(lo * 18446744073709551616.0);
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    return (uint32_t)from_f<T>(lo) | (uint32_t)from_f<T>(hi) << 16;
}

// a' and b' of one pair.  The products' rounding is written out, so that all kernels agree to the bit; kOther: b' with the other of
// its products rounded, as the pair by pair rotation of bf16 has it.
template <bool kOther = false>
__device__ __forceinline__ float2 turn(float a, float b, float2 c)
{
    return make_float2(fmaf(a, c.x, -(b * c.y)), kOther ? fmaf(a, c.y, b * c.x) : fmaf(b, c.x, a * c.y));
}

// What a CTA knows of its rows, kRows at most, of which kPairs pairs may turn (0: none does).
template <int kAxes, int kRows = kMaxRowsPerCta, int kPairs = kMaxPairs>
struct Rows {
    static constexpr int kMost = kRows, kOfAxes = kAxes;
    alignas(16) float2 cs[kRows][kPairs ? kPairs : 1];
    uint64_t turns[kPairs ? kPairs : 1];
    SeqRows q[kRows];
    int32_t seq[kRows];   // -1: a row of no sequence
    int32_t page[kRows];  // -1: not stored
    int32_t in_page[kRows], pos[kRows][kAxes];
    uint8_t axis[kAxes > 1 ? kPairs : 1];
};

// By all kRopeThreads threads, as are the next two: the rows' sequences, and the pairs' turns.  axes: with kAxes > 1 only.
// Returns whether this thread has seen nothing wrong.
template <typename R>
__device__ __forceinline__ bool find_sequences(const wino_kv_batch &b, const wino_rope &rope, const wino_rope_axes *axes,
                                               R &sh, int32_t row0, int32_t n_rows)
{
    constexpr int kAxes = R::kOfAxes;
    const int tid = (int)threadIdx.x, n_pairs = rope.rot_dim >> 1;
    if (tid < R::kMost)
        sh.seq[tid] = -1;
    __syncthreads();
    bool ok = true;
    for (int32_t s = tid; s < b.n_seq; s += kRopeThreads) {
        const SeqRows q = load_seq(b, s);
        ok = ok && q.ok;
        const int32_t r1 = min(n_rows, q.start + q.n - row0);
        if (q.n > 0)
            for (int32_t r = max(0, q.start - row0); r < r1; ++r) {
                sh.seq[r] = s;
                sh.q[r] = q;
            }
    }
    for (int j = tid; j < n_pairs; j += kRopeThreads)
        sh.turns[j] = turn_fraction(rope.freq[j]);
    if constexpr (kAxes > 1) {
        for (int j = tid; j < n_pairs; j += kRopeThreads) {
            const uint8_t x = axes->axis[j];
            ok = ok && x < axes->n_axes;
            sh.axis[j] = x < axes->n_axes ? x : 0;
        }
    }
    __syncthreads();
    return ok;
}

// Then the rows' pages (paged: these are wanted), positions, cosines and sines.  ok: what find_sequences returned; put(row of cs, j,
// c, s): stores pair j's.
template <typename R, typename Put>
__device__ __forceinline__ void find_pages(const wino_kv_batch &b, const wino_rope &rope, const wino_rope_axes *axes, bool paged,
                                           StatusWords *status, R &sh, int32_t row0, int32_t n_rows, bool ok, Put put)
{
    constexpr int kAxes = R::kOfAxes;
    const int tid = (int)threadIdx.x, n_pairs = rope.rot_dim >> 1;
    if (tid < n_rows && sh.seq[tid] >= 0) {
        const SeqRows q = sh.q[tid];
        const int32_t i = row0 + tid - q.start, slot = row_slot(b, q, i), cap = b.table_width * b.page_size;
        int32_t page = -1;
        if (paged && slot >= 0) {
            if (slot < cap)
                page = load_page(b, sh.seq[tid], slot / b.page_size, ok);
            else
                ok = false;
        }
        sh.page[tid] = page;
        sh.in_page[tid] = page >= 0 ? slot % b.page_size : 0;
        if constexpr (kAxes > 1) {
#pragma unroll
            for (int x = 0; x < kAxes; ++x)
                sh.pos[tid][x] = x < axes->n_axes ? axes->positions[x * axes->axis_stride + row0 + tid] : 0;
        } else {
            sh.pos[tid][0] = rope.positions ? rope.positions[row0 + tid]
                                            : q.base + (b.mask == WINO_MASK_SHADOW && i >= (q.n >> 1) ? i - (q.n >> 1) : i);
        }
    }
    if (!ok)
        atomicExch(&status->current, (int32_t)WINO_ERR_ARG);
    __syncthreads();
    for (int x = tid; x < n_rows * n_pairs; x += kRopeThreads) {
        const int r = x / n_pairs, j = x - r * n_pairs;
        if (sh.seq[r] < 0)
            continue;
        const uint64_t t = sh.turns[j] * (uint64_t)(int64_t)sh.pos[r][kAxes > 1 ? sh.axis[j] : 0];
        float sn, cn;
        sincospif((float)(int32_t)(t >> 32) * (1.f / 2147483648.f), &sn, &cn);  // half-turns in [-1, 1)
        put(sh.cs[r], j, cn * rope.factor, sn * rope.factor);
    }
    __syncthreads();
}

template <typename R>
__device__ __forceinline__ void find_rows(const wino_kv_batch &b, const wino_rope &rope, const wino_rope_axes *axes, bool paged,
                                          StatusWords *status, R &sh, int32_t row0, int32_t n_rows)
{
    const bool ok = find_sequences(b, rope, axes, sh, row0, n_rows);
    find_pages(b, rope, axes, paged, status, sh, row0, n_rows, ok,
               [](float2 *row, int j, float c, float s) { row[j] = make_float2(c, s); });
}

// Several rows per CTA once there are CTAs enough: the look-up of a CTA's rows is shared, and each thread has more heads
// (replayed, 32 + 2 x 32 heads of 128: 1 against 2 rows: 600 rows 7.0 and 7.7 us, 900 10.6 and 9.2; 2 against 4: 900 9.2 and 11.6,
// 1200 9.7 and 11.0, 2048 19.1 and 16.5; 4 against 8: 2048 16.5 and 23.1, 4096 33.6 and 32.0, 9000 73.1 and 71.8; and 20027 rows of
// 32 + 2 x 8 heads 90.5 and 83.6).
inline int32_t rope_rows_per_cta(int32_t n_rows)
{
    return n_rows >= 8192 ? kFewRowsPerCta : (n_rows >= 1024 ? 4 : (n_rows >= 512 ? 2 : 1));
}

}  // namespace wino
