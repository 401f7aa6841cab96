// attend_few.cu -- wino_attend_scaled for sequences of few rows (single tokens): the codes go from global memory through registers
// to the tensor cores.
//
// out = softmax(scale Q K^T) V as in attend_kernel.cuh.  Up to 8 rows times heads of a kv head are a tile, the 8 columns of
// mma.m16n8k16: S^T = K Q^T and O^T = V^T P^T, with K and V as the A operand.  That is bound by the stream of codes: a token's
// products would fill 8 of the 128 rows that tcgen05 takes, and its operands would have to go through shared memory twice more.
//
// A warp takes 32 slots at a time.  S^T: lane 4 g + t reads 16 codes of slots g and g + 8 at a time; which dims meet in a step of 16
// does not matter as long as Q's do the same, so the four codes of a word are the four values that a step wants from a
// lane.  O^T: lane 4 g + t reads 16 neighbouring dims of four slots, and a row of the product is any dim: two of the lane's dims per step,
// whose codes of two slots are put side by side and converted.  Both ways 64 or 128 neighbouring bytes are read together, and
// nothing passes through shared memory but the 11 warps' results at the end of a part.
//
// Precision: codes are exact in fp16.  Q is brought to fp16 with a power of two per row that leaves its largest value in
// [2^14, 2^15): all bits are kept down to 2^-28 of it.  K's scales multiply the scores in fp32.  V's scales are part of the weights:
// w = 2^(t + e - c) with t the score behind the running maximum m, e the slot's exponent and c the running maximum of t + e; w is
// rounded to fp16 (half a step; 2^-40 of the largest below its normal range), l sums the unrounded 2^t without e, and the result is
// 2^c O / l.  Differences of scores are formed before they are scaled, so that scores may lie anywhere.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attend_kernel.cuh"

namespace wino {
namespace {

using namespace attend;

constexpr int kWorkers = 11, kFewThreads = 32 * (kWorkers + 1);  // and the planning warp: 12 warps have 168 registers a thread
constexpr int kFewRows = 8, kChunk = 32;  // rows of a tile, slots at a time of a warp
constexpr float kWeightTop = 15.f;        // the largest weight is 2^this

struct alignas(16) FewShared {
    Part parts[kParts];
    uint64_t part_full[kParts], part_empty[kParts];
    int32_t abort, last;
    float m[kWorkers][kFewRows], c[kWorkers][kFewRows], l[kWorkers][kFewRows], f[kWorkers][kFewRows];  // f: factors of O
    float joined[3][kFewRows];  // m, c, l of all workers
    alignas(16) float o[kWorkers][kFewRows][128 + 4];
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two codes of the low or high half of a word as fp16.
__device__ __forceinline__ uint32_t half2_of(uint32_t word, bool high)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)(high ? word >> 16 : word)));
    return r;
}

// An 8 x 8 matrix of 16-bit elements across the warp, turned over.
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ void worker_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkers * 32) : "memory"); }

// The barrier with a vote: whether any worker says so.
__device__ __forceinline__ bool worker_any(bool x)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r)
                 : "r"((uint32_t)x), "n"(kWorkers * 32)
                 : "memory");
    return r != 0;
}

__device__ __forceinline__ float max_of_rows(float x)  // over the lanes of one t
{
#pragma unroll
    for (int i = 4; i < 32; i <<= 1)
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, i));
    return x;
}

template <int DP, typename T>
__global__ void __launch_bounds__(kFewThreads, 1) attend_few_kernel(const __grid_constant__ AttendArgs a)
{
    constexpr int kLoadsK = DP / 64;      // 16 codes each, per slot
    constexpr int kSteps = DP / 16;       // of 16 dims: K's words, and O's tiles
    constexpr int kWordsV = DP / 32;      // codes of a slot that a lane has of V: DP / 8 dims
    extern __shared__ __align__(16) uint8_t smem_few[];
    FewShared &sh = *reinterpret_cast<FewShared *>(smem_few);
    const wino_kv_batch &b = a.b;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kParts; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh.part_full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh.part_empty[s]), kWorkers);
        }
        sh.abort = 0;
        ptx::fence_barrier_init();
    }
    __syncthreads();
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();
    bool ok = true;
    if (warp == kWorkers) {
        if (a.wide)
            plan<uint64_t, FewShared, 1>(a, sh, lane);
        else
            plan<uint32_t, FewShared, 1>(a, sh, lane);
    } else {
        const int g = lane >> 2, t4 = lane & 3;
        const float sl2 = a.scale_log2;
        PartReader reader;
        while (true) {
            // Together: a worker that gave up alone would leave the others at their barriers.  Behind it the part before is out of
            // shared memory.
            if (worker_any(!warp_wait(ptx::smem_u32(&sh.part_full[reader.slot()]), reader.parity(), &sh.abort)))
                break;
            const Part part = sh.parts[reader.slot()];
            __syncwarp();
            if (part.flags & kEnd)
                break;
            if (lane == 0)
                ptx::mbar_arrive(ptx::smem_u32(&sh.part_empty[reader.slot()]));
            ++reader.count;

            // ---- Q: row g of the tile is head g % group of the task's position g / group
            uint32_t q[kSteps][2];
            float inv;
            {
                const int pos = g / a.group, i = part.i0 + pos;
                const bool valid = pos < a.positions && i < part.q.n;
                const uint16_t *const src = a.q.data + (int64_t)(part.q.start + i) * a.q.row_stride +
                                            (int64_t)(part.kv_head * a.group + g - pos * a.group) * a.q.head_stride;
                uint2 raw[kSteps];
                float most = 0.f;
                auto value = [](uint32_t bits) {
                    if constexpr (__is_same(T, __nv_bfloat16))
                        return __uint_as_float(bits << 16);
                    else
                        return __half2float(__ushort_as_half((uint16_t)bits));
                };
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int dim = 64 * (s / 4) + 16 * t4 + 4 * (s % 4);
                    raw[s] = make_uint2(0, 0);
                    if (valid && dim < b.head_dim)
                        raw[s] = *reinterpret_cast<const uint2 *>(src + dim);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t w = k ? raw[s].y : raw[s].x;
                        most = fmaxf(most, fmaxf(fabsf(value(w & 0xffffu)), fabsf(value(w >> 16))));
                    }
                }
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                const uint32_t e = max(__float_as_uint(most) >> 23, 15u);
                const float by = __uint_as_float((268u - e) << 23);
                inv = __uint_as_float((e - 14u) << 23);
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t w = k ? raw[s].y : raw[s].x;
                        q[s][k] = pack2<false>(value(w & 0xffffu) * by, value(w >> 16) * by);
                    }
            }
            // ---- rows 2 t4 and 2 t4 + 1, whose scores and results this lane holds
            float inv_row[2], m[2], c[2], l[2];
            int32_t lim[2], hole[2], all = 1 << 30;  // all: slots that every row of the tile sees, holes apart
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int row = 2 * t4 + k, pos = row / a.group, i = part.i0 + pos;
                inv_row[k] = __shfl_sync(0xffffffffu, inv, row * 4);
                m[k] = c[k] = -INFINITY;
                l[k] = 0.f;
                lim[k] = 0;
                hole[k] = -1;
                if (pos < a.positions && i < part.q.n) {
                    const RowSees sees = row_sees(b, part.q, i);
                    lim[k] = sees.lim;
                    hole[k] = sees.hole;
                    all = min(all, hole[k] >= 0 ? min(lim[k], hole[k]) : lim[k]);
                }
            }
            all = __reduce_min_sync(0xffffffffu, all);
            float o[kSteps][4];
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[s][k] = 0.f;

            // ---- the part's slots, 32 at a time; pages a turn ahead of the codes, codes a turn ahead of their use
            const int32_t end = min(part.kv_end, (part.j0 + part.n) * kTileN);
            const int32_t *const table = b.page_table + (int64_t)part.seq * b.table_width;
            int32_t at = part.j0 * kTileN + warp * kChunk;
            auto page_of = [&](int32_t slot) { return slot < end ? table[page_entry(a, slot)] : -1; };
            int32_t pages[2] = {page_of(at), page_of(at + 16)};
            uint4 k_codes[2][2][kLoadsK];         // [16 slots][slot g or g + 8]
            uint32_t v_codes[2][4][kWordsV];      // [16 slots][slots 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9]
            uint32_t k_scale[2][2], v_scale[2][2];  // of slots g and g + 8
            // The base of 16 slots that lie in one page; null where nothing is read.
            auto base_of = [&](int32_t slot, int32_t page, int64_t &codes, int64_t &scales) {
                const int32_t in_page = slot - page_entry(a, slot) * b.page_size;
                codes = (int64_t)page * b.page_stride + (int64_t)in_page * b.slot_stride + (int64_t)part.kv_head * b.head_stride;
                scales = scale_at(b, page, in_page, part.kv_head);
            };
            auto fetch = [&](int32_t slot, auto is_v) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int32_t first = slot + 16 * x, left = end - first, page = pages[x];
                    const bool there = left > 0 && (uint32_t)page < (uint32_t)b.n_pages;
                    int64_t codes = 0, scales = 0;
                    if (there)
                        base_of(first, page, codes, scales);
                    const uint8_t *const from = reinterpret_cast<const uint8_t *>(decltype(is_v)::value ? b.v_cache : b.k_cache) + codes;
                    const uint8_t *const scale = (decltype(is_v)::value ? a.scales.v_scale : a.scales.k_scale) + scales;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        (decltype(is_v)::value ? v_scale : k_scale)[x][k] = there && g + 8 * k < left ? (uint32_t)scale[g + 8 * k] : 0u;
                    if constexpr (decltype(is_v)::value) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int in = 2 * t4 + (k & 1) + 8 * (k >> 1);
                            const bool some = there && in < left && g * (DP / 8) < b.head_dim;
                            const uint8_t *const p = from + (int64_t)in * b.slot_stride + g * (DP / 8);
                            if constexpr (DP == 128) {
                                const uint4 w = some ? ptx::ld_stream(p) : make_uint4(0, 0, 0, 0);
                                v_codes[x][k][0] = w.x;
                                v_codes[x][k][1] = w.y;
                                v_codes[x][k][2] = w.z;
                                v_codes[x][k][3] = w.w;
                            } else {
                                const uint2 w = some ? ptx::ld_stream2(p) : make_uint2(0, 0);
                                v_codes[x][k][0] = w.x;
                                v_codes[x][k][1] = w.y;
                            }
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int n = 0; n < kLoadsK; ++n) {
                                const int dim = 64 * n + 16 * t4;
                                const bool some = there && g + 8 * k < left && dim < b.head_dim;
                                k_codes[x][k][n] = some ? ptx::ld_stream(from + (int64_t)(g + 8 * k) * b.slot_stride + dim)
                                                        : make_uint4(0, 0, 0, 0);
                            }
                    }
                    ok = ok && (left <= 0 || there);
                }
            };
            const std::false_type of_k{};
            const std::true_type of_v{};
            if (at < end) {
                fetch(at, of_k);
                fetch(at, of_v);
            }
            for (; at < end; at += kWorkers * kChunk) {
                const int32_t next = at + kWorkers * kChunk;
                const int32_t next_pages[2] = {page_of(next), page_of(next + 16)};
                float s[2][4];  // scores of slots g (0, 1) and g + 8 (2, 3) with rows 2 t4 and 2 t4 + 1
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        s[x][k] = 0.f;
#pragma unroll
                    for (int n = 0; n < kLoadsK; ++n) {
                        const uint4 lo = k_codes[x][0][n], hi = k_codes[x][1][n];
                        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            mma_f16(s[x], half2_of(wl[w], false), half2_of(wh[w], false), half2_of(wl[w], true), half2_of(wh[w], true),
                                    q[4 * n + w][0], q[4 * n + w][1]);
                    }
                }
                float nan[2][2];  // NaN where a slot's K is held as that
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t e = k_scale[x][k];
                        nan[x][k] = e == kScaleNan ? NAN : 0.f;
                        const float f = e == kScaleNan ? 0.f : __uint_as_float(e << 23);
                        s[x][2 * k] = s[x][2 * k] * f * inv_row[0];
                        s[x][2 * k + 1] = s[x][2 * k + 1] * f * inv_row[1];
                    }
                uint32_t v_exp[2][2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        v_exp[x][k] = v_scale[x][k];
                const int32_t here = at;
                pages[0] = next_pages[0];
                pages[1] = next_pages[1];
                if (next < end)
                    fetch(next, of_k);  // into the registers that the products above have read
                if (here + kChunk > all) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int32_t slot = here + 16 * x + g + 8 * (k >> 1);
                            if (slot >= lim[k & 1] || slot == hole[k & 1])
                                s[x][k] = -INFINITY;
                        }
                }
                float fo[2];
                uint32_t w[2][2];  // weights of slot g and g + 8, rows side by side
                float p[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float mx = fmaxf(m[r], max_of_rows(fmaxf(fmaxf(s[0][r], s[0][2 + r]), fmaxf(s[1][r], s[1][2 + r]))));
                    const float base = mx == -INFINITY ? 0.f : mx;  // nothing seen yet: every t is -inf
                    const float moved = m[r] == -INFINITY ? 0.f : (m[r] - base) * sl2;
                    float top = -INFINITY;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float &t = s[x][2 * k + r];
                            t = (t - base) * sl2;
                            const float e = v_exp[x][k] == kScaleNan ? 0.f : (float)((int)v_exp[x][k] - kScaleBias);
                            p[x][2 * k + r] = t + e;
                            top = fmaxf(top, t + e);
                        }
                    top = max_of_rows(top);
                    const float before = c[r] + moved;  // -inf stays
                    c[r] = fmaxf(before, top);
                    fo[r] = before == -INFINITY ? 0.f : ptx::ex2(before - c[r]);
                    l[r] *= ptx::ex2(moved);
                    m[r] = mx;
                    const float up = c[r] == -INFINITY ? 0.f : kWeightTop - c[r];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float t = s[x][2 * k + r];
                            const bool seen = t != -INFINITY;
                            l[r] += seen ? ptx::ex2(t) + nan[x][k] : 0.f;
                            const float weight = ptx::ex2(p[x][2 * k + r] + up) + nan[x][k] + (v_exp[x][k] == kScaleNan ? NAN : 0.f);
                            p[x][2 * k + r] = seen ? weight : 0.f;
                        }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        w[x][k] = transposed(pack2<false>(p[x][2 * k], p[x][2 * k + 1]));
                if (__any_sync(0xffffffffu, fo[0] != 1.f || fo[1] != 1.f)) {
#pragma unroll
                    for (int i = 0; i < kSteps; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            o[i][k] *= fo[k & 1];
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        // dims 2 i and 2 i + 1 of the lane's: codes of two slots side by side, then the other two's
                        const uint32_t sel = (i & 1) ? 0x7362 : 0x5140;
                        const uint32_t lo = __byte_perm(v_codes[x][0][i / 2], v_codes[x][1][i / 2], sel);
                        const uint32_t hi = __byte_perm(v_codes[x][2][i / 2], v_codes[x][3][i / 2], sel);
                        mma_f16(o[i], half2_of(lo, false), half2_of(lo, true), half2_of(hi, false), half2_of(hi, true), w[x][0], w[x][1]);
                    }
                if (next < end)
                    fetch(next, of_v);
            }

            // ---- the warps' results become the part's
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 4; i < 32; i <<= 1)
                    l[r] += __shfl_xor_sync(0xffffffffu, l[r], i);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = 2 * t4 + r;
                if (g == 0) {
                    sh.m[warp][row] = m[r];
                    sh.c[warp][row] = c[r];
                    sh.l[warp][row] = l[r];
                }
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    *reinterpret_cast<float2 *>(&sh.o[warp][row][g * (DP / 8) + 2 * i]) = make_float2(o[i][r], o[i][2 + r]);
            }
            worker_barrier();
            // Joins `n` results (m, c, l, O): their maxima, the factors of each O, and the sum of l.
            auto factors = [&](int n, auto m_of, auto c_of, auto l_of, auto put, float &big, float &top, float &sum) {
                big = -INFINITY;
                for (int i = 0; i < n; ++i)
                    big = fmaxf(big, m_of(i));
                top = -INFINITY;
                sum = 0.f;
                for (int i = 0; i < n; ++i) {
                    const float mi = m_of(i);
                    if (mi == -INFINITY)
                        continue;
                    const float behind = (mi - big) * sl2;
                    top = fmaxf(top, c_of(i) + behind);
                    sum += l_of(i) * ptx::ex2(behind);
                }
                for (int i = 0; i < n; ++i) {
                    const float mi = m_of(i);
                    put(i, mi == -INFINITY ? 0.f : ptx::ex2(c_of(i) + (mi - big) * sl2 - top));
                }
            };
            const int tid = (int)threadIdx.x;
            float big = -INFINITY, top = -INFINITY, sum = 0.f;
            if (tid < kFewRows) {
                factors(kWorkers, [&](int i) { return sh.m[i][tid]; }, [&](int i) { return sh.c[i][tid]; },
                        [&](int i) { return sh.l[i][tid]; }, [&](int i, float x) { sh.f[i][tid] = x; }, big, top, sum);
                sh.joined[0][tid] = big;
                sh.joined[1][tid] = top;
                sh.joined[2][tid] = sum;
            }
            worker_barrier();
            // A thread has 4 neighbouring dims of a row.
            const int row = tid / (DP / 4), dim = tid % (DP / 4) * 4;
            const bool mine = row < kFewRows;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mine) {
#pragma unroll
                for (int i = 0; i < kWorkers; ++i) {
                    const float f = sh.f[i][row];
                    const float4 z = *reinterpret_cast<const float4 *>(&sh.o[i][row][dim]);
                    if (f != 0.f) {
                        y.x = fmaf(f, z.x, y.x);
                        y.y = fmaf(f, z.y, y.y);
                        y.z = fmaf(f, z.z, y.z);
                        y.w = fmaf(f, z.w, y.w);
                    }
                }
                big = sh.joined[0][row];
                top = sh.joined[1][row];
                sum = sh.joined[2][row];
            }
            bool whole = true;
            if ((part.flags & kWhole) == 0) {
                // The task's parts meet in the workspace; the one that comes last joins them all in their order.
                const int n = part.last - part.first + 1;
                auto place = [&](int cta) { return (int64_t)cta * 2 + (cta == part.first ? 1 : 0); };
                float *const ml = reinterpret_cast<float *>(a.part_ml);
                const int64_t of_ml = 2 * a.quarters * 64, of_o = (int64_t)2 * a.quarters * 32 * a.piece;
                float *const po = reinterpret_cast<float *>(a.part_o);
                if (mine) {
                    const int64_t to = place((int)blockIdx.x);
                    if (dim == 0) {
                        ml[to * of_ml + row] = big;
                        ml[to * of_ml + 8 + row] = top;
                        ml[to * of_ml + 16 + row] = sum;
                    }
                    *reinterpret_cast<float4 *>(&po[to * of_o + row * DP + dim]) = y;
                }
                __threadfence();
                worker_barrier();
                int32_t *const node = a.nodes + (int64_t)part.first * kLevels * 8;
                if (tid == 0) {
                    const int there = atomicAdd(node, 1);
                    sh.last = there == n - 1;
                    if (there == n - 1)
                        *node = 0;  // for the next call
                }
                worker_barrier();
                whole = sh.last != 0;
                if (whole && mine) {
                    __threadfence();
                    auto value = [&](int i, int k) { return __ldcg(&ml[place(part.first + i) * of_ml + 8 * k + row]); };
                    y = make_float4(0.f, 0.f, 0.f, 0.f);
                    factors(n, [&](int i) { return value(i, 0); }, [&](int i) { return value(i, 1); },
                            [&](int i) { return value(i, 2); },
                            [&](int i, float f) {
                                if (f != 0.f) {
                                    const float4 z = __ldcg(reinterpret_cast<const float4 *>(&po[place(part.first + i) * of_o + row * DP + dim]));
                                    y.x = fmaf(f, z.x, y.x);
                                    y.y = fmaf(f, z.y, y.y);
                                    y.z = fmaf(f, z.z, y.z);
                                    y.w = fmaf(f, z.w, y.w);
                                }
                            },
                            big, top, sum);
                }
            }
            if (whole && mine && dim < b.head_dim) {
                const int pos = row / a.group, i = part.i0 + pos;
                if (pos < a.positions && i < part.q.n) {
                    // no slot seen: zeros; NaN stays NaN
                    const float by = sum == 0.f ? 0.f : ptx::ex2(top - kWeightTop) / sum;
                    uint16_t *const dst = a.out.data + (int64_t)(part.q.start + i) * a.out.row_stride +
                                          (int64_t)(part.kv_head * a.group + row - pos * a.group) * a.out.head_stride;
                    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
                    *reinterpret_cast<uint2 *>(dst + dim) =
                        make_uint2(pack2<kBf16>(y.x * by, y.y * by), pack2<kBf16>(y.z * by, y.w * by));
                }
            }
        }
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_DEVICE_TIMEOUT);
    publish(a, kFewThreads);
}

template <int DP, typename T>
int launch_few(const AttendArgs &a, int ctas, cudaStream_t stream)
{
    static std::mutex mu;
    static bool done[64];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64)
        return WINO_ERR_CUDA;
    {
        std::lock_guard<std::mutex> g(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(attend_few_kernel<DP, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)sizeof(FewShared)) != cudaSuccess)
                return WINO_ERR_CUDA;
            done[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = sizeof(FewShared);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_few_kernel<DP, T>, a) == cudaSuccess ? WINO_OK : WINO_ERR_CUDA;
}

}  // namespace

namespace attend {

bool few_rows(const wino_kv_batch &b)
{
    const int32_t group = b.n_q_heads / b.n_kv_heads;
    return group <= kFewRows && b.n_rows <= (int64_t)b.n_seq * (kFewRows / group);
}

int launch_few(AttendArgs a, int ctas, cudaStream_t stream)
{
    const wino_kv_batch &b = a.b;
    a.positions = kFewRows / a.group;
    for (int i = 0; i < 2; ++i) {
        const uint64_t w = (uint64_t)(i + 1) * a.positions;
        a.magic[i] = (uint32_t)(((uint64_t(1) << 32) + w - 1) / w);
    }
    a.min_units = 6;
    a.wide = (double)b.n_seq * (b.n_rows / a.positions + 1) * b.n_kv_heads * ((double)b.table_width * b.page_size / kTileN + 1 + kTaskCost) >=
             2147483648.0;
    const bool bf16 = (b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16;
    if (b.head_dim <= 64)
        return bf16 ? wino::launch_few<64, __nv_bfloat16>(a, ctas, stream) : wino::launch_few<64, __half>(a, ctas, stream);
    return bf16 ? wino::launch_few<128, __nv_bfloat16>(a, ctas, stream) : wino::launch_few<128, __half>(a, ctas, stream);
}

}  // namespace attend
}  // namespace wino
