// attend_few.cu -- wino_attend_scaled for sequences of few rows (single tokens).
//
// out = softmax(scale Q K^T) V as in attend_kernel.cuh, whose planning warp cuts the work here too.  Up to 8 rows times heads of
// a kv head, or half of its heads, are a tile, the 8 columns of mma.m16n8k16: S^T = K Q^T and O^T = V^T P^T, with K and V as the A operand.  The stream of
// codes bounds this: a token's products would fill a few of the 128 rows that tcgen05 takes, and its operands would have to go
// through shared memory as values of the element type (attend_kernel.cuh, 64 tokens: 330 us).
//
// A warp takes 32 slots at a time, whose codes copies bring to its own ring in shared memory, swizzled so that no two of the 8 lanes
// that read at once meet in a bank.  S^T: lane 4 g + t reads 32 codes of slots g and g + 8; which dims meet in a step of 16 does
// not matter as long as Q's do the same, so the four codes of a word are the four values that a step wants from a lane.  O^T: lane
// 4 g + t reads 16 neighbouring dims of four slots, and a row of the product may be any dim: two of the lane's dims per
// step, whose codes of two slots are put side by side and converted.  Weights turn from S^T's layout to O^T's by movmatrix.  At the
// end of a part the 15 warps' results meet in shared memory, and a task's parts in the workspace, where the last to come
// joins them in their order.
//
// Precision: codes are exact in fp16.  Q is brought to fp16 with a power of two per row that leaves its largest value in
// [2^14, 2^15): all bits are kept down to 2^-28 of it.  K's scales multiply the scores in fp32.  V's scales are part of the weights
// (kAlike, below), which are rounded to fp16 (half a step; steps of 2^-33 of the largest below its normal range), l sums the
// unrounded 2^t, and the result is 2^c O / l.  Differences of scores are formed before they are scaled, so that scores may
// lie anywhere.
//
// Measured (us, replayed; floors from 6.7 TB/s): 64 tokens over 500 to 32767 slots, 32 heads over 8 kv heads of 128 (821 MB)
// 154 (floor 122; 143 with pages of 64 slots instead of 16); 64 over 16383 slots each 334 (321); one over 262144 slots (541 MB) 97 (80);
// one over 300 slots 9.1.  In the middle of a part a warp needs 4200 clocks for 32 slots, 29 bytes a clock and SM, with 23 at the
// floor; a part's start and end cost as much as 8 slot tiles, by which the work is cut: with 3 as for
// attend_kernel.cuh 166, with 11 158.  The next part's copies ahead of the join, or the planning warp joining in the
// background, gain nothing that the cut does not, and cost short calls 0.3 us; two CTAs of 7 warps an SM 109 for the one long
// token.  Codes read by the lanes themselves, to registers or by cp.async, 205 to 223 and 137 to 143: such reads ran at 13 bytes
// a clock and SM, whatever was in flight.  11 warps of 168 registers instead of 15 of 128: 210 and 140 against 223 and 143 with
// cp.async.  With 128 dims 32 bytes of registers spill.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attend_kernel.cuh"

namespace wino {
namespace {

using namespace attend;

constexpr int kWorkers = 15, kFewThreads = 32 * (kWorkers + 1);  // and the planning warp: 16 warps have 128 registers a thread
constexpr int kFewRows = 8, kChunk = 32;  // rows of a tile, slots at a time of a warp
constexpr float kWeightTop = 15.f;        // the largest weight is 2^this
constexpr int kAlike = 6;                 // V's exponents within this of one another: see below
constexpr int kUnits = 3;                 // of a worker's ring: the codes of 32 slots' K, or V
constexpr uint32_t kUnitBytes = kChunk * 128;
constexpr uint32_t kWorkerBytes = kUnits * kUnitBytes, kRingBytes = kWorkers * kWorkerBytes;
constexpr int kRowFloats = 128 + 4;       // of O in shared memory
static_assert(kFewRows * kRowFloats * sizeof(float) <= kWorkerBytes, "O takes the ring's place at the end of a part");
static_assert(kMaxCtas * 4 * kFewRows * sizeof(float) <= kRingBytes, "and then the parts' m, c, l and factors");

struct alignas(16) FewShared {
    Part parts[kParts];
    uint64_t part_full[kParts], part_empty[kParts];
    uint64_t full[kWorkers][kUnits];
    int32_t abort, last;
    float m[kWorkers][kFewRows], c[kWorkers][kFewRows], l[kWorkers][kFewRows], f[kWorkers][kFewRows];  // f: factors of O
    float joined[kFewRows][3];  // m, c and l of a row, of all workers and then of all parts
};
constexpr uint32_t kFewSmem = kRingBytes + sizeof(FewShared);
static_assert(kFewSmem <= kSmemLimit, "shared memory");

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Four codes of a word as pairs of fp16.
__device__ __forceinline__ void halves_of(uint32_t word, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(word));
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
__global__ void __launch_bounds__(kFewThreads, 1)
    attend_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ AttendArgs a)
{
    constexpr int kLoadsK = DP / 64;      // chunks of 16 codes that a lane has of a slot's K
    constexpr int kSteps = DP / 16;       // of 16 dims: K's words, and O's tiles
    constexpr int kWordsV = DP / 32;      // words of a slot that a lane has of V: DP / 8 dims
    extern __shared__ __align__(1024) uint8_t smem_few[];  // swizzle atoms
    FewShared &sh = *reinterpret_cast<FewShared *>(smem_few + kRingBytes);
    const wino_kv_batch &b = a.b;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kParts; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh.part_full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh.part_empty[s]), kWorkers);
        }
        for (int w = 0; w < kWorkers; ++w)
            for (int u = 0; u < kUnits; ++u)
                ptx::mbar_init(ptx::smem_u32(&sh.full[w][u]), 1);
        sh.abort = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kWorkers && lane == 0) {
        ptx::prefetch_tensormap(&tmK);
        ptx::prefetch_tensormap(&tmV);
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
        uint32_t issued = 0, used = 0;  // units of the ring so far
        bool good = true;
        uint8_t *const ring = smem_few + warp * kWorkerBytes;
        while (true) {
            // Together: a worker that gave up alone would leave the others at their barriers.  Behind it the part before is out of
            // shared memory.
            ptx::fence_proxy_async();  // O's stores to the ring, before the next copies into it
            good = good && warp_wait(ptx::smem_u32(&sh.part_full[reader.slot()]), reader.parity(), &sh.abort);
            if (worker_any(!good))
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
                    const int dim = kLoadsK * 16 * t4 + 4 * s;  // the lane's codes in their order
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
            int e_most = -1000, e_least = 1000;  // of the exponents of V so far
            float o[kSteps][4];
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[s][k] = 0.f;

            // ---- the part's slots, 32 at a time; pages and scales a turn ahead of the codes, codes a turn ahead of their use
            const int32_t end = min(part.kv_end, (part.j0 + part.n) * kTileN);
            const int32_t *const table = b.page_table + (int64_t)part.seq * b.table_width;
            const int32_t kv_head = part.kv_head >> (a.split - 1);
            int32_t at = part.j0 * kTileN + warp * kChunk;
            constexpr int32_t kStep = kWorkers * kChunk;
            // of a slot behind the last one: the last one's, which nothing reads
            auto page_of = [&](int32_t slot) { return table[page_entry(a, min(slot, end - 1))]; };
            int32_t pages[2] = {-1, -1};
            // The 32 slots from `slot` on, whose pages are at hand: a lane's box (its page, or n_pages for zeros), and its slot's scales.
            int32_t box_page = 0, box_slot = 0, box_bytes = 0;
            auto locate = [&](int32_t slot, uint32_t (&scales)[2]) {
                const int32_t left = end - slot, boxes = min(kChunk / a.box_rows, (left + a.box_rows - 1) / a.box_rows);
                const int x = lane >> 4;
                const int32_t mine = slot + 16 * x, page = x ? pages[1] : pages[0];
                const bool there = 16 * x < left && (uint32_t)page < (uint32_t)b.n_pages;
                ok = ok && (16 * x >= left || there);
                const int32_t in_page = mine - page_entry(a, mine) * b.page_size;
                // lane 0 has the first box, lane 16 the second
                box_page = there ? page : a.end;
                box_slot = in_page;
                box_bytes = (lane == 0 || (lane == 16 && boxes > 1)) ? a.box_rows * DP : 0;
                scales[0] = scales[1] = 0;
                if (there && lane < left) {
                    const int64_t scale = scale_at(b, page, in_page + (lane & 15), kv_head);
                    scales[0] = a.scales.k_scale[scale];
                    scales[1] = a.scales.v_scale[scale];
                }
            };
            // K or V of the 32 slots that were located last into the next unit, swizzled by 128 (64) bytes.
            auto copy = [&](const CUtensorMap *map) {
                const uint32_t u = issued++ % kUnits, bar = ptx::smem_u32(&sh.full[warp][u]);
                const uint32_t to = ptx::smem_u32(ring) + u * kUnitBytes;
                const int32_t second = __shfl_sync(0xffffffffu, box_bytes, 16);
                if (lane == 0)
                    ptx::mbar_arrive_expect_tx(bar, (uint32_t)(box_bytes + second));
                __syncwarp();
                if (box_bytes)
                    ptx::tma_load_4d(to + (uint32_t)(lane ? 16 * DP : 0), map, bar, 0, box_slot, kv_head, box_page);
                __syncwarp();
            };
            auto next_unit = [&]() -> const uint8_t * {  // waits for it
                const uint32_t u = used % kUnits;
                good = warp_wait(ptx::smem_u32(&sh.full[warp][u]), used / kUnits & 1u, &sh.abort) && good;
                ++used;
                return ring + u * kUnitBytes;
            };
            uint32_t scales_now[2] = {0, 0}, scales_next[2] = {0, 0};  // of slot `lane`: K's and V's
            if (at < end) {
                pages[0] = page_of(at);
                pages[1] = page_of(at + 16);
                locate(at, scales_now);
                copy(&tmK);
                copy(&tmV);
                pages[0] = page_of(at + kStep);
                pages[1] = page_of(at + kStep + 16);
                if (at + kStep < end) {
                    locate(at + kStep, scales_next);
                    copy(&tmK);
                }
            }
            for (; good && at < end; at += kStep) {
                const int32_t next = at + kStep;
                pages[0] = page_of(next + kStep);  // for the K copied at the end of this turn
                pages[1] = page_of(next + kStep + 16);
                const uint32_t k_scale = scales_now[0], v_scale = scales_now[1];
                const uint8_t *const k_unit = next_unit();
                float s[2][kLoadsK][4];  // scores of slots g (0, 1) and g + 8 (2, 3) with rows 2 t4 and 2 t4 + 1, in kLoadsK sums
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int n = 0; n < kLoadsK; ++n) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            s[x][n][k] = 0.f;
                        // 16 bytes of a row lie at the place of their number xor the row's (by 8, or by pairs by 4)
                        const int c = kLoadsK * t4 + n, place = DP == 128 ? c ^ g : c ^ (g >> 1 & 3);
                        const uint4 lo = *reinterpret_cast<const uint4 *>(k_unit + (16 * x + g) * DP + place * 16);
                        const uint4 hi = *reinterpret_cast<const uint4 *>(k_unit + (16 * x + g + 8) * DP + place * 16);
                        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            uint32_t a0, a1, a2, a3;
                            halves_of(wl[w], a0, a2);
                            halves_of(wh[w], a1, a3);
                            mma_f16(s[x][n], a0, a1, a2, a3, q[4 * n + w][0], q[4 * n + w][1]);
                        }
                    }
                if constexpr (kLoadsK == 2) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            s[x][0][k] += s[x][1][k];
                }
                // K's scales as factors.  A slot that is held as NaN counts as a score of 0 over zeros and makes l NaN.
                const float k_factor = k_scale == kScaleNan ? 0.f : __uint_as_float(k_scale << 23);
                float2 t[2][2];  // slots g and g + 8, the rows side by side
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float f = __shfl_sync(0xffffffffu, k_factor, 16 * x + g + 8 * k);
                        t[x][k] = ptx::mul2(ptx::mul2(make_float2(s[x][0][2 * k], s[x][0][2 * k + 1]), make_float2(f, f)),
                                            make_float2(inv_row[0], inv_row[1]));
                    }
                __syncwarp();
                if (good && next < end)  // the products above have used K's unit up
                    copy(&tmV);
                const int32_t here = at;
                if (here + kChunk > all) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int32_t slot = here + 16 * x + g + 8 * k;
                            if (slot >= lim[0] || slot == hole[0])
                                t[x][k].x = -INFINITY;
                            if (slot >= lim[1] || slot == hole[1])
                                t[x][k].y = -INFINITY;
                        }
                }
                // t: how far each score is behind the running maximum, in powers of two; moved: how far that has moved
                float2 moved, base;
                {
                    const float mx = fmaxf(m[0], max_of_rows(fmaxf(fmaxf(t[0][0].x, t[0][1].x), fmaxf(t[1][0].x, t[1][1].x))));
                    const float my = fmaxf(m[1], max_of_rows(fmaxf(fmaxf(t[0][0].y, t[0][1].y), fmaxf(t[1][0].y, t[1][1].y))));
                    base = make_float2(mx == -INFINITY ? 0.f : mx, my == -INFINITY ? 0.f : my);  // nothing seen yet: every t is -inf
                    moved.x = m[0] == -INFINITY ? 0.f : (m[0] - base.x) * sl2;
                    moved.y = m[1] == -INFINITY ? 0.f : (m[1] - base.y) * sl2;
                    m[0] = mx;
                    m[1] = my;
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        t[x][k] = ptx::mul2(ptx::add2(t[x][k], make_float2(-base.x, -base.y)), make_float2(sl2, sl2));
                const uint8_t *const v_unit = next_unit();
                const uint32_t nan = __ballot_sync(0xffffffffu, k_scale == kScaleNan || v_scale == kScaleNan);
                // Slots that were not written, zeros at any scale, count as of the least exponent: c is then no less, and 2^c normal.
                constexpr int kLeast = kScaleBias + kMinScaleExp<__is_same(T, __nv_bfloat16)>;
                const int exponent = v_scale == kScaleNan ? 0 : max((int)v_scale, kLeast) - kScaleBias;
                // Weights 2^(t + e - c + kWeightTop) of slots with V's exponent e, c no less than any t + e: the largest e so far where
                // the slots' are alike, else the largest t + e itself, so that weights far below 1 do not leave fp16.
                const int most = __reduce_max_sync(0xffffffffu, here + lane < end ? exponent : -1000);
                const int least = __reduce_min_sync(0xffffffffu, here + lane < end ? exponent : 1000);
                e_most = max(e_most, most);
                e_least = min(e_least, least);
                float2 p[2][2], weight[2][2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        p[x][k] = make_float2(ptx::ex2(t[x][k].x), ptx::ex2(t[x][k].y));
                const float2 before = ptx::add2(make_float2(c[0], c[1]), moved);  // -inf stays
                if (e_most - e_least <= kAlike) {
                    c[0] = c[1] = (float)e_most;
                    const float factor = __uint_as_float((uint32_t)max(exponent - e_most + (int)kWeightTop + 127, 0) << 23);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float f = __shfl_sync(0xffffffffu, factor, 16 * x + g + 8 * k);
                            weight[x][k] = ptx::mul2(p[x][k], make_float2(f, f));
                        }
                } else {
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float e = __shfl_sync(0xffffffffu, (float)exponent, 16 * x + g + 8 * k);
                            t[x][k] = ptx::add2(t[x][k], make_float2(e, e));
                            top[0] = fmaxf(top[0], t[x][k].x);
                            top[1] = fmaxf(top[1], t[x][k].y);
                        }
                    c[0] = fmaxf(before.x, max_of_rows(top[0]));
                    c[1] = fmaxf(before.y, max_of_rows(top[1]));
                    const float2 up = make_float2(c[0] == -INFINITY ? 0.f : kWeightTop - c[0], c[1] == -INFINITY ? 0.f : kWeightTop - c[1]);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            weight[x][k] = make_float2(ptx::ex2(t[x][k].x + up.x), ptx::ex2(t[x][k].y + up.y));
                }
                const float2 fo = make_float2(before.x == -INFINITY ? 0.f : ptx::ex2(before.x - c[0]),
                                              before.y == -INFINITY ? 0.f : ptx::ex2(before.y - c[1]));
                const float2 sum = ptx::add2(ptx::add2(p[0][0], p[0][1]), ptx::add2(p[1][0], p[1][1]));
                const float2 kept = ptx::fma2(make_float2(l[0], l[1]), make_float2(ptx::ex2(moved.x), ptx::ex2(moved.y)), sum);
                l[0] = kept.x;
                l[1] = kept.y;
                if (__builtin_expect(nan != 0, 0)) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            if (nan >> (16 * x + g + 8 * k) & 1u) {
                                if (p[x][k].x != 0.f || t[x][k].x != -INFINITY)
                                    l[0] = NAN;
                                if (p[x][k].y != 0.f || t[x][k].y != -INFINITY)
                                    l[1] = NAN;
                            }
                }
                uint32_t w[2][2];  // weights of slots g and g + 8, then of the lane's row and slots 2 t4 and 2 t4 + 1
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        w[x][k] = transposed(pack2<false>(weight[x][k].x, weight[x][k].y));
                if (__any_sync(0xffffffffu, fo.x != 1.f || fo.y != 1.f)) {
#pragma unroll
                    for (int i = 0; i < kSteps; ++i)
#pragma unroll
                        for (int k = 0; k < 4; k += 2) {
                            const float2 y = ptx::mul2(make_float2(o[i][k], o[i][k + 1]), fo);
                            o[i][k] = y.x;
                            o[i][k + 1] = y.y;
                        }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    uint32_t v[4][kWordsV];  // slots 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = 16 * x + 2 * t4 + (k & 1) + 8 * (k >> 1);
                        if constexpr (DP == 128)
                            *reinterpret_cast<uint4 *>(v[k]) = *reinterpret_cast<const uint4 *>(v_unit + r * DP + (g ^ (r & 7)) * 16);
                        else
                            *reinterpret_cast<uint2 *>(v[k]) =
                                *reinterpret_cast<const uint2 *>(v_unit + r * DP + ((g >> 1) ^ (r >> 1 & 3)) * 16 + (g & 1) * 8);
                        if (here + kChunk > end && here + r >= end) {  // behind the last slot: whatever was there
#pragma unroll
                            for (int i = 0; i < kWordsV; ++i)
                                v[k][i] = 0;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        // dims 2 i and 2 i + 1 of the lane's: codes of two slots side by side, then the other two's
                        const uint32_t sel = (i & 1) ? 0x7362 : 0x5140;
                        const uint32_t lo = __byte_perm(v[0][i / 2], v[1][i / 2], sel);
                        const uint32_t hi = __byte_perm(v[2][i / 2], v[3][i / 2], sel);
                        uint32_t a0, a1, a2, a3;
                        halves_of(lo, a0, a1);
                        halves_of(hi, a2, a3);
                        mma_f16(o[i], a0, a1, a2, a3, w[x][0], w[x][1]);
                    }
                }
                __syncwarp();
                scales_now[0] = scales_next[0];
                scales_now[1] = scales_next[1];
                if (good && next + kStep < end) {
                    locate(next + kStep, scales_next);
                    copy(&tmK);
                }
            }

            // ---- the warps' results become the part's; their O take the rings' places
            auto o_of = [&](int worker) { return reinterpret_cast<float *>(smem_few + worker * kWorkerBytes); };
            __syncwarp();
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
                    *reinterpret_cast<float2 *>(o_of(warp) + row * kRowFloats + g * (DP / 8) + 2 * i) = make_float2(o[i][r], o[i][2 + r]);
            }
            worker_barrier();
            // Joins n results of a row, by a warp: their maxima, the factor of each O, and the sum of l.  of(i): result i's m, c and l.
            auto factors = [&](int n, auto of, auto put, float *joined) {
                float big = -INFINITY, top = -INFINITY, sum = 0.f;
                for (int i = lane; i < n; i += 32)
                    big = fmaxf(big, of(i).x);
#pragma unroll
                for (int i = 16; i; i >>= 1)
                    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, i));
                for (int i = lane; i < n; i += 32) {
                    const float3 y = of(i);
                    if (y.x != -INFINITY) {
                        const float behind = (y.x - big) * sl2;
                        top = fmaxf(top, y.y + behind);
                        sum += y.z * ptx::ex2(behind);
                    } else {
                        sum += y.z;  // 0, or NaN where every score is that
                    }
                }
#pragma unroll
                for (int i = 16; i; i >>= 1) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
                    sum += __shfl_xor_sync(0xffffffffu, sum, i);
                }
                for (int i = lane; i < n; i += 32) {
                    const float3 y = of(i);
                    put(i, y.x == -INFINITY ? 0.f : ptx::ex2(y.y + (y.x - big) * sl2 - top));
                }
                if (lane == 0) {
                    joined[0] = big;
                    joined[1] = top;
                    joined[2] = sum;
                }
            };
            static_assert(kWorkers >= kFewRows, "a warp per row");
            const int tid = (int)threadIdx.x;
            if (warp < kFewRows)
                factors(kWorkers, [&](int i) { return make_float3(sh.m[i][warp], sh.c[i][warp], sh.l[i][warp]); },
                        [&](int i, float f) { sh.f[i][warp] = f; }, sh.joined[warp]);
            worker_barrier();
            // A thread has 4 neighbouring dims of a row.
            const int row = tid / (DP / 4), dim = tid % (DP / 4) * 4;
            const bool mine = row < kFewRows;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](float f, const float4 &z) {  // f = 0: z may be anything
                if (f != 0.f) {
                    y.x = fmaf(f, z.x, y.x);
                    y.y = fmaf(f, z.y, y.y);
                    y.z = fmaf(f, z.z, y.z);
                    y.w = fmaf(f, z.w, y.w);
                }
            };
            if (mine) {
#pragma unroll 5
                for (int i = 0; i < kWorkers; ++i)
                    add(sh.f[i][row], *reinterpret_cast<const float4 *>(o_of(i) + row * kRowFloats + dim));
            }
            bool whole = true;
            if ((part.flags & kWhole) == 0) {
                // The task's parts meet in the workspace; the one that comes last joins them all in their order.
                const int n = part.last - part.first + 1;
                auto place = [&](int cta) { return (int64_t)cta * 2 + (cta == part.first ? 1 : 0); };
                float *const ml = reinterpret_cast<float *>(a.part_ml);
                const int64_t of_ml = 2 * a.quarters * 64, of_o = (int64_t)2 * a.quarters * 32 * a.piece;
                float *const po = reinterpret_cast<float *>(a.part_o);
                const int64_t to = place((int)blockIdx.x);
                if (mine)
                    *reinterpret_cast<float4 *>(&po[to * of_o + row * DP + dim]) = y;
                if (tid < 3 * kFewRows)
                    ml[to * of_ml + tid] = sh.joined[tid / 3][tid % 3];
                __threadfence();
                worker_barrier();
                int32_t *const node = a.nodes + (int64_t)part.first * kLevels * 8;
                if (tid == 0) {
                    const int before = atomicAdd(node, 1);
                    sh.last = before == n - 1;
                    if (before == n - 1)
                        *node = 0;  // for the next call
                }
                worker_barrier();
                whole = sh.last != 0;
                if (whole) {
                    __threadfence();
                    float *const all_ml = reinterpret_cast<float *>(smem_few);  // O is out of the rings
                    for (int i = tid; i < n * 3 * kFewRows; i += kWorkers * 32) {
                        const int of = i / (3 * kFewRows);
                        all_ml[i] = __ldcg(&ml[place(part.first + of) * of_ml + i - of * 3 * kFewRows]);
                    }
                    worker_barrier();
                    float *const all_f = all_ml + kMaxCtas * 3 * kFewRows;
                    if (warp < kFewRows)
                        factors(n,
                                [&](int i) {
                                    const float *const p = all_ml + (i * kFewRows + warp) * 3;
                                    return make_float3(p[0], p[1], p[2]);
                                },
                                [&](int i, float f) { all_f[i * kFewRows + warp] = f; }, sh.joined[warp]);
                    worker_barrier();
                    y = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (mine) {
#pragma unroll 4
                        for (int i = 0; i < n; ++i)
                            add(all_f[i * kFewRows + row],
                                __ldcg(reinterpret_cast<const float4 *>(&po[place(part.first + i) * of_o + row * DP + dim])));
                    }
                }
            }
            const float top = mine ? sh.joined[row][1] : 0.f, sum = mine ? sh.joined[row][2] : 0.f;
            if (whole && mine && dim < b.head_dim) {
                const int pos = row / a.group, i = part.i0 + pos;
                if (pos < a.positions && i < part.q.n) {
                    // No slot seen: zeros; NaN stays NaN.  2^c last: with 1 / l it would leave fp32's range for V near 2^-110.
                    const float by = sum == 0.f ? 0.f : 1.f / sum, up = ptx::ex2(top - kWeightTop);
                    uint16_t *const dst = a.out.data + (int64_t)(part.q.start + i) * a.out.row_stride +
                                          (int64_t)(part.kv_head * a.group + row - pos * a.group) * a.out.head_stride;
                    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
                    *reinterpret_cast<uint2 *>(dst + dim) =
                        make_uint2(pack2<kBf16>(y.x * by * up, y.y * by * up), pack2<kBf16>(y.z * by * up, y.w * by * up));
                }
            }
        }
        // Copies in flight land before the shared memory goes away: none in a call that went well.
        if (lane == 0)
            for (uint32_t u = 0; u < kUnits && u < issued; ++u)
                wait_drain(ptx::smem_u32(&sh.full[warp][u]), last_parity(issued, u, kUnits));
        __syncwarp();
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_DEVICE_TIMEOUT);
    publish(a, kFewThreads);
}

template <int DP, typename T>
int launch_few(const CUtensorMap &tk, const CUtensorMap &tv, const AttendArgs &a, int ctas, cudaStream_t stream)
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
                                     (int)kFewSmem) != cudaSuccess)
                return WINO_ERR_CUDA;
            done[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = kFewSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attend_few_kernel<DP, T>, tk, tv, a) == cudaSuccess ? WINO_OK : WINO_ERR_CUDA;
}

}  // namespace

namespace attend {

namespace {

// How the query heads of a kv head go into tiles: the most that divide them, up to kFewRows.
int32_t few_group(const wino_kv_batch &b)
{
    const int32_t heads = b.n_q_heads / b.n_kv_heads;
    int32_t group = std::min(heads, kFewRows);
    while (heads % group != 0)
        --group;
    return group;
}

// The units that a batch may have at most in tasks of one tile, as attend_units counts them.
double few_units(const wino_kv_batch &b)
{
    const int32_t group = few_group(b), positions = kFewRows / group;
    return (double)b.n_seq * (b.n_rows / positions + 1) * (b.n_q_heads / group) *
           ((double)b.table_width * b.page_size / kTileN + 1 + kFewTaskCost);
}

}  // namespace

// A tile of rows per sequence and kv head on average, or two where the heads of one row need them: each tile reads K and V, the
// second mostly from the L2 cache. This kernel and wino_attend's over tiles of the element type (us), heads of 128: 64 tokens of 4
// heads to a kv head over up to 32767 slots 154 and 330, one over 262144 97 and about 180, one over 300 9.1 and 13; 64 of 16 heads
// to a kv head over up to 16000 142 and 174, of 32 (four tiles) 134 and 107. Two tiles of rows gain less and would lose
// the bits of wino_attend over the values: 64 sequences of 4 rows over up to 16000 252 and 279, one over 262144 171 and 181.
// The host does not know the lengths, so averages decide: 127 single tokens over up to 8000 with a chunk of 100 rows behind 7900
// take 307 here and 474 there (the tokens alone 200 and 410), but 2 sequences of 64 rows over 4000 in a batch of 64 whose others are
// absent 94 and 35.
bool few_rows(const wino_kv_batch &b)
{
    const int32_t group = few_group(b);
    return b.n_q_heads / b.n_kv_heads <= 2 * group && b.n_rows <= (int64_t)b.n_seq * (kFewRows / group) &&
           few_units(b) < 4611686018427387904.0;
}

int launch_few(AttendArgs a, int ctas, cudaStream_t stream)
{
    const wino_kv_batch &b = a.b;
    a.end = b.n_pages;
    a.box_rows = std::min(b.page_size, kChunk);
    const int32_t width = b.head_dim <= 64 ? 64 : 128;
    CUtensorMap tk, tv;
    int rc;
    if ((rc = encode_codes(&tk, b.k_cache, b, width, a.box_rows, true)) != WINO_OK ||
        (rc = encode_codes(&tv, b.v_cache, b, width, a.box_rows, true)) != WINO_OK)
        return rc;
    a.group = few_group(b);
    a.split = b.n_q_heads / b.n_kv_heads / a.group;
    a.positions = kFewRows / a.group;
    for (int i = 0; i < 2; ++i) {
        const uint64_t w = (uint64_t)(i + 1) * a.positions;
        a.magic[i] = (uint32_t)(((uint64_t(1) << 32) + w - 1) / w);
    }
    a.min_units = 3;  // one token over 1500 slots 13.1 us, with 6 14.4; over 300 9.1, over 16384 19.3 with either
    a.wide = few_units(b) >= 2147483648.0;
    const bool bf16 = (b.dtype & ~WINO_CACHE_E4M3) == WINO_BF16;
    if (width == 64)
        return bf16 ? wino::launch_few<64, __nv_bfloat16>(tk, tv, a, ctas, stream) : wino::launch_few<64, __half>(tk, tv, a, ctas, stream);
    return bf16 ? wino::launch_few<128, __nv_bfloat16>(tk, tv, a, ctas, stream) : wino::launch_few<128, __half>(tk, tv, a, ctas, stream);
}

}  // namespace attend
}  // namespace wino
