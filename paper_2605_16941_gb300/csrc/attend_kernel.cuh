// attend_kernel.cuh -- the kernel of wino_attend (attend.cu) and wino_attend_scaled (attend_scaled.cu): attention of a step's
// rows over a paged cache.
//
// out = softmax(scale Q K^T) V with the running maximum m, sum l and unnormalised product O of an online softmax: per tile
// of 128 slots S = Q K^T, m' = max(m, max S), P = exp(S - m'), l' = l exp(m - m') + sum P, O' = O exp(m - m') + P V.
//
// Rows.  The G query heads of a kv head share its K and V, so a tile of M = 128 rows is floor(128 / G) row positions times
// G heads.  A task is one sequence, one kv head and two such tiles: both tiles multiply every K and V tile that is
// staged.  Where a task has rows in its first tile only (single tokens, short blocks, or all tasks of a call that has few),
// its two softmax warpgroups take even and odd slot tiles instead, each with its own m, l and O, joined at the end.
//
// Work.  A task costs one unit per slot tile.  The units of all tasks in order are cut into equal runs, one per CTA, from
// lengths that are read on the device.  The parts of a task that several runs hold are joined in a binary tree over their
// order: of two neighbours, whichever is done first leaves its (m, l, O) in the workspace, and the other goes on with the
// join.  No CTA waits for another, the tree does not depend on who is first, and each softmax warp joins its own rows.
//
// A CTA has 12 warps: two softmax warpgroups (one thread per row), and one warp each for the plan, the copies of Q and K,
// the copies of V (TMA, a box per page), and the MMAs.  S lies in tensor memory, 128 columns per warpgroup; P, as 16-bit
// pairs, is the A operand of P V from there (over S with 128 dims, beside it with 64); O lies beside it, DP columns per
// warpgroup.  K and V tiles go through a ring of shared-memory slots each.
//
// What bounds it (us; floors from 6.7 TB/s and 1.9 PFLOP/s):
//   few rows per slot: the K and V stream from HBM.  64 tokens over 500 to 32767 slots, 32 heads over 8 kv heads of 128:
//     2.05 GB in 303 to 308 = 6.7 TB/s (floor 306).  With one warp for all copies 407: a warp issues a 2 KB box in 68 to 130
//     clocks, so K and V have a warp each and a page's halves one box.
//   many rows, 128 dims: each warpgroup's chain of scores (512 clocks), softmax (1400) and P V (512, half of it behind the
//     second half of the weights); two warpgroups overlap to 2500 to 2700 clocks per pair of tiles, against 2048 of MMAs.
//     Four prompts of up to 8192 tokens, 32 heads: 380 (floor 313), 1.56 PFLOP/s of products that the mask keeps; 416 where
//     calls follow one another for long and the power cap lowers the clock.
//   many rows, 64 dims: the softmax, 2100 to 2400 clocks per pair of tiles, 1024 of them exponentials (32 a clock and SM)
//     and the rest mostly latencies of loads, votes and barriers, which two warps per scheduler do not hide.  Two threads
//     per row (16 softmax warps of 104 registers) take the same time, at 128 dims too: each repeats the latencies.
//   short calls: 1.4 of launch, 1.5 of plan, then one latency after the other; 32 heads over 300 slots 9.7.
//   many short sequences: every CTA's plan loads all lengths, 32 sequences a round and twice where there are more, and each task
//     pays its own chain of latencies.  Single tokens over 61 slots, 8 heads of 64 over 2: 10 for 32 sequences, 29 for 256, 92
//     for 1024, 371 for 4096, 1620 for 16384 (floor 81).
//
// An 8-bit cache (kScaled).  Two warps copy the codes of a slot tile and their scales into stages, one of K and one of V (two each
// with 64 dims), and four warps more write them as the tiles of the element type that TMA would have brought, swizzled, into one ring
// for both in the order of their use; from there on all is as above, and so are the results.  Rows that are held as NaN become
// something finite (0 times NaN is not 0), and the sums of the rows that see them NaN.  Few rows have a kernel of their own
// (attend_few.cu).  What bounds it: those four warps, some 1600 clocks a tile in bf16 and 1170
// in fp16 (804 and 581 of conversion by themselves, the rest reads of shared memory and waits, with one such warp to a
// scheduler), K's and V's one after the other: 4 x 512 rows of 32 heads over 8-bit caches of 1605 to 3890 slots 69 us, 57 over 16-bit ones.
// Shared memory alone would take 2560 clocks per pair of tiles at 128 bytes a clock (MMAs 1536, copies 256, conversion 768).
// Tried, same case: codes straight from global memory to registers 122 (latency), eight warps for them 84 (the other roles' registers
// then do not suffice), the next half tile's codes read while one is written 89, stages of 64 slots 70.5, a form that spilled
// registers in its loops 79 (spills of 44 bytes in the planning warp and ahead of the roles cost nothing; now there are none).
// Code counts: a tenth of the warps' stalls is for instructions, and one wait and ten instructions more per part in the softmax's role
// cost prompts 5 %.
//
// Times in these comments are of calls replayed from a CUDA graph on one input, both sides of a rule on one device.
//
// Precision: S, m, l and O in fp32; P is rounded to the element type because the tensor cores take no wider weights beside
// 16-bit values (half a step per weight, as much as the result's own rounding); l sums the unrounded weights.  Against 64 bits out
// is 1.2 to 1.4 times as far off as with fp32 weights.  In the online softmax (arXiv 1805.02867) any m serves that keeps the
// exponentials in range: here it follows the row's maximum only when that has grown by more than some bits (kRescaleBits), so
// that O is rarely rescaled; the quotient O / l does not depend on m.  fp16 has 40 bits of range, subnormals included, and many
// small weights may add up to the result: there P, l and O carry a factor 2^kTopBits that the quotient drops.  P ends at
// 2^15.9 < 65504, a weight keeps all its bits down to 2^-23.9 of the row's largest, and what is lost below is 2^-34.9 each.
// Scores may lie anywhere in fp32: only their differences count, and far from zero these are formed before they are scaled.
// More bits above leave fewer to grow and rescale O more often: with 4 / 5 / 6 / 8 to grow, four prompts in fp16 take 430 / 399 /
// 393 / 389 us, the chunks of 64 dims 76.7 / 75.6 / 74.7 / 72.8.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cstring>
#include <mutex>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "e4m3.cuh"
#include "kv_batch.cuh"
#include "ptx_attend.cuh"
#include "wait.cuh"

namespace wino {
namespace attend {

constexpr int kTileM = 128, kTileN = 128;  // rows and slots of a tile
constexpr int kSoftmaxThreads = 256;
constexpr int kWarpK = 8, kWarpMma = 9, kWarpV = 10, kWarpPlan = 11, kWarpDecode = 12;  // the last: the first of four
template <bool kScaled>
constexpr int kAttendThreads = kSoftmaxThreads + (kScaled ? 256 : 128);
constexpr int32_t kNoSlot = 1 << 30;    // behind every slot
constexpr int kMaxCtas = 160;           // an SM each
constexpr int kLevels = 8;              // of the tree over the parts of a task: 2^8 >= kMaxCtas
constexpr int kParts = 4;               // parts of tasks that the planning warp may be ahead
constexpr int kTaskCost = 3;            // what a task costs beside its slot tiles, in slot tiles
constexpr int kFewTaskCost = 8;         // and one of few rows, whose tiles take less (attend_few.cu)
constexpr int kSnap = 2;                // a cut this near to a task's border (in slot tiles) is moved there
constexpr float kRescaleBits[2] = {6.f, 8.f};  // fp16, bf16
constexpr float kTopBits[2] = {9.9f, 0.f};     // the P of a score of m is 2^this
constexpr float kFarBits = 65536.f;            // up to here m sl2 is rounded by 2^-8 at most: P stays below 65504
constexpr uint32_t kTmemAll = 512;
constexpr uint32_t kSharedBytes = 3 * 1024;  // for struct Shared, behind the tiles
constexpr uint32_t kHalfBytes = kTileN * 128;  // 128 rows of 64 elements: one 128-byte swizzled block
// Where slot row r, dims 64 h .. 64 h + 63 of a K or V tile lie: (r / 8) group + h half + (r % 8) 128 bytes.  With 128 dims
// one copy brings both halves of a page's rows, interleaved by groups of 8 rows, if the cache's strides let one
// coordinate of the tensor map count heads and pages (`joint`); else each half has a copy and a block of its own.
struct TileLayout {
    uint32_t group, half;
};

struct AttendArgs {
    wino_heads q, out;
    wino_kv_batch b;
    float scale_log2;  // scale * log2(e)
    StatusWords *status;
    int32_t *nodes;   // [kMaxCtas][kLevels][8 warps], zero between calls: how many of a node's two children are there
    float2 *part_ml;  // [kMaxCtas][2][2 quarters][32 lanes]: m, l of the rows of a warp
    float4 *part_o;   // [kMaxCtas][2][2 quarters][piece / 4][32 lanes]
    int32_t quarters, piece;   // warps of a warpgroup with rows at most, columns that a warp keeps at most
    int32_t group, positions;  // query heads per kv head, row positions per tile
    int32_t split;             // 2: a task has half of a kv head's query heads (`group`), and each half counts as a kv head in Part
    uint32_t magic[2];         // ceil(2^32 / w) for tasks of w = positions and of 2 positions
    int32_t box_rows, boxes;   // slots per copy (a page, or 128 of one), copies per slot tile and 64 dims
    int32_t min_units;         // a CTA's run is at least this long
    int32_t wide;              // units may need 64 bits
    int32_t wide_rows;         // rows of out are 32-byte aligned
    int32_t page_shift;        // log2(page_size), or -1
    int32_t joint;             // heads per page in the tensor map's last coordinate, page * joint + head; 0: two coordinates
    int32_t end;               // a coordinate behind the cache's last page
    TileLayout tile;
    wino_kv_scales scales;  // of an 8-bit cache
};

// Tasks of `tiles` row tiles (1 or 2) of one kv head of a sequence.  A row count is at most 2^24 and 2 positions at most 256,
// so that the product with the magic number is the quotient (its error is below 2^24 / 2^32 < 1 / 256).
__device__ __forceinline__ int32_t tasks_of(const AttendArgs &a, const SeqRows &q, int32_t tiles)
{
    const int32_t w = tiles * a.positions;
    return w == 1 ? q.n : (int32_t)__umulhi((uint32_t)(q.n + w - 1), a.magic[tiles - 1]);
}

__device__ __forceinline__ int32_t page_entry(const AttendArgs &a, int32_t slot)
{
    return a.page_shift >= 0 ? slot >> a.page_shift : slot / a.b.page_size;
}

// Slots that some row of task `x` sees: its last row sees as many as any.
__device__ __forceinline__ int32_t task_slots(const AttendArgs &a, const SeqRows &q, int32_t tiles, int32_t x)
{
    return row_sees(a.b, q, min(q.n, (x + 1) * tiles * a.positions) - 1).lim;
}

__device__ __forceinline__ int32_t tiles_of(int32_t slots) { return max(1, (slots + kTileN - 1) / kTileN); }

// The cut of `total` units into n runs: run c starts at unit floor(c total / n).  U: 32 bits unless the host finds that the
// units may need more (64-bit arithmetic, divisions above all, is slow and much code).
template <typename U>
struct Cut {
    U total, per;
    int32_t n, more;  // total = n per + more
    float inv_n, runs_per_unit;
    // Up to as many tasks as CTAs: a multiple of the tasks, so that tasks of one length are cut alike, unless that makes the
    // runs longer by more than joining a part costs.  Quotients of integers below 2^11 are taken in fp32, half a unit off the
    // border: exact, and shorter than an integer division.
    __device__ __forceinline__ Cut(U units, U tasks, int32_t ctas, int32_t min_units) : total(units)
    {
        n = ctas;
        if (total < (U)(ctas * min_units))
            n = max(1, (int32_t)__fdividef((float)(int32_t)total + 0.5f, (float)min_units));
        inv_n = __fdividef(1.f, (float)n);
        if (tasks > 0 && tasks <= (U)n) {
            const int32_t whole = (int32_t)tasks * (int32_t)__fdividef((float)n + 0.5f, (float)(int32_t)tasks);
            const float inv_whole = __fdividef(1.f, (float)whole);
            if ((float)total * (inv_whole - inv_n) < (float)min_units) {
                n = whole;
                inv_n = inv_whole;
            }
        }
        runs_per_unit = __fdividef((float)n, (float)total);
        per = total / (U)n;
        more = (int32_t)(total - per * (U)n);
    }
    // c more < 2^15 and n <= 160: the quotient's distance from an integer, at least 1 / (2 n), is far above its rounding
    __device__ __forceinline__ U start(int32_t c) const
    {
        return (U)c * per + (U)(int32_t)(((float)(c * more) + 0.5f) * inv_n);
    }
    // The run that holds a unit: off by one at most from the quotient in fp32.
    __device__ __forceinline__ int32_t run_of(U unit) const
    {
        int32_t c = min(n - 1, (int32_t)((float)unit * runs_per_unit));
        while (start(c) > unit)
            --c;
        while (c + 1 < n && start(c + 1) <= unit)
            ++c;
        return c;
    }
    // A start inside the task [t0, t1), moved to the task's border where that is near: joining parts costs more than it
    // evens out.
    static __device__ __forceinline__ U snap(U unit, U t0, U t1, int32_t cost)
    {
        return unit < t0 + cost + kSnap ? t0 : (t1 < unit + kSnap ? t1 : unit);
    }
};

// One part of a task, as the planning warp hands it to the others: slot tiles [j0, j0 + n) of one sequence, kv head and
// one or two row tiles.
enum : int32_t { kTwo = 1, kTail = 2, kWhole = 4, kEnd = 8 };
struct alignas(16) Part {
    int32_t flags;   // kTwo: rows in both tiles; kTail: the last tile ends behind kv_end; kWhole: the task's only part
    int32_t kv_end;  // slots that some row sees
    int32_t j0, n;   // n = 0: nothing to see, the rows get zeros
    int32_t seq, kv_head;
    int32_t i0;      // the sequence's row of the first position
    int32_t first, last;  // without kWhole: the CTAs whose runs hold slot tiles of the task
    SeqRows q;
};

template <int DP, bool kScaled>
struct Config {
    static constexpr uint32_t kTileBytes = (DP / 64) * kHalfBytes;  // 128 rows or slots
    // Ring slots of K and of V, beside the two Q tiles.  V waits for its weights, K for nothing.  Codes: one ring for the
    // values of both, in the order of their use, and behind it stages of codes, of K and as many of V.
    static constexpr int kSlotsK = kScaled ? 0 : (DP == 128 ? 2 : 5), kSlotsV = kScaled ? (DP == 128 ? 4 : 6) : (DP == 128 ? 3 : 7);
    static constexpr int kSlots = kSlotsK + kSlotsV;
    static constexpr int kStages = kScaled ? (DP == 128 ? 1 : 2) : 0;
    static constexpr uint32_t kStageBytes = kTileN * DP;
    static constexpr uint32_t kRing = kSlots * kTileBytes + 2 * kStages * kStageBytes;
    static constexpr uint32_t kShared = kSharedBytes + (kScaled && DP == 64 ? 1024 : 0);
    // Tensor memory columns of warpgroup g: S at kTmemS + g 128, P at kTmemP + g kStrideP, O at kTmemO + g DP.  With 64 dims
    // P has columns of its own, and the scores of the next tile are computed as soon as S is in registers; with 128
    // they are taken by O, P overwrites S, and the next scores wait for P V.
    static constexpr bool kEarly = DP == 64;
    static constexpr uint32_t kTmemS = 0, kTmemP = kEarly ? 256 : 0, kStrideP = kEarly ? 64 : 128;
    static constexpr uint32_t kTmemO = kEarly ? 384 : 256;
    static constexpr uint32_t kSmem = 2 * kTileBytes + kRing + kShared;
};

// With codes the ring has at most 6 slots, V's slots need no zeroing apart, and each stage (of K, then of V) has its scales.
template <bool kScaled, int kStages>
struct alignas(16) Shared {
    static constexpr int kRing = kScaled ? 6 : 12, kAll = kScaled ? 2 * kStages : 1;
    Part parts[kParts];
    uint64_t part_full[kParts], part_empty[kParts];
    uint64_t q_full, q_empty;
    uint64_t full[kRing], empty[kRing];
    uint64_t s_full[2], s_free[2], p_half[2], p_ready[2], o_done[2];
    uint64_t lead[4];  // warpgroup 0's warp of this quarter is half through its first tile's weights
    uint64_t zeroed[kScaled ? 1 : kRing];  // per ring slot of V: the cache slots behind the last one hold zeros
    uint64_t stage_full[kAll], stage_free[kAll];
    uint64_t ml_ready, ml_done;
    uint64_t mma_done;
    uint32_t tmem;
    int32_t abort;
    float2 ml[2][kTileM];
    alignas(16) uint8_t scale[kAll][kScaled ? kTileN : 16];
    // Of a part: the first two of its slots whose K or V is held as NaN, kNoSlot where there are none.  Two suffice, since a row
    // sees all slots before its limit but one.
    alignas(8) int32_t nan[kScaled ? kParts : 1][2];
};

template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    if (kBf16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Bounded wait of a whole warp: the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int32_t *abort)
{
    return __all_sync(0xffffffffu, wait_bounded(bar, parity, abort));
}

// A reader's place in the ring of parts.
struct PartReader {
    uint32_t count = 0;
    __device__ __forceinline__ uint32_t parity() const { return (count / kParts) & 1u; }
    __device__ __forceinline__ int slot() const { return (int)(count % kParts); }
};

// The parity of the last copy into slot s of a ring of `slots`, after `issued` > s copies that took the slots in turn.
__host__ __device__ constexpr uint32_t last_parity(uint32_t issued, uint32_t s, uint32_t slots) { return ((issued - 1 - s) / slots) & 1u; }

// Walks the ring as the copying warps do, slot by slot with the phase turned over at its end.
constexpr bool last_parity_holds()
{
    for (uint32_t slots = 1; slots <= 8; ++slots) {
        uint32_t last[8] = {}, slot = 0, phase = 0;
        for (uint32_t issued = 1; issued <= 40; ++issued) {
            last[slot] = phase;
            if (++slot == slots) {
                slot = 0;
                phase ^= 1u;
            }
            for (uint32_t s = 0; s < slots && s < issued; ++s)
                if (last_parity(issued, s, slots) != last[s])
                    return false;
        }
    }
    return true;
}
static_assert(last_parity_holds(), "drained parities");

template <typename U>
__device__ __forceinline__ U warp_sum(U x, int width)  // over groups of `width` lanes
{
    for (int i = width >> 1; i; i >>= 1)
        x += __shfl_xor_sync(0xffffffffu, x, i);
    return x;
}

template <typename U>
__device__ __forceinline__ U warp_total(U x)
{
    if constexpr (sizeof(U) == 4)
        return __reduce_add_sync(0xffffffffu, x);
    else
        return warp_sum(x, 32);
}

template <typename U>
__device__ __forceinline__ U warp_scan(U x, int lane)  // inclusive
{
#pragma unroll
    for (int i = 1; i < 32; i <<= 1) {
        const U up = __shfl_up_sync(0xffffffffu, x, i);
        if (lane >= i)
            x += up;
    }
    return x;
}

// The planning warp: cuts the work and hands this CTA's run out part by part.  U is unsigned.  kMostTiles: row tiles of a task.
template <typename U, typename S, int kMostTiles = 2, bool kOverCodes = false>
__device__ __forceinline__ void plan(const AttendArgs &a, S &sh, int lane)
{
    constexpr int kCost = kMostTiles == 1 ? kFewTaskCost : kTaskCost;
    const int32_t n_seq = a.b.n_seq, n_kv = a.b.n_kv_heads * a.split;
    bool ok = true;
    int width = 32;  // lanes per sequence
    while (width > 1 && n_seq * width > 32)
        width >>= 1;
    const int per_round = 32 / width, sub = lane & (width - 1);
    SeqRows q;
    U share = 0, mine = 0;  // units of this lane's tasks, and of its sequence, of one kv head
    int32_t n_tasks = 0;    // and its tasks
    int32_t row_tiles = kMostTiles;  // of a task
    auto load_round = [&](int32_t s0) {
        const int32_t s = s0 + lane / width;
        q.n = 0;
        q.ok = true;
        if (s < n_seq)
            q = load_seq(a.b, s);
        ok = ok && q.ok;
    };
    auto count = [&]() {
        share = 0;
        n_tasks = q.n > 0 ? tasks_of(a, q, row_tiles) : 0;
#pragma unroll 1
        for (int32_t x = sub; x < n_tasks; x += width)
            share += (U)(tiles_of(task_slots(a, q, row_tiles, x)) + kCost);
        mine = warp_sum(share, width);
    };
    U total, tasks;
#pragma unroll 1
    while (true) {
        total = tasks = 0;
#pragma unroll 1
        for (int32_t s0 = 0; s0 < n_seq; s0 += per_round) {
            if (row_tiles == kMostTiles || n_seq > per_round)
                load_round(s0);
            count();
            total += warp_total(share);
            tasks += warp_total(sub == 0 ? (U)n_tasks : (U)0);
        }
        // Few and short tasks: one row tile each gives twice as many, for twice the copies of K and V, and fewer parts to
        // join.  256 rows of each of 32 heads behind 1025 / 4097 / 16385 slots (runs of 3 / 8 / 28 units): 16.8 / 28.1 / 97.4 us
        // with one row tile, 22.5 / 32.7 / 66.8 with two; 64 rows of 4 heads to each of 8 behind 8193 (14): 28.7 and 35.8.
        if (row_tiles == 1 || a.b.n_rows <= a.positions || tasks * (U)n_kv * 2 > (U)gridDim.x ||
            total * (U)n_kv > (U)gridDim.x * 16)
            break;
        row_tiles = 1;
    }
    total *= (U)n_kv;
    const Cut<U> cut(total, tasks * (U)n_kv, (int32_t)gridDim.x, a.min_units);
    const int32_t c = (int32_t)blockIdx.x;
    U at = cut.start(c);  // the next unit to hand out
    const U end = c < cut.n && total > 0 ? cut.start(c + 1) : at;
    // The current task: `index` among its kv head's.  A sequence's tasks come by kv head and index while there are no more
    // than CTAs: neighbours of nearly one length are then cut alike.  More of them come by index and kv head, so that
    // CTAs some way apart read one head's K and V at the same time and one of them finds it in the L2 cache.  4 x 512 rows of 32
    // heads (256 tasks) 82.1 and 79.7 us; 256 rows of 32 heads behind 1025 slots (64 tasks) 16.8 and 23.5.
    const bool by_index = tasks * (U)n_kv > (U)cut.n;
    int32_t seq = 0, kv_head = 0, index = 0;
    U task = 0;  // the unit at which the current task starts
    uint32_t sent = 0;
    bool go = at < end;
    if (go) {
        // the sequence that holds unit `at`
        U before = 0;
#pragma unroll 1
        for (int32_t s0 = 0; s0 < n_seq && n_seq > 1; s0 += per_round) {  // one sequence: every lane has it
            if (n_seq > per_round) {
                load_round(s0);
                count();
            }
            const U pre = warp_scan(sub == 0 ? mine * (U)n_kv : (U)0, lane);
            const unsigned hit = __ballot_sync(0xffffffffu, before + pre > at);
            if (hit) {
                const int src = __ffs(hit) - 1;  // a sequence's first lane: `pre` grows there only
                seq = s0 + src / width;
                mine = __shfl_sync(0xffffffffu, mine, src);
                task = before + __shfl_sync(0xffffffffu, pre, src) - mine * (U)n_kv;
                q.start = __shfl_sync(0xffffffffu, q.start, src);
                q.n = __shfl_sync(0xffffffffu, q.n, src);
                q.kv = __shfl_sync(0xffffffffu, q.kv, src);
                q.base = __shfl_sync(0xffffffffu, q.base, src);
                n_tasks = __shfl_sync(0xffffffffu, n_tasks, src);
                break;
            }
            before += __shfl_sync(0xffffffffu, pre, 31);
        }
        // its kv head, and by the sum over 32 tasks at a time the task; or the other way round
        auto to_head = [&](U each) {
            const U behind = at - task;
            kv_head = (int32_t)__fdividef((float)behind, (float)each);  // off by one at most
            while ((U)kv_head * each > behind)
                --kv_head;
            while ((U)(kv_head + 1) * each <= behind)
                ++kv_head;
            task += (U)kv_head * each;
        };
        if (!by_index)
            to_head(mine);
        const U heads = by_index ? (U)n_kv : (U)1;
#pragma unroll 1
        for (int32_t p0 = 0; p0 < n_tasks && n_tasks > 1; p0 += 32) {
            const int32_t p = p0 + lane;
            const U cost = p < n_tasks ? (U)(tiles_of(task_slots(a, q, row_tiles, p)) + kCost) * heads : (U)0;
            const U pre = warp_scan(cost, lane);
            const unsigned hit = __ballot_sync(0xffffffffu, task + pre > at);
            if (hit) {
                const int src = __ffs(hit) - 1;
                index = p0 + src;
                task += __shfl_sync(0xffffffffu, pre - cost, src);
                break;
            }
            task += __shfl_sync(0xffffffffu, pre, 31);
        }
        const U cost = (U)(tiles_of(task_slots(a, q, row_tiles, index)) + kCost);
        if (by_index)
            to_head(cost);
        // a start that moves to the task's end belongs to the next one, which the walk below finds
        at = Cut<U>::snap(at, task, task + cost, kCost);
    }
#pragma unroll 1
    while (true) {
        Part part;
        part.flags = kEnd;
        part.kv_end = part.j0 = part.n = part.i0 = part.first = part.last = 0;
        if (go) {
            const int32_t slots = task_slots(a, q, row_tiles, index), tiles = tiles_of(slots);
            const U tile0 = task + kCost, next = tile0 + (U)tiles;  // a task's own cost comes before its tiles
            const U stop = end >= next ? next : Cut<U>::snap(end, task, next, kCost);
            part.j0 = at > tile0 ? (int32_t)(at - tile0) : 0;
            part.n = (stop > tile0 ? (int32_t)(stop - tile0) : 0) - part.j0;
            part.kv_end = slots;
            part.i0 = index * row_tiles * a.positions;
            const bool to_end = stop == next;
            // the part's first pages, which the copying warps read next, on their way to the L1 cache
            const int32_t entry = page_entry(a, part.j0 * kTileN) + lane;
            if (part.n > 0 && slots > 0 && entry <= page_entry(a, slots - 1))
                ptx::touch(a.b.page_table + (int64_t)seq * a.b.table_width + entry);
            part.flags = (row_tiles == 2 && q.n - part.i0 > a.positions ? kTwo : 0) |
                         (to_end && (slots & (kTileN - 1)) != 0 ? kTail : 0) | (to_end && part.j0 == 0 ? kWhole : 0);
            if ((part.flags & kWhole) == 0 && part.n > 0) {
                // the cuts that stay inside the task are those of starts in [tile0 + kSnap, next - kSnap]
                part.first = cut.run_of(tile0 + kSnap - 1);
                part.last = cut.run_of(next - kSnap);
            }
            task = next;
            at = max(at, next);
            go = at < end;
        }
        part.seq = seq;
        part.kv_head = kv_head;
        part.q = q;
        const bool last = (part.flags & kEnd) != 0;
        if (last || part.n > 0) {  // a run may hold none of a task's tiles
            if (part.kv_end == 0)
                part.n = 0;
            const int slot = (int)(sent % kParts);
            if (!warp_wait(ptx::smem_u32(&sh.part_empty[slot]), ((sent / kParts) & 1u) ^ 1u, &sh.abort))
                break;
            if (lane == 0) {
                sh.parts[slot] = part;
                if constexpr (kOverCodes)
                    sh.nan[slot][0] = sh.nan[slot][1] = kNoSlot;
                ptx::mbar_arrive(ptx::smem_u32(&sh.part_full[slot]));
            }
            __syncwarp();
            ++sent;
        }
        if (last)
            break;
        if (go) {
            int32_t &inner = by_index ? kv_head : index, &outer = by_index ? index : kv_head;
            if (++inner == (by_index ? n_kv : n_tasks)) {
                inner = 0;
                ++outer;
            }
            if (outer == (by_index ? n_tasks : n_kv)) {
                outer = 0;
                do {  // there are units left, so there is a sequence with rows
                    ++seq;
                    q.n = 0;
                    if (seq < n_seq)
                        q = load_seq(a.b, seq);
                } while (q.n == 0 && seq < n_seq);
                go = q.n > 0;
                n_tasks = go ? tasks_of(a, q, row_tiles) : 0;
            }
        }
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
}

// Joins this warp's rows of a part with the task's other parts: climbs the tree over parts first .. last while the other
// child of a node is there already, and leaves what it has got where it is not.  O is in tensor memory (columns [c0, c1)
// from t_o), m (units of S) and l in registers; true: they are the whole task's now.
__device__ __forceinline__ bool join_parts(const AttendArgs &a, const Part &part, uint32_t t_o, int c0, int c1, int warp_piece,
                                           int warp, int lane, float &m, float &l, float sl2)
{
    const int32_t n = part.last - part.first + 1;
    int32_t i = (int32_t)blockIdx.x - part.first;  // this subtree among those of its level
    const int64_t floats4 = a.piece / 4 * 32;
    auto place = [&](int32_t cta) {  // where the subtree whose first part is CTA cta's lies
        return ((int64_t)cta * 2 + (cta == part.first ? 1 : 0)) * (2 * a.quarters) + warp_piece;
    };
#pragma unroll 1
    for (int level = 0; (1 << level) < n; ++level, i >>= 1) {
        if ((i & 1) == 0 && ((i + 1) << level) >= n)
            continue;  // no right neighbour
        int32_t *const node = a.nodes + ((part.first + ((i & ~1) << level)) * kLevels + level) * 8 + warp;
        int32_t there = 0;
        if (lane == 0)
            there = ptx::ld_acquire(node);
        there = __shfl_sync(0xffffffffu, there, 0);
        if (!there) {
            const int64_t to = place(part.first + (i << level));
            a.part_ml[to * 32 + lane] = make_float2(m, l);
            float4 *const po = a.part_o + to * floats4 + lane;
#pragma unroll 1
            for (int c = c0; c < c1; c += 32) {
                float o[32];
                ptx::tmem_ld_32x32b_x32(t_o + (uint32_t)c, o);
                ptx::tmem_ld_wait(o);
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    po[(c - c0 + k) / 4 * 32] = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            }
            __threadfence();
            __syncwarp();
            if (lane == 0)
                there = atomicAdd(node, 1);
            there = __shfl_sync(0xffffffffu, there, 0);
            if (!there)
                return false;
        }
        __threadfence();
        __syncwarp();
        if (lane == 0)
            *node = 0;  // for the next call
        const int64_t from = place(part.first + ((i ^ 1) << level));
        const float2 ml = __ldcg(&a.part_ml[from * 32 + lane]);
        const float4 *const po = a.part_o + from * floats4 + lane;
        const float big = fmaxf(m, ml.x);
        const float f = m == -INFINITY ? 0.f : ptx::ex2((m - big) * sl2);
        const float h = ml.x == -INFINITY ? 0.f : ptx::ex2((ml.x - big) * sl2);
        const bool left = (i & 1) == 0;  // the sum's rounding does not depend on who joins: left child in the fma
        float4 y[8], next[8];  // the neighbour's 32 columns at hand, and the 32 behind them on their way
#pragma unroll
        for (int k = 0; k < 8; ++k)
            next[k] = __ldcg(&po[k * 32]);
#pragma unroll 1
        for (int c = c0; c < c1; c += 32) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                y[k] = next[k];
            if (c + 32 < c1) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    next[k] = __ldcg(&po[((c + 32 - c0) / 4 + k) * 32]);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t o[16];
                ptx::tmem_ld_32x32b_x16(t_o + (uint32_t)(c + 16 * half), o);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float own = __uint_as_float(o[k]);
                    const float4 &q = y[4 * half + k / 4];
                    const float other = k % 4 == 0 ? q.x : (k % 4 == 1 ? q.y : (k % 4 == 2 ? q.z : q.w));
                    o[k] = __float_as_uint(left ? fmaf(f, own, h * other) : fmaf(h, other, f * own));
                }
                ptx::tmem_st_32x32b_x16(t_o + (uint32_t)(c + 16 * half), o);
            }
        }
        ptx::tmem_st_wait();
        l = left ? fmaf(f, l, h * ml.y) : fmaf(h, ml.y, f * l);
        m = big;
    }
    return true;
}

// By all threads of a CTA at its end, after its failures are recorded: the last CTA publishes a failure and clears it for
// the next call, and with it the nodes, which parts that never came may have left.
__device__ __forceinline__ void publish(const AttendArgs &a, int threads)
{
    int32_t failed = 0;
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.status->finished, 1u) + 1u == gridDim.x) {
            __threadfence();
            failed = -abs(atomicExch(&a.status->current, (int32_t)WINO_OK));  // positive: an append's, already read
            if (failed && a.status->first == WINO_OK)
                a.status->first = failed;
            a.status->finished = 0;
        }
    }
    if (__syncthreads_or(failed))
        for (int x = (int)threadIdx.x; x < kMaxCtas * kLevels * 8; x += threads)
            a.nodes[x] = 0;
}

template <int DP, bool kBf16, bool kScaled>
__global__ void __launch_bounds__(kAttendThreads<kScaled>, 1)
    attend_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const AttendArgs a)
{
    using C = Config<DP, kScaled>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];  // swizzle atoms
    const uint32_t raw = ptx::smem_u32(smem_raw);
    const uint32_t sq = raw, ring = raw + 2 * C::kTileBytes;
    using SharedBlock = Shared<kScaled, C::kStages>;
    static_assert(sizeof(SharedBlock) <= C::kShared, "shared block must fit its reserve");
    static_assert(C::kSlots <= SharedBlock::kRing, "ring slots");
    SharedBlock &sh = *reinterpret_cast<SharedBlock *>(smem_raw + 2 * C::kTileBytes + C::kRing);
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    auto full = [&](int s) { return ptx::smem_u32(&sh.full[s]); };
    auto empty = [&](int s) { return ptx::smem_u32(&sh.empty[s]); };
    auto zeroed = [&](int s) { return ptx::smem_u32(&sh.zeroed[s]); };
    auto s_full = [&](int g) { return ptx::smem_u32(&sh.s_full[g]); };
    auto p_ready = [&](int g) { return ptx::smem_u32(&sh.p_ready[g]); };
    auto s_free = [&](int g) { return ptx::smem_u32(&sh.s_free[g]); };
    auto p_half = [&](int g) { return ptx::smem_u32(&sh.p_half[g]); };
    auto o_done = [&](int g) { return ptx::smem_u32(&sh.o_done[g]); };
    auto part_full = [&](int s) { return ptx::smem_u32(&sh.part_full[s]); };
    auto part_empty = [&](int s) { return ptx::smem_u32(&sh.part_empty[s]); };
    const uint32_t q_full = ptx::smem_u32(&sh.q_full), q_empty = ptx::smem_u32(&sh.q_empty);
    const uint32_t ml_ready = ptx::smem_u32(&sh.ml_ready), ml_done = ptx::smem_u32(&sh.ml_done);
    const uint32_t mma_done = ptx::smem_u32(&sh.mma_done);
    auto slot_addr = [&](int s) { return ring + (uint32_t)s * C::kTileBytes; };
    auto stage_full = [&](int s) { return ptx::smem_u32(&sh.stage_full[s]); };
    auto stage_free = [&](int s) { return ptx::smem_u32(&sh.stage_free[s]); };
    constexpr uint32_t kStage0 = (2 + C::kSlots) * C::kTileBytes;  // where the stages start

    if (threadIdx.x == 0) {
        for (int s = 0; s < kParts; ++s) {
            ptx::mbar_init(part_full(s), 1);
            ptx::mbar_init(part_empty(s), kScaled ? 15 : 11);  // 8 softmax warps, 2 for the copies, MMAs, 4 for codes
        }
        ptx::mbar_init(q_full, 1);
        ptx::mbar_init(q_empty, 1);
        for (int s = 0; s < C::kSlots; ++s) {
            ptx::mbar_init(full(s), kScaled ? 4 : 1);
            ptx::mbar_init(empty(s), 1);
            if (!kScaled)
                ptx::mbar_init(zeroed(s), 1);
        }
        for (int s = 0; s < 2 * C::kStages; ++s) {
            ptx::mbar_init(stage_full(s), 1);
            ptx::mbar_init(stage_free(s), 4);
        }
        for (int g = 0; g < 2; ++g) {
            ptx::mbar_init(s_full(g), 1);
            ptx::mbar_init(s_free(g), 4);
            ptx::mbar_init(p_half(g), 4);
            ptx::mbar_init(p_ready(g), 4);
            ptx::mbar_init(o_done(g), 1);
        }
        for (int k = 0; k < 4; ++k)
            ptx::mbar_init(ptx::smem_u32(&sh.lead[k]), 1);
        ptx::mbar_init(ml_ready, 8);
        ptx::mbar_init(ml_done, 8);
        ptx::mbar_init(mma_done, 1);
        sh.abort = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kWarpK && lane == 0) {
        ptx::prefetch_tensormap(&tmQ);
        ptx::prefetch_tensormap(&tmK);
        ptx::prefetch_tensormap(&tmV);
    }
    if (warp == kWarpMma) {
        ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), kTmemAll);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = sh.tmem;
    ptx::grid_dep_launch_dependents();
    ptx::grid_dep_wait();  // lengths, pages, q and the cache may come from the kernel before
    bool ok = true;
    PartReader reader;
    // the next part; false after the last one or an abort.  done_with() gives its place back.
    auto next_part = [&]() -> bool {
        if (!wait_bounded(part_full(reader.slot()), reader.parity(), &sh.abort))
            return false;
        return (sh.parts[reader.slot()].flags & kEnd) == 0;
    };
    auto done_with = [&]() {  // by one lane, after the warp's reads
        ptx::mbar_arrive(part_empty(reader.slot()));
    };

    // A softmax thread holds its row of S: the launch's 384 x 168 registers are split 208 / 88, its 512 x 128 with codes
    // 184 / 72 / 72.
    if (warp < 8) {
        // ------------------------------------------------------------ softmax: one thread per row
        ptx::regs_inc<kScaled ? 184 : 208>();
        const int g = warp >> 2;               // warpgroup
        const int r = (warp & 3) * 32 + lane;  // row of the tile, its TMEM lane
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = lanes + C::kTmemS + (uint32_t)g * kTileN;
        const uint32_t t_p = lanes + C::kTmemP + (uint32_t)g * C::kStrideP;
        const int pos_in_tile = r / a.group;
        const float sl2 = a.scale_log2;
        constexpr float kTop = kTopBits[kBf16];
        const float rescale = fminf(kRescaleBits[kBf16] / sl2, FLT_MAX);  // the growth that m does not follow, in units of S
        uint32_t done = 0;   // slot tiles of this warpgroup so far
        uint32_t joins = 0;  // joined parts so far
        uint32_t leads = 0;  // parts with both row tiles so far
        while (__all_sync(0xffffffffu, next_part())) {
            const Part &part = sh.parts[reader.slot()];
            const bool two = (part.flags & kTwo) != 0;
            const int32_t n = part.n;
            const int32_t i = part.i0 + (two ? g : 0) * a.positions + pos_in_tile;  // row of the sequence
            const bool valid = pos_in_tile < a.positions && i < part.q.n;
            int32_t lim = 0, hole = -1;  // what the row sees, from the current tile's first slot on
            if (valid) {
                const RowSees sees = row_sees(a.b, part.q, i);
                lim = sees.lim;
                hole = sees.hole;
            }
            const bool any = __any_sync(0xffffffffu, valid);
            float m = -INFINITY, l = 0.f;  // m in units of S
            bool far = false;              // of any of the warp's rows
            const int32_t step = two ? 1 : 2, first = two ? 0 : g;
            lim -= (part.j0 + first) * kTileN;
            hole -= (part.j0 + first) * kTileN;
            int32_t t = first;
            bool good = true;
            for (; t < n; t += step, lim -= step * kTileN, hole -= step * kTileN) {
                if (!(good = warp_wait(s_full(g), done & 1u, &sh.abort)))
                    break;
                if (C::kEarly && two && g == 1 && t == 0 &&
                    !(good = warp_wait(ptx::smem_u32(&sh.lead[warp & 3]), leads & 1u, &sh.abort)))
                    break;
                if (any) {
                    ptx::tc_fence_after();
                    float x[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        ptx::tmem_ld_32x32b_x32(t_s + 32 * c, x[c]);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        ptx::tmem_ld_wait(x[c]);
                    if (C::kEarly) {  // S is free for the next tile's scores
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0)
                            ptx::mbar_arrive(s_free(g));
                    }
                    if (__any_sync(0xffffffffu, valid && (lim < kTileN || (hole >= 0 && hole < kTileN)))) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {  // bit k: the row sees column 32 c + k
                            const int here = lim - 32 * c, not_here = hole - 32 * c;
                            uint32_t seen = here >= 32 ? 0xffffffffu : (here > 0 ? (1u << here) - 1u : 0u);
                            if (not_here >= 0 && not_here < 32)
                                seen &= ~(1u << not_here);
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if ((seen & (1u << k)) == 0)
                                    x[c][k] = -INFINITY;
                        }
                    }
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        y[k] = ptx::max3(x[0][k], x[0][k + 8], x[0][k + 16]);
                        y[k] = ptx::max3(y[k], x[0][k + 24], x[1][k]);
                        y[k] = ptx::max3(y[k], x[1][k + 8], x[1][k + 16]);
                        y[k] = ptx::max3(y[k], x[1][k + 24], x[2][k]);
                        y[k] = ptx::max3(y[k], x[2][k + 8], x[2][k + 16]);
                        y[k] = ptx::max3(y[k], x[2][k + 24], x[3][k]);
                        y[k] = ptx::max3(y[k], x[3][k + 8], x[3][k + 16]);
                        y[k] = fmaxf(y[k], x[3][k + 24]);
                    }
                    const float mx = ptx::max3(ptx::max3(y[0], y[1], y[2]), ptx::max3(y[3], y[4], y[5]), fmaxf(y[6], y[7]));
                    const bool grow = mx - m > rescale;  // the difference is exact where it is close
                    if (__any_sync(0xffffffffu, grow)) {
                        if (t != first) {
                            // the O of earlier tiles is scaled to the new maximum; P V of the tile before is done first
                            if (!(good = warp_wait(o_done(g), (done - 1u) & 1u, &sh.abort)))
                                break;
                            ptx::tc_fence_after();
                            const float f = (grow && m != -INFINITY) ? ptx::ex2((m - mx) * sl2) : 1.f;
                            l *= f;
#pragma unroll 1
                            for (int c = 0; c < DP; c += 16) {
                                uint32_t o[16];
                                ptx::tmem_ld_32x32b_x16(lanes + C::kTmemO + (uint32_t)(g * DP + c), o);
                                ptx::tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 16; ++k)
                                    o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                                ptx::tmem_st_32x32b_x16(lanes + C::kTmemO + (uint32_t)(g * DP + c), o);
                            }
                        }
                        if (grow)
                            m = mx;
                        // a row that no head uses has whatever lay in shared memory for its query
                        far = __any_sync(0xffffffffu, valid && m != -INFINITY && fabsf(m * sl2) >= kFarBits);
                    }
                    // Where some row's m sl2 is far from zero its rounding would show in P, all of it from 2^24 on: the differences
                    // are formed first there, which are exact near the maximum.
                    float neg = m == -INFINITY ? 0.f : fmaf(-m, sl2, kTop);
                    if (__builtin_expect(far, 0)) {
                        const float base = m == -INFINITY ? 0.f : -m;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int k = 0; k < 32; k += 2) {
                                const float2 d = ptx::add2(make_float2(x[c][k], x[c][k + 1]), make_float2(base, base));
                                x[c][k] = d.x;
                                x[c][k + 1] = d.y;
                            }
                        neg = kTop;
                    }
                    const float2 s2 = make_float2(sl2, sl2), n2 = make_float2(neg, neg);
                    float2 l0 = make_float2(0.f, 0.f), l1 = l0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t p[16];
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            float2 u = ptx::fma2(make_float2(x[c][k], x[c][k + 1]), s2, n2);
                            float2 v = ptx::fma2(make_float2(x[c][k + 2], x[c][k + 3]), s2, n2);
                            u = make_float2(ptx::ex2(u.x), ptx::ex2(u.y));
                            v = make_float2(ptx::ex2(v.x), ptx::ex2(v.y));
                            l0 = ptx::add2(l0, u);
                            l1 = ptx::add2(l1, v);
                            p[k / 2] = pack2<kBf16>(u.x, u.y);
                            p[k / 2 + 1] = pack2<kBf16>(v.x, v.y);
                        }
                        if (C::kEarly && c == 1 && two && g == 0 && t == 0 && lane == 0)
                            ptx::mbar_arrive(ptx::smem_u32(&sh.lead[warp & 3]));
                        if (C::kEarly && c == 0 && t != first) {  // P's columns are free: P V of the tile before is done
                            if (!(good = warp_wait(o_done(g), (done - 1u) & 1u, &sh.abort)))
                                break;
                            ptx::tc_fence_after();
                        }
                        if (!C::kEarly && c == 2) {  // the first 64 slots' weights are in place: their half of P V starts
                            ptx::tmem_st_wait();
                            ptx::tc_fence_before();
                            __syncwarp();
                            if (lane == 0)
                                ptx::mbar_arrive(p_half(g));
                        }
                        ptx::tmem_st_32x32b_x16(t_p + 16 * c, p);
                    }
                    if (!good)
                        break;
                    l += (l0.x + l0.y) + (l1.x + l1.y);
                    ptx::tmem_st_wait();
                } else {
                    // A warp without rows arrives as the others do, and no tile ahead of them: with S free early that takes
                    // the wait for P V of the tile before.
                    if (C::kEarly && t != first && !(good = warp_wait(o_done(g), (done - 1u) & 1u, &sh.abort)))
                        break;
                    if (lane == 0)
                        ptx::mbar_arrive(C::kEarly ? s_free(g) : p_half(g));
                    if (C::kEarly && two && g == 0 && t == 0 && lane == 0)
                        ptx::mbar_arrive(ptx::smem_u32(&sh.lead[warp & 3]));
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    ptx::mbar_arrive(p_ready(g));
                ++done;
            }
            if (!good)
                break;
            leads += C::kEarly && two && n > 0 ? 1u : 0u;
            if (n > first) {  // this warpgroup had slot tiles
                if (!warp_wait(o_done(g), (done - 1u) & 1u, &sh.abort))
                    break;
                ptx::tc_fence_after();
            }
            // Columns [c0, c1) of O, as f0 O_0 + f1 O_1 where two warpgroups join.
            float f0 = 1.f, f1 = 0.f;
            float big = m, sum = l;
            int c0 = 0, c1 = DP;
            if (!two) {
                sh.ml[g][r] = make_float2(m, l);
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    ptx::mbar_arrive(ml_ready);
                if (!warp_wait(ml_ready, joins & 1u, &sh.abort))
                    break;
                ptx::tc_fence_after();
                const float2 m0 = sh.ml[0][r], m1 = sh.ml[1][r];
                big = fmaxf(m0.x, m1.x);
                f0 = m0.x == -INFINITY ? 0.f : ptx::ex2((m0.x - big) * sl2);
                f1 = m1.x == -INFINITY ? 0.f : ptx::ex2((m1.x - big) * sl2);
                sum = m0.y * f0 + m1.y * f1;
                c0 = g * (DP / 2);
                c1 = c0 + DP / 2;
            }
            if constexpr (kScaled) {  // what the converting warps found of the part is there: its last tile has been used
                const int2 nan = *reinterpret_cast<const int2 *>(sh.nan[reader.slot()]);
                if (__builtin_expect(nan.x != kNoSlot, 0) && valid) {
                    const RowSees sees = row_sees(a.b, part.q, i);
                    if ((nan.x < sees.lim && nan.x != sees.hole) || (nan.y < sees.lim && nan.y != sees.hole))
                        sum = NAN;
                }
            }
            if (any) {
                const uint32_t t_o = lanes + C::kTmemO + (uint32_t)(two ? g * DP : 0);
                bool mine = true;  // this warp ends the task
                if ((part.flags & kWhole) == 0) {
                    if (!two) {  // O_0 becomes the joined O, in this warpgroup's columns
#pragma unroll 1
                        for (int c = c0; c < c1; c += 16) {
                            uint32_t o[16], o1[16];
                            ptx::tmem_ld_32x32b_x16(t_o + (uint32_t)c, o);
                            if (n > 1)
                                ptx::tmem_ld_32x32b_x16(t_o + (uint32_t)(DP + c), o1);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                const float y = __uint_as_float(o[k]) * f0;
                                o[k] = __float_as_uint(n > 1 ? fmaf(f1, __uint_as_float(o1[k]), y) : y);
                            }
                            ptx::tmem_st_32x32b_x16(t_o + (uint32_t)c, o);
                        }
                        ptx::tmem_st_wait();
                        f0 = 1.f;
                        f1 = 0.f;
                    }
                    mine = join_parts(a, part, t_o, c0, c1, g * a.quarters + (warp & 3), warp, lane, big, sum, sl2);
                }
                if (mine) {  // no slot seen: zeros; NaN stays NaN
                    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
                    f0 *= inv;
                    f1 *= inv;
                    const bool both = !two && n > 1 && (part.flags & kWhole) != 0;
                    const int head = part.kv_head * a.group + (r - pos_in_tile * a.group);
                    uint16_t *const dst =
                        a.out.data + (int64_t)(part.q.start + i) * a.out.row_stride + (int64_t)head * a.out.head_stride;
#pragma unroll 1
                    for (int c = c0; c < c1; c += 32) {
                        float o[32];
                        if (n > 0) {
                            ptx::tmem_ld_32x32b_x32(t_o + (uint32_t)c, o);
                            if (both) {
                                float o1[32];
                                ptx::tmem_ld_32x32b_x32(t_o + (uint32_t)(DP + c), o1);
                                ptx::tmem_ld_wait(o);
                                ptx::tmem_ld_wait(o1);
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    o[k] = fmaf(f1, o1[k], f0 * o[k]);
                            } else {
                                ptx::tmem_ld_wait(o);
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    o[k] *= f0;
                            }
                        } else {
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                o[k] = 0.f;
                        }
                        if (valid) {
                            // A store covers 32 rows: 32 bytes of each where the rows are aligned for that, else 16.
                            uint32_t y[16];
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                y[k] = pack2<kBf16>(o[2 * k], o[2 * k + 1]);
#pragma unroll
                            for (int k = 0; k < 16; k += 8) {
                                uint16_t *const at = dst + c + 2 * k;
                                if (a.wide_rows && c + 2 * k + 16 <= a.b.head_dim) {
                                    ptx::st_global_v8(at, &y[k]);
                                } else {
                                    if (c + 2 * k < a.b.head_dim)
                                        *reinterpret_cast<uint4 *>(at) = make_uint4(y[k], y[k + 1], y[k + 2], y[k + 3]);
                                    if (c + 2 * k + 8 < a.b.head_dim)
                                        *reinterpret_cast<uint4 *>(at + 8) = make_uint4(y[k + 4], y[k + 5], y[k + 6], y[k + 7]);
                                }
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            __syncwarp();
            if (lane == 0)
                done_with();
            ++reader.count;
            if (!two) {  // both have read both accumulators and (m, l)
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    ptx::mbar_arrive(ml_done);
                if (!warp_wait(ml_done, joins & 1u, &sh.abort))
                    break;
                ++joins;
            }
        }
    } else if (!kScaled || warp < kWarpDecode) {
        ptx::regs_dec<kScaled ? 72 : 88>();
        if (warp == kWarpPlan) {
            if (a.wide)
                plan<uint64_t, SharedBlock, 2, kScaled>(a, sh, lane);
            else
                plan<uint32_t, SharedBlock, 2, kScaled>(a, sh, lane);
        } else if (warp == kWarpK || warp == kWarpV) {
            // -------------------------------------------------------- copies of Q and K, and of V
            // The issue of small boxes bounds a warp (68 clocks per box of 16 slots x 64 dims from 16 lanes, 174 from one
            // lane; two warps 39), so there are two, each with a ring of its own.
            constexpr int kHalves = DP / 64;
            const bool is_v = warp == kWarpV;
            const CUtensorMap *const map = is_v ? &tmV : &tmK;
            constexpr int kOfK = kScaled ? C::kStages : C::kSlotsK, kOfBoth = kScaled ? 2 * C::kStages : C::kSlots;
            const int slot0 = is_v ? kOfK : 0, slot1 = is_v ? kOfBoth : kOfK;
            int slot = slot0;  // the next to fill, and its phase
            uint32_t phase = 0;
            uint32_t issued = 0;  // slots filled so far
            uint32_t parts = 0;   // parts whose Q was loaded
            bool aborted = false;
            const int halves = a.joint ? 1 : kHalves;             // copies per page
            const int box = lane / halves, half = lane % halves;  // this lane's copy of a slot tile
            while (!aborted && __all_sync(0xffffffffu, next_part())) {
                const Part part = sh.parts[reader.slot()];
                __syncwarp();
                if (lane == 0)
                    done_with();
                ++reader.count;
                const int32_t n = part.n;
                if (n == 0)
                    continue;
                const bool two = (part.flags & kTwo) != 0;
                // Page numbers: 32 consecutive table entries in the lanes, and the 32 behind them on their way.  They are
                // checked where they are used, so that nothing waits for a load before that.
                const int32_t last_entry = page_entry(a, part.kv_end - 1);
                int32_t window = page_entry(a, part.j0 * kTileN);  // first entry of `near`
                const int32_t *const table = a.b.page_table + (int64_t)part.seq * a.b.table_width;
                auto entries = [&](int32_t e0) { return e0 + lane <= last_entry ? table[e0 + lane] : 0; };
                int32_t near = entries(window), ahead = entries(window + 32);
                if (!is_v) {  // Q: the part's one or two tiles
                    if (!warp_wait(q_empty, (parts & 1u) ^ 1u, &sh.abort)) {
                        aborted = true;
                        break;
                    }
                    if (lane == 0)
                        ptx::mbar_arrive_expect_tx(q_full,
                                                   (uint32_t)(two ? 2 : 1) * kHalves * (uint32_t)(a.positions * a.group) * 128u);
                    __syncwarp();
                    if (lane < kHalves * (two ? 2 : 1)) {
                        const int tile = lane / kHalves, h = lane % kHalves;
                        ptx::tma_load_3d(sq + (uint32_t)tile * C::kTileBytes + (uint32_t)h * kHalfBytes, &tmQ, q_full, h * 64,
                                         part.kv_head * a.group, part.q.start + part.i0 + tile * a.positions);
                    }
                    ++parts;
                }
                if constexpr (kScaled) {
                    // codes and scales, a box and an untiled copy per page
                    const int32_t box_rows = a.box_rows;
                    for (int32_t x = 0; x < n; ++x) {
                        const int32_t first = part.j0 * kTileN + x * kTileN;
                        const int32_t boxes = min(a.boxes, (part.kv_end - first + box_rows - 1) / box_rows);
                        const int32_t at = first + lane * box_rows;
                        const int32_t entry = page_entry(a, at);
                        if (page_entry(a, first + boxes * box_rows - 1) - window >= 32) {  // no stage straddles the border
                            near = ahead;
                            window += 32;
                            ahead = entries(window + 32);
                        }
                        int32_t page = __shfl_sync(0xffffffffu, near, (entry - window) & 31);
                        if ((uint32_t)page >= (uint32_t)a.b.n_pages) {
                            ok = ok && lane >= boxes;
                            page = -1;  // a bad entry: behind the cache, read as zeros
                        }
                        if (!warp_wait(stage_free(slot), phase ^ 1u, &sh.abort)) {
                            aborted = true;
                            break;
                        }
                        if (lane == 0)
                            ptx::mbar_arrive_expect_tx(stage_full(slot), (uint32_t)(boxes * box_rows) * (DP + 1u));
                        __syncwarp();
                        if (lane < boxes) {
                            const int32_t in_page = at - entry * a.b.page_size;
                            ptx::tma_load_4d(raw + kStage0 + (uint32_t)slot * C::kStageBytes + (uint32_t)(lane * box_rows) * DP, map,
                                             stage_full(slot), 0, in_page, part.kv_head, page < 0 ? a.end : page);
                            ptx::bulk_load(ptx::smem_u32(&sh.scale[slot][lane * box_rows]),
                                           (is_v ? a.scales.v_scale : a.scales.k_scale) +
                                               scale_at(a.b, max(page, 0), in_page, part.kv_head),
                                           (uint32_t)box_rows, stage_full(slot));
                        }
                        __syncwarp();
                        ++issued;
                        if (++slot == slot1) {
                            slot = slot0;
                            phase ^= 1u;
                        }
                    }
                } else {
                    for (int32_t t = 0; t < n; ++t) {
                        const int32_t first = (part.j0 + t) * kTileN;
                        const int32_t boxes = min(a.boxes, (part.kv_end - first + a.box_rows - 1) / a.box_rows);
                        const int32_t at = first + box * a.box_rows;  // this lane's first slot
                        const int32_t entry = page_entry(a, at);
                        if (page_entry(a, first + boxes * a.box_rows - 1) - window >= 32) {  // no tile straddles the border
                            near = ahead;
                            window += 32;
                            ahead = entries(window + 32);
                        }
                        int32_t page = __shfl_sync(0xffffffffu, near, (entry - window) & 31);
                        if ((uint32_t)page >= (uint32_t)a.b.n_pages) {
                            ok = ok && box >= boxes;
                            page = -1;  // a bad entry: behind the cache, read as zeros
                        }
                        if (!warp_wait(empty(slot), phase ^ 1u, &sh.abort)) {
                            aborted = true;
                            break;
                        }
                        if (lane == 0)
                            ptx::mbar_arrive_expect_tx(full(slot), (uint32_t)(boxes * kHalves * a.box_rows) * 128u);
                        __syncwarp();
                        if (box < boxes) {
                            const uint32_t dst = slot_addr(slot) + (uint32_t)half * a.tile.half +
                                                 (uint32_t)(box * a.box_rows / 8) * a.tile.group;
                            const int32_t in_page = at - entry * a.b.page_size;
                            if (a.joint)
                                ptx::tma_load_5d(dst, map, full(slot), 0, 0, 0, in_page >> 3,
                                                 page < 0 ? a.end : page * a.joint + part.kv_head);
                            else
                                ptx::tma_load_4d(dst, map, full(slot), half * 64, in_page, part.kv_head, page < 0 ? a.end : page);
                        }
                        __syncwarp();
                        ++issued;
                        if (is_v && t == n - 1 && (part.flags & kTail) != 0) {
                            // V of slots that no row sees may be anything, and P = 0 times NaN is not 0: zeros
                            if (!warp_wait(full(slot), phase, &sh.abort)) {
                                aborted = true;
                                break;
                            }
                            uint8_t *const v = smem_raw + (slot_addr(slot) - raw);
                            for (int x = (part.kv_end & (kTileN - 1)) * 8 + lane; x < kTileN * 8; x += 32)
#pragma unroll
                                for (int h = 0; h < kHalves; ++h)  // 8 pieces of 16 bytes per row, 64 per group
                                    *reinterpret_cast<uint4 *>(v + (x >> 6) * a.tile.group + h * a.tile.half + (x & 63) * 16) =
                                        make_uint4(0, 0, 0, 0);
                            ptx::fence_proxy_async();
                            __syncwarp();
                            if (lane == 0)
                                ptx::mbar_arrive(zeroed(slot));
                        }
                        if (++slot == slot1) {
                            slot = slot0;
                            phase ^= 1u;
                        }
                    }
                }
            }
            // All copies issued land before the shared memory goes away.  In a call that went well their readers waited for
            // them, and each wait is one try.  Where any role gave up, this one may already be behind its last part.
            if (lane == 0) {
                if (parts > 0)
                    wait_drain(q_full, (parts - 1) & 1u);
                const uint32_t slots = (uint32_t)(slot1 - slot0);
                for (uint32_t s = 0; s < slots && s < issued; ++s)
                    wait_drain(kScaled ? stage_full(slot0 + (int)s) : full(slot0 + (int)s), last_parity(issued, s, slots));
            }
            __syncwarp();
        } else if (warp == kWarpMma) {
            // -------------------------------------------------------- MMAs, issued by one thread
            if (ptx::elect_one()) {
                const uint32_t id_s = ptx::idesc_f16_f32(kTileM, kTileN, kBf16, false);
                const uint32_t id_o = ptx::idesc_f16_f32(kTileM, DP, kBf16, true);
                int k_slot = 0, v_slot = C::kSlotsK;  // the next ring slots, and their phases; with codes v_slot for both
                uint32_t k_phase = 0, v_phase = 0;
                uint32_t parts = 0;
                uint32_t zero_phases = 0;  // bit s: phase of zeroed(s)
                uint32_t n_p0 = 0, n_p1 = 0;  // slot tiles of each warpgroup whose weights were taken
                uint32_t n_s0 = 0, n_s1 = 0;  // and whose scores were issued
                bool aborted = false;
                auto scores = [&](int g, int qt, int ks) -> bool {  // S_g = Q_qt K^T
                    if (C::kEarly) {
                        uint32_t &count = g ? n_s1 : n_s0;
                        if (!wait_bounded(s_free(g), (count++ & 1u) ^ 1u, &sh.abort))
                            return false;
                        ptx::tc_fence_after();
                    }
                    const uint64_t da = ptx::sdesc_kmajor_sw128(sq + (uint32_t)qt * C::kTileBytes);
                    const uint64_t db = ptx::sdesc_kmajor_sw128(slot_addr(ks), a.tile.group);
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
                        ptx::mma_bf16(tmem + C::kTmemS + (uint32_t)g * kTileN,
                                      da + (uint64_t)((k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2),
                                      db + (uint64_t)((k >> 2) * (a.tile.half >> 4) + (k & 3) * 2), id_s, k != 0);
                    ptx::mma_commit(s_full(g));
                    return true;
                };
                // O_g (+)= P_g V.  Where the next scores wait for it, each half of the slots as soon as its weights are in
                // tensor memory.  zeros: V's slots behind the last one are zeroed first.
                auto values = [&](int g, int vs, bool add, bool zeros) -> bool {
                    const uint64_t db = ptx::sdesc_mnmajor_sw128(slot_addr(vs), a.tile.half, a.tile.group);
                    uint32_t &count = g ? n_p1 : n_p0;
                    const uint32_t parity = count++ & 1u;
#pragma unroll
                    for (int k = 0; k < kTileN / 16; ++k) {
                        if (k == 0) {
                            if (!wait_bounded(C::kEarly ? p_ready(g) : p_half(g), parity, &sh.abort) ||
                                (!kScaled && zeros && !wait_bounded(zeroed(vs), zero_phases >> vs & 1u, &sh.abort)))
                                return false;
                            ptx::tc_fence_after();
                        }
                        if (!C::kEarly && k == kTileN / 32) {
                            if (!wait_bounded(p_ready(g), parity, &sh.abort))
                                return false;
                            ptx::tc_fence_after();
                        }
                        ptx::mma_f16_ts(tmem + C::kTmemO + (uint32_t)(g * DP),
                                        tmem + C::kTmemP + (uint32_t)g * C::kStrideP + (uint32_t)(k * 8),
                                        db + (uint64_t)(k * (a.tile.group >> 3)), id_o, (add || k != 0) ? 1u : 0u);
                    }
                    ptx::mma_commit(o_done(g));
                    return true;
                };
                auto take = [&](int &s, uint32_t &parity) {
                    s = v_slot;
                    parity = v_phase;
                    if (++v_slot == C::kSlots) {
                        v_slot = 0;
                        v_phase ^= 1u;
                    }
                };
                while (!aborted && next_part()) {
                    const int32_t n = sh.parts[reader.slot()].n, flags = sh.parts[reader.slot()].flags;
                    done_with();
                    ++reader.count;
                    if (n == 0)
                        continue;
                    const bool two = (flags & kTwo) != 0;
                    const int lead = two ? 1 : 2;
                    if (!wait_bounded(q_full, parts & 1u, &sh.abort)) {
                        aborted = true;
                        break;
                    }
                    ++parts;
                    // Scores run `lead` tiles ahead of the values.  With S free early, both tiles' scores go out before the
                    // values; without, each warpgroup's scores behind its own values, which free S.
                    for (int32_t t = -lead; t < n; ++t) {
                        const int g = two ? 0 : (t & 1);
                        const bool v_now = t >= 0, k_now = t + lead < n;
                        const bool zeros = t == n - 1 && (flags & kTail) != 0;
                        int vs = v_slot, ks = k_slot;
                        uint32_t v_par = v_phase, k_par = k_phase;
                        if constexpr (kScaled) {  // one ring for both
                            if (C::kEarly && k_now)
                                take(ks, k_par);
                            if (v_now)
                                take(vs, v_par);
                            if (!C::kEarly && k_now)
                                take(ks, k_par);
                        }
                        bool good = true;
                        if (k_now && C::kEarly)
                            good = wait_bounded(full(ks), k_par, &sh.abort) && scores(g, 0, ks) && (!two || scores(1, 1, ks));
                        if (good && v_now) {
                            good = wait_bounded(full(vs), v_par, &sh.abort) && values(g, vs, t >= lead, zeros);
                            if (good && !two)
                                ptx::mma_commit(empty(vs));
                        }
                        if (good && k_now && !C::kEarly)
                            good = wait_bounded(full(ks), k_par, &sh.abort) && scores(g, 0, ks);
                        if (good && v_now && two) {
                            good = values(1, vs, t > 0, false);
                            if (good)
                                ptx::mma_commit(empty(vs));
                        }
                        if (good && k_now) {
                            if (two && !C::kEarly)
                                good = scores(1, 1, ks);
                            ptx::mma_commit(empty(ks));
                            if (t + lead == n - 1)
                                ptx::mma_commit(q_empty);
                        }
                        if (!good) {
                            aborted = true;
                            break;
                        }
                        if (zeros)
                            zero_phases ^= 1u << vs;
                        if (!kScaled && v_now && ++v_slot == C::kSlots) {
                            v_slot = C::kSlotsK;
                            v_phase ^= 1u;
                        }
                        if (!kScaled && k_now && ++k_slot == C::kSlotsK) {
                            k_slot = 0;
                            k_phase ^= 1u;
                        }
                    }
                }
                ptx::mma_commit(mma_done);  // nothing may still write tensor memory when it is released
                wait_drain(mma_done, 0);
            }
            __syncwarp();
        }
    } else if constexpr (kScaled) {
        // ------------------------------------------------------------ codes to values
        ptx::regs_dec<72>();
        constexpr int kChunks = DP / 16, kAtOnce = 32 / kChunks;  // chunks of 16 codes per slot, slots per turn of a warp
        constexpr int kHalfN = kTileN / 2, kTurns = 16 / kAtOnce;  // a warp's 16 slots of half a tile
        const int of_warp = (warp & 3) * 16 + lane / kChunks, chunk = lane % kChunks;
        const bool swap = chunk >= 4;  // which 8 of 16 values are written first: no two of 8 lanes meet in a bank
        int tile = 0, stage_k = 0, stage_v = 0;  // the next of each ring, and their phases
        uint32_t phase = 0, phase_k = 0, phase_v = 0;
        while (__all_sync(0xffffffffu, next_part())) {
            const Part &part = sh.parts[reader.slot()];
            // Tiles in the order in which the MMAs take them: the first scores' K, then K and V in turn, then the last V.
            const int32_t n = part.n, lead = min(n, (part.flags & kTwo) != 0 ? 1 : 2);
            const int32_t slots = part.kv_end - part.j0 * kTileN;  // from the part's first on
            int32_t *const nan = sh.nan[reader.slot()];
            __syncwarp();
            if (lane == 0)
                done_with();  // the softmax warps hold the part, and its `nan`, until its last tile has been used
            ++reader.count;
            bool good = true;
            int32_t next_k = 0, next_v = 0;
            while (good && next_v < n) {
                const bool is_v = next_k == n || (C::kEarly ? next_k - next_v > lead : next_k - next_v >= lead);
                int32_t left = slots - (is_v ? next_v : next_k) * kTileN;
                ++(is_v ? next_v : next_k);
                if (!(good = warp_wait(empty(tile), phase ^ 1u, &sh.abort)))
                    break;
                const int stage = is_v ? C::kStages + stage_v : stage_k;
                if (!(good = warp_wait(stage_full(stage), is_v ? phase_v : phase_k, &sh.abort)))
                    break;
                // A tile as TMA would write it: swizzled blocks of 64 dims, in which 16 bytes of row r lie at the place of
                // their number xor r % 8.
                uint8_t *const to = smem_raw + (slot_addr(tile) - raw) + (chunk >> 2) * kHalfBytes;
                const uint8_t *const codes = smem_raw + kStage0 + (uint32_t)stage * C::kStageBytes;
                uint32_t most = 0;  // of the scales
#pragma unroll 1
                for (int half = 0; half < 2; ++half, left -= kHalfN) {
                    uint4 c[kTurns];
                    uint32_t f[kTurns];
#pragma unroll
                    for (int k = 0; k < kTurns; ++k) {
                        c[k] = *reinterpret_cast<const uint4 *>(codes + (half * kHalfN + of_warp + k * kAtOnce) * DP + chunk * 16);
                        f[k] = sh.scale[stage][half * kHalfN + of_warp + k * kAtOnce];
                    }
                    if (left < kHalfN) {  // behind the last slot: zeros, which V needs
#pragma unroll
                        for (int k = 0; k < kTurns; ++k)
                            if (of_warp + k * kAtOnce >= left) {
                                c[k] = make_uint4(0, 0, 0, 0);
                                f[k] = 0;
                            }
                    }
#pragma unroll
                    for (int k = 0; k < kTurns; ++k) {
                        const int r = half * kHalfN + of_warp + k * kAtOnce;
                        const uint32_t factor = finite_factor<kBf16>(f[k]);
                        uint4 lo, hi;
                        decode4<kBf16>(c[k].x, factor, lo.x, lo.y);
                        decode4<kBf16>(c[k].y, factor, lo.z, lo.w);
                        decode4<kBf16>(c[k].z, factor, hi.x, hi.y);
                        decode4<kBf16>(c[k].w, factor, hi.z, hi.w);
                        const int at = ((chunk & 3) * 2) ^ (r & 7);
                        *reinterpret_cast<uint4 *>(to + r * 128 + (swap ? at ^ 1 : at) * 16) = swap ? hi : lo;
                        *reinterpret_cast<uint4 *>(to + r * 128 + (swap ? at : at ^ 1) * 16) = swap ? lo : hi;
                    }
#pragma unroll
                    for (int k = 0; k < kTurns; ++k)
                        most = max(most, f[k]);
                }
                if (__builtin_expect(__any_sync(0xffffffffu, most == kScaleNan), 0)) {
                    // a slot of the warp's 16 of each half per lane
                    const int r = (lane >> 4) * kHalfN + (warp & 3) * 16 + (lane & 15);
                    if (r < left + kTileN && sh.scale[stage][r] == kScaleNan) {
                        const int32_t slot = part.kv_end - left - kTileN + r, least = atomicMin(&nan[0], slot);
                        if (slot != least)
                            atomicMin(&nan[1], max(slot, least));
                    }
                    __syncwarp();
                }
                ptx::fence_proxy_async();
                __syncwarp();
                // The stage is given back once its values have been used, not once they have been asked for: a copy was seen to
                // overtake reads that were still on their way.
                if (lane == 0) {
                    ptx::mbar_arrive(full(tile));
                    ptx::mbar_arrive(stage_free(stage));
                }
                if (++tile == C::kSlots) {
                    tile = 0;
                    phase ^= 1u;
                }
                int &s = is_v ? stage_v : stage_k;
                if (++s == C::kStages) {
                    s = 0;
                    (is_v ? phase_v : phase_k) ^= 1u;
                }
            }
            if (!good)
                break;
        }
    }
    if (!ok)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_ARG);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == kWarpMma)
        ptx::tmem_dealloc(tmem, kTmemAll);
    if (threadIdx.x == 0 && sh.abort)
        atomicExch(&a.status->current, (int32_t)WINO_ERR_DEVICE_TIMEOUT);
    publish(a, kAttendThreads<kScaled>);
}

template <int DP, bool kBf16, bool kScaled>
int launch(const CUtensorMap &tq, const CUtensorMap &tk, const CUtensorMap &tv, const AttendArgs &a, int ctas,
           cudaStream_t stream)
{
    static std::mutex mu;
    static bool done[64];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64)
        return WINO_ERR_CUDA;
    {
        std::lock_guard<std::mutex> g(mu);
        if (!done[dev]) {
            if (cudaFuncSetAttribute(attend_kernel<DP, kBf16, kScaled>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)Config<DP, kScaled>::kSmem) != cudaSuccess)
                return WINO_ERR_CUDA;
            done[dev] = true;
        }
    }
    static_assert(Config<DP, kScaled>::kSmem <= kSmemLimit, "shared memory");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kAttendThreads<kScaled>);
    cfg.dynamicSmemBytes = Config<DP, kScaled>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, attend_kernel<DP, kBf16, kScaled>, tq, tk, tv, a) != cudaSuccess)
        return WINO_ERR_CUDA;
    return WINO_OK;
}

// What both calls give the kernel (attend.cu): the arguments but for the cache's layout, and the map of Q.
int attend_args(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b, uint8_t *scratch,
                StatusWords *status, AttendArgs *a, CUtensorMap *tq);

// A tensor map over an 8-bit cache's codes (attend_scaled.cu): boxes of box_rows slots of one head and page, `width` (64 or 128)
// bytes wide, as they are or swizzled by that width.
int encode_codes(CUtensorMap *m, const void *cache, const wino_kv_batch &b, int32_t width, int32_t box_rows, bool swizzled);

// Few rows per sequence over an 8-bit cache (attend_few.cu): whether a batch is of that kind, and its launch with the arguments
// of attend_args and the scales.
bool few_rows(const wino_kv_batch &b);
int launch_few(AttendArgs a, int ctas, cudaStream_t stream);

}  // namespace attend
}  // namespace wino
