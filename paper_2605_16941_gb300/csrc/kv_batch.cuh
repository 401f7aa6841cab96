// kv_batch.cuh -- the rows and slots of a wino_kv_batch as the device reads them: every value that comes from a device
// array is checked here before it becomes an address, and what fails is left out and recorded.
#pragma once

#include "kv.h"

namespace wino {

constexpr int32_t kMaxSlots = 1 << 30;  // table_width * page_size
constexpr int32_t kFarSlot = 1 << 30;   // new_slot is kept within +- this, which no table reaches

// One sequence.  n = 0 leaves it out.
struct SeqRows {
    int32_t start, n;  // rows [start, start + n)
    int32_t kv;        // slots that its rows see, before the shadow block's
    int32_t base;      // new_slot
    bool ok;           // false: an entry out of range
};

__device__ __forceinline__ SeqRows load_seq(const wino_kv_batch &b, int32_t s)
{
    SeqRows q;
    q.start = b.q_start[s];
    q.n = b.q_len[s];
    q.kv = b.kv_len[s];
    q.base = max(-kFarSlot, min(kFarSlot, b.new_slot[s]));
    const int32_t cap = b.table_width * b.page_size;  // at most kMaxSlots
    q.ok = q.n >= 0 && q.kv >= 0 && q.kv <= cap;
    if (q.n > 0) {
        q.ok = q.ok && q.start >= 0 && q.n <= b.n_rows && q.start <= b.n_rows - q.n;
        if (b.mask == WINO_MASK_SHADOW)
            q.ok = q.ok && (q.n & 1) == 0 && q.n / 2 <= cap - q.kv;
    }
    if (!q.ok)
        q.n = 0;
    return q;
}

// The slot at which row i is stored.
__device__ __forceinline__ int32_t row_slot(const wino_kv_batch &b, const SeqRows &q, int32_t i)
{
    const int32_t half = q.n >> 1;
    return (b.mask == WINO_MASK_SHADOW && i >= half) ? q.kv + (i - half) : q.base + i;
}

// What row i sees: the slots [0, lim) but for `hole` (-1: none).
struct RowSees {
    int32_t lim, hole;
};

__device__ __forceinline__ RowSees row_sees(const wino_kv_batch &b, const SeqRows &q, int32_t i)
{
    RowSees r{q.kv, -1};
    if (b.mask == WINO_MASK_CAUSAL) {
        r.lim = max(0, min(q.kv, q.base + i + 1));
    } else if (b.mask == WINO_MASK_SHADOW) {
        const int32_t half = q.n >> 1;
        if (i >= half) {
            r.lim = q.kv + half;
            r.hole = q.base + (i - half);
        }
    }
    return r;
}

// A row's page: the table's entry, or -1 and an error where it is out of range.
__device__ __forceinline__ int32_t load_page(const wino_kv_batch &b, int32_t s, int32_t entry, bool &ok)
{
    const int32_t p = b.page_table[(int64_t)s * b.table_width + entry];
    if (p >= 0 && p < b.n_pages)
        return p;
    ok = false;
    return -1;
}

}  // namespace wino
