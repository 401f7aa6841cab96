// kv_abi.cu -- the extern "C" entry points over a paged cache (see include/wino.h): host-side checks and launches.
#include <cmath>

#include "kv.h"
#include "trace.h"

namespace wino {
namespace {

constexpr size_t kStatusBytes = 256;
constexpr int64_t kMaxStride = int64_t(1) << 36;  // elements: byte strides stay inside a tensor map's 2^40
constexpr int kMaxSeqs = 16384;

int check_batch(const wino_kv_batch *b)
{
    if (!b)
        return WINO_ERR_ARG;
    if (!b->q_start || !b->q_len || !b->kv_len || !b->new_slot || !b->page_table || !b->k_cache || !b->v_cache)
        return WINO_ERR_ARG;
    if (!aligned(b->q_start, 4) || !aligned(b->q_len, 4) || !aligned(b->kv_len, 4) || !aligned(b->new_slot, 4) ||
        !aligned(b->page_table, 4) || !aligned(b->k_cache, 16) || !aligned(b->v_cache, 16))
        return WINO_ERR_ARG;
    if ((b->dtype != WINO_BF16 && b->dtype != WINO_FP16) || b->mask < WINO_MASK_FULL || b->mask > WINO_MASK_SHADOW)
        return WINO_ERR_ARG;
    if (b->n_seq < 1 || b->n_seq > kMaxSeqs || b->n_rows < 1 || b->n_rows > (1 << 24) || b->n_kv_heads < 1 ||
        b->n_kv_heads > 1024 || b->n_q_heads < b->n_kv_heads || b->n_q_heads % b->n_kv_heads != 0 ||
        b->n_q_heads / b->n_kv_heads > 128)
        return WINO_ERR_SHAPE;
    if (b->head_dim < 8 || b->head_dim > 128 || b->head_dim % 8 != 0)
        return WINO_ERR_SHAPE;
    if (b->page_size != 16 && b->page_size != 32 && b->page_size != 64 && (b->page_size < 128 || b->page_size % 128 != 0))
        return WINO_ERR_SHAPE;
    if (b->n_pages < 1 || b->table_width < 1 || (int64_t)b->table_width * b->page_size > (int64_t(1) << 30))
        return WINO_ERR_SHAPE;
    const int64_t st[3] = {b->page_stride, b->slot_stride, b->head_stride};
    const int64_t extent[3] = {b->n_pages, b->page_size, b->n_kv_heads};
    for (int i = 0; i < 3; ++i)
        if (extent[i] > 1 && (st[i] < b->head_dim || st[i] % 8 != 0 || st[i] > kMaxStride))
            return WINO_ERR_SHAPE;
    return WINO_OK;
}

int check_heads(const wino_heads *h, const wino_kv_batch &b, int32_t heads)
{
    if (!h || !h->data || !aligned(h->data, 16))
        return WINO_ERR_ARG;
    if (b.n_rows > 1 && (h->row_stride < b.head_dim || h->row_stride % 8 != 0 || h->row_stride > kMaxStride))
        return WINO_ERR_SHAPE;
    if (heads > 1 && (h->head_stride < b.head_dim || h->head_stride % 8 != 0 || h->head_stride > kMaxStride))
        return WINO_ERR_SHAPE;
    return WINO_OK;
}

}  // namespace
}  // namespace wino

using namespace wino;

extern "C" {

int wino_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double scale, int64_t trained_len,
                          double *freq, float *factor)
{
    if (!freq || !factor || !std::isfinite(base) || base <= 1.0)
        return WINO_ERR_ARG;
    if (scaling != WINO_ROPE_PLAIN && scaling != WINO_ROPE_LINEAR && scaling != WINO_ROPE_PARTS)
        return WINO_ERR_ARG;
    if (scaling != WINO_ROPE_PLAIN && (!std::isfinite(scale) || scale < 1.0))
        return WINO_ERR_ARG;
    if (scaling == WINO_ROPE_PARTS && trained_len < 1)
        return WINO_ERR_ARG;
    if (rot_dim < 0 || rot_dim > 128 || rot_dim % 2 != 0)
        return WINO_ERR_SHAPE;
    for (int32_t j = 0; j < rot_dim / 2; ++j) {
        const double f = std::pow(base, -2.0 * j / rot_dim);
        double g = f;
        if (scaling == WINO_ROPE_LINEAR) {
            g = f / scale;
        } else if (scaling == WINO_ROPE_PARTS) {
            const double turns = (double)trained_len * f / 6.283185307179586477;
            const double keep = std::fmin(1.0, std::fmax(0.0, (turns - 1.0) / (32.0 - 1.0)));
            g = f * keep + f / scale * (1.0 - keep);
        }
        freq[j] = g;
    }
    *factor = scaling == WINO_ROPE_PARTS ? (float)(0.1 * std::log(scale) + 1.0) : 1.f;
    return WINO_OK;
}

int wino_rope_append(const wino_heads *q, const wino_heads *q_out, const wino_heads *k, const wino_heads *v,
                     const wino_kv_batch *b, const wino_rope *rope, void *ws, void *stream)
{
    const Range range("wino_rope_append");
    if (!rope || !ws || !aligned(ws, kStatusBytes) || (q == nullptr) != (q_out == nullptr) ||
        (k == nullptr) != (v == nullptr) || (!q && !k))
        return WINO_ERR_ARG;
    int rc = check_batch(b);
    if (rc != WINO_OK)
        return rc;
    if (q && ((rc = check_heads(q, *b, b->n_q_heads)) != WINO_OK || (rc = check_heads(q_out, *b, b->n_q_heads)) != WINO_OK))
        return rc;
    if (k && ((rc = check_heads(k, *b, b->n_kv_heads)) != WINO_OK || (rc = check_heads(v, *b, b->n_kv_heads)) != WINO_OK))
        return rc;
    if (rope->rot_dim < 0 || rope->rot_dim > b->head_dim || rope->rot_dim % 2 != 0)
        return WINO_ERR_SHAPE;
    if ((rope->rot_dim > 0 && (!rope->freq || !aligned(rope->freq, 8))) || !aligned(rope->positions, 4) ||
        !std::isfinite(rope->factor))
        return WINO_ERR_ARG;
    // in place means the very same array: elements shared in any other way would be read after they were written
    if (q && q->data == q_out->data &&
        ((b->n_rows > 1 && q->row_stride != q_out->row_stride) || (b->n_q_heads > 1 && q->head_stride != q_out->head_stride)))
        return WINO_ERR_ARG;
    DeviceInfo info;
    if ((rc = device_info(&info)) != WINO_OK)
        return rc;
    return launch_rope_append(q, q_out, k, v, *b, *rope, static_cast<StatusWords *>(ws),
                              static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? WINO_OK
               : WINO_ERR_CUDA;
}

int wino_attend_workspace_size(const wino_kv_batch *b, size_t *bytes)
{
    if (!bytes)
        return WINO_ERR_ARG;
    const int rc = check_batch(b);
    if (rc != WINO_OK)
        return rc;
    *bytes = kStatusBytes + attend_scratch_bytes(*b);
    return WINO_OK;
}

int wino_attend(const wino_heads *q, const wino_heads *out, float scale, const wino_kv_batch *b, void *ws,
                size_t ws_bytes, void *stream)
{
    const Range range("wino_attend");
    // scale * log2(e) is a normal number: a subnormal counts as zero in the kernel, and zero times a masked -inf is NaN
    if (!ws || !aligned(ws, kStatusBytes) || !(scale >= 0x1p-126f) || !(scale < 0x1p127f))
        return WINO_ERR_ARG;
    int rc = check_batch(b);
    if (rc != WINO_OK)
        return rc;
    if ((rc = check_heads(q, *b, b->n_q_heads)) != WINO_OK || (rc = check_heads(out, *b, b->n_q_heads)) != WINO_OK)
        return rc;
    if (q->data == out->data)
        return WINO_ERR_ARG;
    if (attend_units(*b) >= 4611686018427387904.0)
        return WINO_ERR_SHAPE;
    if (ws_bytes < kStatusBytes + attend_scratch_bytes(*b))
        return WINO_ERR_WORKSPACE;
    DeviceInfo info;
    if ((rc = device_info(&info)) != WINO_OK)
        return rc;
    return launch_attend(*q, *out, scale, *b, static_cast<uint8_t *>(ws) + kStatusBytes, static_cast<StatusWords *>(ws),
                         info.sm_count, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
