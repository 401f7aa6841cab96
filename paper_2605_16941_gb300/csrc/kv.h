// kv.h -- declarations shared by the entry points and the kernels over a paged cache (not installed).
#pragma once

#include <cudaTypedefs.h>  // PFN_cuTensorMapEncodeTiled

#include "internal.h"

namespace wino {

// ---------------------------------------------------------------- host helpers of the entry points (wino_abi.cu)

struct DeviceInfo {
    int sm_count = 0;
    bool supported = false;
};
int device_info(DeviceInfo *out);  // of the current device; WINO_ERR_UNSUPPORTED on others than 10.3
PFN_cuTensorMapEncodeTiled_v12000 encode_fn();
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// wino_rope_append: rows' rotation and the cache's writes (rope.cu).
cudaError_t launch_rope_append(const wino_heads *q, const wino_heads *q_out, const wino_heads *k, const wino_heads *v,
                               const wino_kv_batch &b, const wino_rope &rope, StatusWords *status,
                               cudaStream_t stream);

// wino_attend (attend.cu): the bytes behind the status words that its kernel uses, the most work units that a batch may
// have (below 2^62), and its launch.
size_t attend_scratch_bytes(const wino_kv_batch &b);
double attend_units(const wino_kv_batch &b);
int launch_attend(const wino_heads &q, const wino_heads &out, float scale, const wino_kv_batch &b, uint8_t *scratch,
                  StatusWords *status, int sm_count, cudaStream_t stream);

}  // namespace wino
