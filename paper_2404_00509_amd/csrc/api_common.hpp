// What the files of the C ABI share: checks of the caller's arguments before anything is launched.
#pragma once

#include "../../include/mae_hip.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mae {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether this process sees a HIP device; asked once (the answer does not change while the
// process lives) so that the launch paths do not query the runtime on every call.
inline int have_device() {
  static const int status = [] {
    int n = 0;
    if (hipGetDeviceCount(&n) != hipSuccess || n <= 0) {
      (void)hipGetLastError();  // do not leave a sticky error for the caller's next HIP call
      return (int)MAE_ERR_NO_DEVICE;
    }
    return (int)MAE_OK;
  }();
  return status;
}

inline int validate_embed(const mae_embed_desc* d) {
  if (!d) return MAE_ERR_NULL;
  if (!d->visible || !d->weight) return MAE_ERR_NULL;
  if (d->pos && !d->ids_keep) return MAE_ERR_NULL;
  if (d->M <= 0 || d->D <= 0 || d->E <= 0 || d->L <= 0) return MAE_ERR_SHAPE;
  if (d->D % 4 != 0) return MAE_ERR_SHAPE;
  if (d->M > (int64_t(1) << 28) || d->D > 3072 || d->E > 8192) return MAE_ERR_RANGE;
  if (d->out_dtype != MAE_F32 && d->out_dtype != MAE_BF16) return MAE_ERR_DTYPE;
  if (!aligned(d->visible, 16) || !aligned(d->weight, 16) || (d->pos && !aligned(d->pos, 16)))
    return MAE_ERR_RANGE;
  return MAE_OK;
}

}  // namespace mae
