// Paged attention kernels of fp16 caches (one file per element type: they build in parallel).
#include "paged_attn_dev.h"

namespace mpc {

hipError_t launch_paged_attn_fp16(const PagedAttnArgs& a, int D, hipStream_t st) {
  return dev::launch_paged_dtype<F16>(a, D, st);
}

}  // namespace mpc
