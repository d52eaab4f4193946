// Attention behind shared rows, fp32 caches (one file per element type: they build in parallel).
#include "shared_launch.h"

namespace mpc {

hipError_t launch_shared_fp32(const SharedArgs& a, int D, hipStream_t st) {
  return a.c.format == MPC_PAGE_E4M3 ? dev::launch_shared_format<F32, MPC_PAGE_E4M3>(a, D, st) : dev::launch_shared_format<F32, MPC_PAGE_SAME>(a, D, st);
}

}  // namespace mpc
