// Attention behind shared rows, caches of 4-bit codes.
#include "shared_launch.h"

namespace mpc {

hipError_t launch_shared_mx4(const SharedArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return dev::launch_shared_format<F32, MPC_PAGE_MX4>(a, D, st);
  if (dtype == MPC_FP16) return dev::launch_shared_format<F16, MPC_PAGE_MX4>(a, D, st);
  return dev::launch_shared_format<BF16, MPC_PAGE_MX4>(a, D, st);
}

}  // namespace mpc
