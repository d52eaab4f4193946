// Launches of the shared rows' and the own rows' kernels by head size and page format.
#pragma once
#include "shared_wide_dev.h"

namespace mpc {
namespace dev {

template <class DT, int D, int FMT>
hipError_t launch_shared_d(const SharedArgs& a, hipStream_t st) {
  if constexpr (DT::kElt == 2) {
    if (a.wide) {
      hipLaunchKernelGGL((k_shared_wide<DT, D, FMT>), dim3((unsigned)a.shared.workers), dim3(kWideWaves * kWave), 0, st, a);
      return hipGetLastError();
    }
  }
  return launch_narrow<DT, D, FMT>(a, st);
}
template <class DT, int FMT>
hipError_t launch_shared_format(const SharedArgs& a, int D, hipStream_t st) {
  return D == 64 ? launch_shared_d<DT, 64, FMT>(a, st) : launch_shared_d<DT, 128, FMT>(a, st);
}

}  // namespace dev
}  // namespace mpc
