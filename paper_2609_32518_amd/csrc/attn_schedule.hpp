// The work split of an attention launch, as its kernels see it.
#pragma once

#include "kernels.hpp"
#include "seg_table.hpp"

namespace unstep {

__device__ __forceinline__ Schedule make_schedule(const AttnArgs& a, int32_t* qtiles_out) {
  const int32_t qtiles = (a.N + kAttnBlockQ - 1) / kAttnBlockQ;
  *qtiles_out = qtiles;
  Schedule sc;
  sc.Tk = (a.n_keys + kAttnBlockK - 1) / kAttnBlockK;
  sc.U = int64_t(a.B) * a.H * qtiles * sc.Tk;
  sc.G = a.groups;
  return sc;
}

}  // namespace unstep
