// Token ids of a fragment, shared by the routers' append kernels.
#pragma once

#include "aep_internal.h"

namespace aep {

// The layer-local id of token t of a fragment: token_base + t, or the
// caller's id, whose pool entry lane 0 claims (an id still claimed, or out of
// range, is an error; the row is filed under a clamped id).
__device__ __forceinline__ int token_id(int t, int g, int k, int token_base, const int32_t* __restrict__ token_ids,
                                        int n_ids, int32_t* __restrict__ live, int32_t* __restrict__ pend,
                                        int32_t* __restrict__ err) {
  if (!token_ids) return token_base + t;
  int tok = token_ids[t];
  if (tok < 0 || tok >= n_ids) {
    if (g == 0) atomicOr(err, kErrTokenRange);
    tok = tok < 0 ? 0 : n_ids - 1;
  } else if (g == 0 && atomicExch(&live[tok], 1) != 0) {
    atomicOr(err, kErrCollision);
  }
  if (g == 0) pend[tok] = k;
  return tok;
}

}  // namespace aep
