// Scored attention, backward: dQ over the rows of the layout, dK and dV over its columns.  The kernel is in attn_scored.h.
#include "attn_scored.h"

namespace ca {

hipError_t launch_scored_dq(const ScoredArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_scored<kScoredDQ, 64>(a, stream) : launch_scored<kScoredDQ, 128>(a, stream);
}

hipError_t launch_scored_dkv(const ScoredArgs& a, hipStream_t stream) {
  // Head dim 128: the sums of dK and dV and the key's K and V alone are 192 registers, and both in one kernel spill; apart they take one product more.
  if (a.D == 64) return launch_scored<kScoredDKV, 64>(a, stream);
  const hipError_t e = launch_scored<kScoredDV, 128>(a, stream);
  return e == hipSuccess ? launch_scored<kScoredDK, 128>(a, stream) : e;
}

}  // namespace ca
