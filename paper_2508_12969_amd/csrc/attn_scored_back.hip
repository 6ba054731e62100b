// Scored attention, backward: dQ over the rows of the layout, dK and dV over its columns.  The kernel is in attn_scored.h.
#include "attn_scored.h"

namespace ca {

hipError_t launch_scored_dq(const ScoredArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_scored<kScoredDQ, 64, 32>(a, stream) : launch_scored<kScoredDQ, 128, 32>(a, stream);
}

hipError_t launch_scored_dkv(const ScoredArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_scored<kScoredDKV, 64, 32>(a, stream) : launch_scored<kScoredDKV, 128, 32>(a, stream);
}

}  // namespace ca
