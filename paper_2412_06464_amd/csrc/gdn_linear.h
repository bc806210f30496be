// Kernel argument block and launchers of linear attention with a decay.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gdn_kernels.h"

namespace gdn {

struct LinearArgs {
  const void *q, *k, *v;
  void* o;
  const float* log_alpha;  // [tokens, H], or [H] (per_head), or nullptr: alpha == 1
  const float* h0;
  float* ht;
  const int32_t* cu;  // device boundaries [N + 1] or nullptr (dense: N sequences of T tokens)
  int N, T, H, dk, dv, per_head;
  // Segments: pieces of `len` tokens of a sequence that are walked side by side;
  // len == 0: a sequence is one.  Slots of packed sequence n begin at
  // floor(cu[n] / len) + n, which leaves at least ceil(tokens / len) and one of them
  // before the next one's.
  int len, slots;
  float* states;  // [slots, H, dk, dv]: what a segment adds, then its entry state
  float* fade;    // [slots, H]: product of a segment's alphas
};

// Columns of a workgroup's slice of the state.
int linear_slice(Dt dt, int dk, int dv);
// Segments: what each adds (all but a sequence's last), then their entry states.
hipError_t launch_linear_states(Dt dt, const LinearArgs& a, hipStream_t s);
hipError_t launch_linear_walk(Dt dt, const LinearArgs& a, hipStream_t s);
hipError_t launch_linear_recurrent(Dt dt, const LinearArgs& a, hipStream_t s);

}  // namespace gdn
