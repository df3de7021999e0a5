// Attention over the paged cache: the launches.
#include "dyn_attn.h"

hipError_t dyn_launch_paged_attention(const AttnArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_ATTENTION, s);
  hipError_t e = hipSuccess;
  if (a.n_tile_wide > 0 && (e = dyn_launch_attend_wide(a, s)) != hipSuccess) return e;
  return a.rows_narrow >= a.group ? dyn_launch_attend_narrow(a, s) : e;
}
