// The windowed float32 attention kernels (attn_f32_impl.h).
#define HSTU_WINDOWED 1
#include "attn_f32_impl.h"

namespace hstu {

hipError_t launch_window_fwd_f32(const AttnArgs &a, void *o, bool direct, hipStream_t s) {
  return launch_fwd(a, o, direct, s);
}

hipError_t launch_window_bwd_f32(const AttnArgs &a, const void *dO, void *dq, void *dk, void *dv,
                                 float *d_pos, float *d_time, hipStream_t s) {
  return launch_bwd(a, dO, dq, dk, dv, d_pos, d_time, s);
}

}  // namespace hstu
