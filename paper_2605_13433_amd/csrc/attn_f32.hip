// The causal float32 attention kernels (attn_f32_impl.h) and the choice between them
// and the windowed ones (attn_window_f32.hip).
#define HSTU_WINDOWED 0
#include "attn_f32_impl.h"

namespace hstu {

hipError_t launch_attn_fwd_f32(const AttnArgs &a, void *o, bool direct, hipStream_t s) {
  return a.p.windowed ? launch_window_fwd_f32(a, o, direct, s) : launch_fwd(a, o, direct, s);
}

hipError_t launch_attn_bwd_f32(const AttnArgs &a, const void *dO, void *dq,
                               void *dk, void *dv, float *d_pos, float *d_time,
                               hipStream_t s) {
  return a.p.windowed ? launch_window_bwd_f32(a, dO, dq, dk, dv, d_pos, d_time, s)
                      : launch_bwd(a, dO, dq, dk, dv, d_pos, d_time, s);
}

}  // namespace hstu
