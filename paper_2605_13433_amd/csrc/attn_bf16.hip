// The causal bf16 attention kernels (attn_bf16_impl.h) and the choice between them
// and the windowed ones (attn_window.hip).
#define HSTU_WINDOWED 0
#include "attn_bf16_impl.h"

namespace hstu {

namespace {
const AttnBf16 causal{direct_fits, bwd_grid, bwd_dq_grid, bwd_dkv_grid, launch_fwd, launch_bwd};
const AttnBf16 &kernels(const Problem &p) { return p.windowed ? attn_bf16_windowed() : causal; }
}  // namespace

bool fwd_direct(const Problem &p, int dev) { return kernels(p).direct_fits(p, dev); }

bool fwd_pairs(const Problem &p) {
  return p.dtype == HSTU_BF16 && p.d == 64 && p.T >= FWD_PAIR_MIN_AVG_LEN * (int64_t)p.B;
}

int attn_bwd_grid(const Problem &p, int dev) { return kernels(p).bwd_grid(p, dev); }
int attn_bwd_dq_grid(const Problem &p, int dev) { return kernels(p).bwd_dq_grid(p, dev); }
int attn_bwd_dkv_grid(const Problem &p, int dev) { return kernels(p).bwd_dkv_grid(p, dev); }

hipError_t launch_attn_fwd_bf16(const AttnArgs &a, void *o, bool direct, hipStream_t s) {
  return kernels(a.p).fwd(a, o, direct, s);
}

hipError_t launch_attn_bwd_bf16(const AttnArgs &a, const void *dO, void *dq, void *dk,
                                void *dv, const GradOut *go, hipStream_t s) {
  return kernels(a.p).bwd(a, dO, dq, dk, dv, go, s);
}

}  // namespace hstu
