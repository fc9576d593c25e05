// The windowed bf16 attention kernels: those of attn_bf16_impl.h with the key
// tiles that a window and the first tokens leave (a translation unit of their own,
// so that the two sets compile side by side).
#define HSTU_WINDOWED 1
#include "attn_bf16_impl.h"

namespace hstu {

const AttnBf16 &attn_bf16_windowed() {
  static const AttnBf16 k{direct_fits, bwd_grid, bwd_dq_grid, bwd_dkv_grid, launch_fwd, launch_bwd};
  return k;
}

}  // namespace hstu
