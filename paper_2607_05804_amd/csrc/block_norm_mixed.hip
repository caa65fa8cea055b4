// Block norms (block_norm.h) of bf16 branches over an fp32 residual stream.
#include "block_norm.h"

namespace turnkl {

hipError_t launch_block_norm_mixed(const BlockNormParams& p, bool bwd, hipStream_t s) {
  return p.ragged ? launch_block_typed<true, false, true>(p, bwd, s) : launch_block_typed<true, false, false>(p, bwd, s);
}

}  // namespace turnkl
