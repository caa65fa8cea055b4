// Block norms (block_norm.h) of fp32 rows.
#include "block_norm.h"

namespace turnkl {

hipError_t launch_block_norm_f32(const BlockNormParams& p, bool bwd, hipStream_t s) {
  return p.ragged ? launch_block_typed<false, false, true>(p, bwd, s) : launch_block_typed<false, false, false>(p, bwd, s);
}

}  // namespace turnkl
