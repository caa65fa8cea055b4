// Block norms (block_norm.h) of bf16 rows.
#include "block_norm.h"

namespace turnkl {

hipError_t launch_block_norm_bf16(const BlockNormParams& p, bool bwd, hipStream_t s) {
  return p.ragged ? launch_block_typed<true, true, true>(p, bwd, s) : launch_block_typed<true, true, false>(p, bwd, s);
}

}  // namespace turnkl
