// Attention with shaped scores for chunks of new tokens: the instances for head dim 128.
#include "shaped_extend.h"

namespace cw {

hipError_t launch_shaped_extend_d128(const ShapedParams& p, bool fp8, hipStream_t stream, const ArgPlanBuf* ap) {
  return shaped::launch_extend_d<128>(p, fp8, stream, ap);
}

}  // namespace cw
