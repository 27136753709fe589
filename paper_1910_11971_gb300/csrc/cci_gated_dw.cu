// cci_gated_dw.cu -- the gated block's gradient of its weights on the tensor cores (kernel in
// cci_gated.cuh; a translation unit of its own, so that the three compile side by side)
#include "cci_gated.cuh"

namespace cci {
namespace gated {

cudaError_t launch_dw(const Job &j, cudaStream_t stream) { return launch<kDw>(j, stream); }

}  // namespace gated
}  // namespace cci
