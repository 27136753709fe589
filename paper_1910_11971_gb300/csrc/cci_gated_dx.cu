// cci_gated_dx.cu -- the gated block's gradient of its input on the tensor cores (kernel in
// cci_gated.cuh; a translation unit of its own, so that the three compile side by side)
#include "cci_gated.cuh"

namespace cci {
namespace gated {

cudaError_t launch_dx(const Job &j, cudaStream_t stream) { return launch<kDx>(j, stream); }

}  // namespace gated
}  // namespace cci
