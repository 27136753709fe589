// cci_gated_fwd.cu -- the gated block's forward product on the tensor cores (kernel in
// cci_gated.cuh; a translation unit of its own, so that the three compile side by side)
#include "cci_gated.cuh"

namespace cci {
namespace gated {

cudaError_t launch_forward(const Job &j, cudaStream_t stream) { return launch<kForward>(j, stream); }

}  // namespace gated
}  // namespace cci
