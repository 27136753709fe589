// cci_head_dw.cu -- a head's gradient of its weights on the tensor cores (kernel in cci_gated.cuh; a translation
// unit of its own, so that they compile side by side)
#include "cci_gated.cuh"

namespace cci {
namespace gated {

cudaError_t launch_dw_one(const Job &j, cudaStream_t stream) { return launch<kDwOne>(j, stream); }

}  // namespace gated
}  // namespace cci
