// cci_head_dw.cu -- a head's gradient of its weights on the tensor cores (kernels in cci_gated.cuh and cci_wide.cuh; a translation
// unit of its own, so that they compile side by side)
#include "cci_wide.cuh"

namespace cci {
namespace gated {

cudaError_t launch_dw_one(const Job &j, cudaStream_t stream) { return launch_one<kDwOne>(j, stream); }

}  // namespace gated
}  // namespace cci
