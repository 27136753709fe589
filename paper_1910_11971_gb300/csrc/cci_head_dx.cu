// cci_head_dx.cu -- a head's gradient of its inputs on the tensor cores (kernels in cci_gated.cuh and cci_wide.cuh; a translation
// unit of its own, so that they compile side by side)
#include "cci_wide.cuh"

namespace cci {
namespace gated {

cudaError_t launch_dx_add(const Job &j, cudaStream_t stream) { return launch_one<kDxAdd>(j, stream); }

}  // namespace gated
}  // namespace cci
