// Layer norm, float32 storage.
#include "o1d_ln_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_ln_fwd_f32(const LnParams& p, hipStream_t stream) { return ln_fwd_t<float>(p, stream); }
hipError_t launch_ln_bwd_f32(const LnParams& p, hipStream_t stream) { return ln_bwd_t<float>(p, stream); }

}  // namespace rows
}  // namespace o1d
