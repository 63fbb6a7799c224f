// Layer norm, bfloat16 storage.
#include "o1d_ln_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_ln_fwd_bf16(const LnParams& p, hipStream_t stream) { return ln_fwd_t<uint16_t>(p, stream); }
hipError_t launch_ln_bwd_bf16(const LnParams& p, hipStream_t stream) { return ln_bwd_t<uint16_t>(p, stream); }

}  // namespace rows
}  // namespace o1d
