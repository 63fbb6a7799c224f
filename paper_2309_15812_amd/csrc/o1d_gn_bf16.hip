// Group norm, bfloat16 storage.
#include "o1d_gn_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_gn_fwd_bf16(const GnPlan& pl, const GnParams& p, hipStream_t stream) { return gn_fwd_t<uint16_t>(pl, p, stream); }
hipError_t launch_gn_bwd_bf16(const GnPlan& pl, const GnParams& p, hipStream_t stream) { return gn_bwd_t<uint16_t>(pl, p, stream); }

}  // namespace rows
}  // namespace o1d
