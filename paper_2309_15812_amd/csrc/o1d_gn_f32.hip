// Group norm, float32 storage.
#include "o1d_gn_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_gn_fwd_f32(const GnPlan& pl, const GnParams& p, hipStream_t stream) { return gn_fwd_t<float>(pl, p, stream); }
hipError_t launch_gn_bwd_f32(const GnPlan& pl, const GnParams& p, hipStream_t stream) { return gn_bwd_t<float>(pl, p, stream); }

}  // namespace rows
}  // namespace o1d
