// Matrix products of rows, float32 storage: wgrad.
#include "o1d_mm_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_mm_wgrad_f32(const MmPlan& pl, hipStream_t stream) { return launch_kind<float, kWgrad>(pl, stream); }

}  // namespace rows
}  // namespace o1d
