// Matrix products of aligned rows, bfloat16 storage: wgrad.
#include "o1d_mmf_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_mmf_wgrad_bf16(const MmPlan& pl, hipStream_t stream) { return launch_fast_kind<uint16_t, kWgrad>(pl, stream); }

}  // namespace rows
}  // namespace o1d
