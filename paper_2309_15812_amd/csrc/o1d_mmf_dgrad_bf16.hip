// Matrix products of aligned rows, bfloat16 storage: dgrad.
#include "o1d_mmf_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_mmf_dgrad_bf16(const MmPlan& pl, hipStream_t stream) { return launch_fast_kind<uint16_t, kDgrad>(pl, stream); }

}  // namespace rows
}  // namespace o1d
