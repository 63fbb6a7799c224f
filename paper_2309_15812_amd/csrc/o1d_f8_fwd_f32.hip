// Products of 8-bit operands, forward, float32 results.
#include "o1d_f8_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_f8_fwd_f32(const F8Plan& pl, hipStream_t stream) { return launch_f8_kind<float, kFwd>(pl, stream); }

}  // namespace rows
}  // namespace o1d
