// Products of 8-bit operands, weight gradient, bfloat16 results.
#include "o1d_f8_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_f8_wgrad_bf16(const F8Plan& pl, hipStream_t stream) { return launch_f8_kind<uint16_t, kWgrad>(pl, stream); }

}  // namespace rows
}  // namespace o1d
