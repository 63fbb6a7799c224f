// Products of few rows, bfloat16 storage.
#include "o1d_few_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_few_bf16(int kind, const MmParams& p, hipStream_t stream) { return launch_few_t<uint16_t>(kind, p, stream); }

}  // namespace rows
}  // namespace o1d
