// Products of few rows, float32 storage.
#include "o1d_few_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_few_f32(int kind, const MmParams& p, hipStream_t stream) { return launch_few_t<float>(kind, p, stream); }

}  // namespace rows
}  // namespace o1d
