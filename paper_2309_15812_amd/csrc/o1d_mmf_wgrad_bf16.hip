// Matrix products of aligned rows, bfloat16 storage: wgrad.
#include "o1d_mmf_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_mmf_wgrad_bf16(const MmPlan& pl, hipStream_t stream) {
  switch (pl.shape) {
    case 0: return launch_fast_shape<uint16_t, kWgrad, 0>(pl, stream);
    case 1: return launch_fast_shape<uint16_t, kWgrad, 1>(pl, stream);
    case 2: return launch_fast_shape<uint16_t, kWgrad, 2>(pl, stream);
    case 3: return launch_fast_shape<uint16_t, kWgrad, 3>(pl, stream);
    case 4: return launch_fast_shape<uint16_t, kWgrad, 4>(pl, stream);
    case 5: return launch_fast_shape<uint16_t, kWgrad, 5>(pl, stream);
    case 6: return launch_fast_shape<uint16_t, kWgrad, 6>(pl, stream);
    default: return launch_fast_shape<uint16_t, kWgrad, 7>(pl, stream);
  }
}

}  // namespace rows
}  // namespace o1d
