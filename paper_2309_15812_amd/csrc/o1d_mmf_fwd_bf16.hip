// Matrix products of aligned rows, bfloat16 storage: fwd.
#include "o1d_mmf_kernels.h"

namespace o1d {
namespace rows {

hipError_t launch_mmf_fwd_bf16(const MmPlan& pl, hipStream_t stream) {
  switch (pl.shape) {
    case 0: return launch_fast_shape<uint16_t, kFwd, 0>(pl, stream);
    case 1: return launch_fast_shape<uint16_t, kFwd, 1>(pl, stream);
    case 2: return launch_fast_shape<uint16_t, kFwd, 2>(pl, stream);
    case 3: return launch_fast_shape<uint16_t, kFwd, 3>(pl, stream);
    case 4: return launch_fast_shape<uint16_t, kFwd, 4>(pl, stream);
    case 5: return launch_fast_shape<uint16_t, kFwd, 5>(pl, stream);
    case 6: return launch_fast_shape<uint16_t, kFwd, 6>(pl, stream);
    default: return launch_fast_shape<uint16_t, kFwd, 7>(pl, stream);
  }
}

}  // namespace rows
}  // namespace o1d
