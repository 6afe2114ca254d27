// Packed-sequence attention, forward, fp32 features.
#include "packed_fwd.h"

namespace gt {
template gt_status packed_fwd<float>(const gt_packed_plan*, int, PackedArgs, hipStream_t);
}  // namespace gt
