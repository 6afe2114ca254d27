// Packed-sequence attention, forward, bf16 features.
#include "packed_fwd.h"

namespace gt {
template gt_status packed_fwd<uint16_t>(const gt_packed_plan*, int, PackedArgs, hipStream_t);
}  // namespace gt
