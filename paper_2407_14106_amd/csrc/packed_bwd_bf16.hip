// Packed-sequence attention, backward, bf16 features.
#include "packed_bwd.h"

namespace gt {
template gt_status packed_bwd<uint16_t>(const gt_packed_plan*, int, PackedArgs, float*, hipStream_t);
}  // namespace gt
