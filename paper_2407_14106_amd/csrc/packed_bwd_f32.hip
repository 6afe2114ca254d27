// Packed-sequence attention, backward, fp32 features.
#include "packed_bwd.h"

namespace gt {
template gt_status packed_bwd<float>(const gt_packed_plan*, int, PackedArgs, float*, hipStream_t);
}  // namespace gt
