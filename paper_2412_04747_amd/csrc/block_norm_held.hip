// The junction's backward from a and s in 8 bits: the kernel of block_norm_bwd.h that unpacks them where it reads them.
#include "rgnn_internal.h"
#include "device_utils.h"
#include "block_norm_bwd.h"

namespace rgnn {

rgnn_status_t block_bwd_rows8(const rgnn_block_norm_desc_t* d, const JunctionPlan& p, const BlockBwdArgs& a, hipStream_t st) { return launch_types<true>(d, p, a, st); }

}  // namespace rgnn
