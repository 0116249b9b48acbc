// Cross attention kernels of one dtype (WBMM_INST_TAG).
#include "wbmm_attn.h"

namespace wbmm {

template struct AttnEntry<WBMM_INST_TAG>;

}  // namespace wbmm
