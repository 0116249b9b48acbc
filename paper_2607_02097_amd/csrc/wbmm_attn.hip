// Cross attention kernels of one dtype (WBMM_INST_TAG), for rows in whole
// 16-byte pieces (WBMM_INST_VEC 1) or at any alignment (0).
#include "wbmm_attn.h"

namespace wbmm {

template hipError_t AttnEntry<WBMM_INST_TAG>::forward<WBMM_INST_VEC != 0>(const AttnArgs &, hipStream_t);
template hipError_t AttnEntry<WBMM_INST_TAG>::backward<WBMM_INST_VEC != 0>(const AttnArgs &, hipStream_t);

}  // namespace wbmm
