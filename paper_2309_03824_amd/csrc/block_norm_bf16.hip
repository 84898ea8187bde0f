// bf16 rows of block_norm.inc.
#include "lrd_device.hpp"
#define ELEM lrd::bf16_t
#include "block_norm.inc"

hipError_t block_norm_fwd_bf16(const BlockNormFwd& g, hipStream_t st) { return dispatch(g, st); }
hipError_t block_norm_bwd_bf16(const BlockNormBwd& g, hipStream_t st) { return dispatch(g, st); }

}  // namespace lrd
