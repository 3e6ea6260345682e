// The block-scaled FP8 GEMM kernel on tiles of 64 x 128, three workgroups on a compute unit.
#include "mx_gemm_block128.h"

namespace mx {

int launch_block128_small(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s) { return launch_b128_types<B128Shape<2, 1, 1, 4, 2>>(g, a_e5m2, b_e5m2, s); }

}  // namespace mx
