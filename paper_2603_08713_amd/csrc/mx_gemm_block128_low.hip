// The block-scaled FP8 GEMM kernel on tiles of 192 x 256, for problems of which they make one round.
#include "mx_gemm_block128.h"

namespace mx {

int launch_block128_low(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s) { return launch_b128_types<B128Shape<3, 2, 2, 4, 2>>(g, a_e5m2, b_e5m2, s); }

}  // namespace mx
