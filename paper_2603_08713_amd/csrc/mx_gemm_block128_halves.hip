// The block-scaled FP8 GEMM kernel on tiles of 64 x 128, one workgroup on a compute unit with loads of three stages under way.
#include "mx_gemm_block128.h"

namespace mx {

int launch_block128_deep(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s) { return launch_b128_types<B128Shape<2, 1, 1, 4, 4>>(g, a_e5m2, b_e5m2, s); }

}  // namespace mx
