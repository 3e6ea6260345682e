// The block-scaled FP8 GEMM kernel on tiles of 64 x 128, two sets of four wavefronts that take the blocks of K in turn: one workgroup on a compute unit, with loads of
// four stages under way.  (512 x 4096 x 4096 17.2 us, one set with loads three stages ahead 17.7; 128 x 4096 x 4096 15.1 and 17.1; 200 x 8192 x 8192 27.4 and
// 30.7.  A workgroup loads 24 KiB a stage: at 512 rows, where every compute unit has one, 201 MB in all, which the L2 gives out at 11 to 13 TB/s.  128 rows are 64
// workgroups that take as long for theirs, 27 bytes a clock each, while the other units idle: to share K among workgroups would want a workspace.)
#include "mx_gemm_block128.h"

namespace mx {

int launch_block128_halves(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s) {
    return launch_b128_types<B128Shape<2, 1, 1, 4, 3, false, 2>>(g, a_e5m2, b_e5m2, s);
}

}  // namespace mx
