// Products over groups of rows that fill the chip, of f16 operands.
#include "gemm_group_big.h"

namespace abft {

hipError_t launch_group_big_f16(bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    if (transB) return protect ? launch_big_one<DT_F16, DT_F16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_F16, DT_F16, false, BIG_ROWS, false>(g, st);
    return protect ? launch_big_one<DT_F16, DT_F16, true, BIG_ROWS, true>(g, st) : launch_big_one<DT_F16, DT_F16, false, BIG_ROWS, true>(g, st);
}

}  // namespace abft
