// Products over groups of rows that fill the chip, of int8 operands.
#include "gemm_group_big.h"

namespace abft {

hipError_t launch_group_big_i8(int ot, bool protect, GroupArgs &g, hipStream_t st)
{
    switch (ot) {
    case DT_I8:   return protect ? launch_big_one<DT_I8, DT_I8, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_I8, DT_I8, false, BIG_ROWS, false>(g, st);
    case DT_BF16: return protect ? launch_big_one<DT_I8, DT_BF16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_I8, DT_BF16, false, BIG_ROWS, false>(g, st);
    case DT_F16:  return protect ? launch_big_one<DT_I8, DT_F16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_I8, DT_F16, false, BIG_ROWS, false>(g, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace abft
