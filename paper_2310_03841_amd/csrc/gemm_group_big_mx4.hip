// Products over groups of rows that fill the chip, of 4-bit operands.
#include "gemm_group_big.h"
#include "gemm_mx4.h"

namespace abft {

hipError_t launch_mx4_big(int ot, bool protect, Mx4Args &g, hipStream_t st)
{
    if (ot == DT_BF16) return protect ? launch_big_one<DT_MX4, DT_BF16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_MX4, DT_BF16, false, BIG_ROWS, false>(g, st);
    return protect ? launch_big_one<DT_MX4, DT_F16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_MX4, DT_F16, false, BIG_ROWS, false>(g, st);
}

}  // namespace abft
