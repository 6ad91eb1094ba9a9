// Products over groups of rows that fill the chip, of 4-bit operands.
//
// A slab of 128 bytes is 256 of K, so tiles are few slabs deep and their start and end, and C, are most of them: 12608 x 4096 x 1024 in 16 groups, bf16 out, 47 us unprotected (2.2 PFLOP/s; C alone,
// 103 MB, is 20 at a large copy's rate) and 60 protected, of which the pass over A is 4 and the sums in the epilogue 10.
#include "gemm_group_big.h"
#include "gemm_mx4.h"

namespace abft {

hipError_t launch_mx4_big(int ot, bool protect, Mx4Args &g, hipStream_t st)
{
    if (ot == DT_BF16) return protect ? launch_big_one<DT_MX4, DT_BF16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_MX4, DT_BF16, false, BIG_ROWS, false>(g, st);
    return protect ? launch_big_one<DT_MX4, DT_F16, true, BIG_ROWS, false>(g, st) : launch_big_one<DT_MX4, DT_F16, false, BIG_ROWS, false>(g, st);
}

}  // namespace abft
