// Gradients of the matrices of groups of rows, of sizes that fill the chip.
#include "gemm_group_big.h"

namespace abft {

hipError_t launch_group_big_wgrad(int dt, GroupArgs &g, hipStream_t st)
{
    return dt == DT_BF16 ? launch_big_one<DT_BF16, DT_BF16, false, BIG_DEPTH, true>(g, st) : launch_big_one<DT_F16, DT_F16, false, BIG_DEPTH, true>(g, st);
}

}  // namespace abft
