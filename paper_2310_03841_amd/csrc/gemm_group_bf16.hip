// Products over groups of rows, and gradients of their matrices, of bf16 operands.
#include "gemm_group.h"

namespace abft {

hipError_t launch_group_rows_bf16(int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    return launch_rows_of<DT_BF16, DT_BF16>(tiles, protect, transB, g, st);
}

hipError_t launch_group_depth_bf16(int tiles, GroupArgs &g, hipStream_t st) { return launch_depth_of<DT_BF16>(tiles, g, st); }

}  // namespace abft
