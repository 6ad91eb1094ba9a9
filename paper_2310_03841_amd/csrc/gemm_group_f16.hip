// Products over groups of rows, and gradients of their matrices, of f16 operands.
#include "gemm_group.h"

namespace abft {

hipError_t launch_group_rows_f16(int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    return launch_rows_of<DT_F16, DT_F16>(tiles, protect, transB, g, st);
}

hipError_t launch_group_depth_f16(int tiles, GroupArgs &g, hipStream_t st) { return launch_depth_of<DT_F16>(tiles, g, st); }

}  // namespace abft
