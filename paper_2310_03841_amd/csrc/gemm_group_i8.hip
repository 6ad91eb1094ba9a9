// Products over groups of rows, of int8 operands.
#include "gemm_group.h"

namespace abft {

hipError_t launch_group_rows_i8(int ot, int tiles, bool protect, bool transB, GroupArgs &g, hipStream_t st)
{
    switch (ot) {
    case DT_I8:   return launch_rows_of<DT_I8, DT_I8>(tiles, protect, transB, g, st);
    case DT_BF16: return launch_rows_of<DT_I8, DT_BF16>(tiles, protect, transB, g, st);
    case DT_F16:  return launch_rows_of<DT_I8, DT_F16>(tiles, protect, transB, g, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace abft
