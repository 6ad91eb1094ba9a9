// Products of 4-bit operands: which kernel a call takes, and the launches.
#pragma once
#include "group_args.h"

namespace abft {

// kind: tiles by four waves (gemm_group.h), of the fast kernel (gemm_group_big.h), or few rows (gemm_mx4_few.hip)
bool mx4_plan(bool protect, Mx4Args &g, GroupKernel *k);
// Rows and columns of C that a workgroup of it takes at a time.
void mx4_tile_shape(bool protect, const GroupKernel &k, const Mx4Args &g, int *rows, int *columns);
hipError_t launch_mx4(const GroupKernel &k, int ot, bool protect, Mx4Args &g, const uint32_t *b_max, float tau_k, float tau_cols, hipStream_t st);
hipError_t launch_mx4_big(int ot, bool protect, Mx4Args &g, hipStream_t st);
bool mx4_few_fits(bool protect, const Mx4Args &g);
int mx4_few_columns(bool protect, const Mx4Args &g);
long mx4_few_workgroups(bool protect, const Mx4Args &g);
hipError_t launch_mx4_few(int ot, bool protect, Mx4Args &g, const uint32_t *b_max, float tau_k, float tau_cols, hipStream_t st);

// K: elements of a row.  zero: words that the pass over B clears besides.
hipError_t launch_mx4_check(const GroupKernel &k, const Mx4Args &g, int K, const Workspace &w, const Verdict &v, const OneLaunch &end, hipStream_t st);
hipError_t launch_mx4_encode(const Mx4Args &g, const Workspace &w, uint32_t *zero, size_t zero_words, hipStream_t st);

}  // namespace abft
