// Arguments of the kernels between a router's logits and the products over groups of rows, and back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace abft {

// Workgroups in a row, dealt out over two directions of a launch where one has not that many (MAX_GRID_X); a few more than asked for.
inline dim3 flat_grid(long wgs)
{
    constexpr long X = 1L << 22;
    return wgs <= X ? dim3((unsigned)wgs) : dim3((unsigned)X, (unsigned)((wgs + X - 1) / X));
}
__device__ __forceinline__ long flat_block() { return (long)blockIdx.y * gridDim.x + blockIdx.x; }

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_TOPK = 64, ROUTE_MAX_GROUPS = 64;

struct RouteArgs {
    const uint8_t *logits;
    long ld, ldd;                         // bytes
    int tokens, experts, topk, sigmoid, normalise, by_logit;
    int groups, top_groups, group_best;
    float scale;
    const float *bias;                    // [experts] or null
    int *expert;                          // [tokens][topk]
    float *weight;
    const float *dweight;                 // the gradient: of the weights, [tokens][topk]
    uint8_t *dlogits;
};
hipError_t launch_route(int dt, bool grad, const RouteArgs &a, hipStream_t st);

// Entries sorted by group.  hist: scratch, group_rows_words(n, groups) words.
constexpr int GROUP_ROWS_MAX = 1024;      // groups
size_t group_rows_words(long n, int groups);
hipError_t launch_group_rows(const int *group, int n, int groups, int *offsets, int *order, int *place, uint32_t *hist, hipStream_t st);

// Rows: pitches in bytes, es of an element.
hipError_t launch_gather_rows(int es, const void *X, int tokens, int cols, long ldx, const int *order, int rows, int topk, void *Y, long ldy, hipStream_t st);
struct CombineArgs {
    const uint8_t *Y, *base;              // base: null, or added
    uint8_t *out;
    const int *place;                     // [tokens][topk]
    const float *weight;                  // null: ones
    int tokens, rows, cols, topk;
    long ldy, ldb, ldo;                   // bytes
    const uint8_t *dout;                  // the gradient: out's, of dout (pitch ldo); Y and dweight null, or both there
    uint8_t *dY;
    float *dweight;
    long lddy;
};
hipError_t launch_combine_rows(int dt, bool grad, const CombineArgs &a, hipStream_t st);

}  // namespace abft
