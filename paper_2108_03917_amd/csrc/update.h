// What update.hip and update_small.hip share.
#pragma once

#include "dense.h"

constexpr int64_t kUpdateChunk = (int64_t)2 << 30;  // scratch of the matrices taken together

// Workgroups that add up the squares of a matrix: a few runs of 2048 values each.
inline int square_parts(const UpdateArgs &a) {
    const int64_t runs = (int64_t)a.m * ((a.n + 2047) / 2048);
    const int64_t p = (runs + 7) / 8;
    return (int)(p < 1024 ? p : 1024);
}
hipError_t launch_squares(hipStream_t stream, const UpdateArgs &a, double *part);

// 1 / (norm + eps) for every thread of the workgroup, from its threads' sums of
// squares, or from the partial sums of launch_squares.  0 for zeros without eps,
// so that they stay zeros; a norm that is NaN stays one.
template <int THREADS>
__device__ __forceinline__ double inverse_norm(double s, float eps, double *red) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += red[w];
    const double d = sqrt(s) + (double)eps;
    return d == 0.0 ? 0.0 : 1.0 / d;
}
template <int THREADS>
__device__ __forceinline__ double inverse_norm(const double *part, int parts, float eps, double *red) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += THREADS) s += part[i];
    return inverse_norm<THREADS>(s, eps, red);
}

// update_small.hip: matrices with at most 128 rows or columns
bool update_small_covers(const UpdateArgs &a);
int64_t update_small_scratch(const UpdateArgs &a);
hipError_t launch_update_small(lattice_dense *D, const UpdateArgs &a);
