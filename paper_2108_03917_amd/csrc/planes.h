// The operands of gemm.h made of a caller's matrix: bf16 planes of its rows,
// padded, and of its columns (the transposed matrix, padded).
#pragma once

#include "dense.h"
#include "gemm.h"

namespace planes {
namespace {

// A value as P bf16 whose sum is the value times scale(P): see split3 for why
// three planes are scaled.
template <int P>
__device__ __forceinline__ void split(float x, uint16_t *h) {
    if constexpr (P == 1) {
        h[0] = (uint16_t)pack_bf16(x, 0.f);
    } else if constexpr (P == 2) {
        h[0] = (uint16_t)pack_bf16(x, 0.f);
        h[1] = (uint16_t)pack_bf16(x - bf16_to_f32(h[0]), 0.f);
    } else {
        uint32_t a, b, c;
        split3(x, 0.f, a, b, c);
        h[0] = (uint16_t)a;
        h[1] = (uint16_t)b;
        h[2] = (uint16_t)c;
    }
}

// What a product of two such operands is multiplied by to be the values' own.
template <int P>
constexpr float kBack = P == 3 ? kSplitBack : 1.f;

struct Source {
    const void *p;
    int64_t stride;   // values between rows
    int64_t batch;    // values between matrices
    int rows, cols;
    const int32_t *label;      // a row whose label is negative is taken as zeros (whatever it holds), or null
    const double *mat_scale;   // every value of matrix b is multiplied by mat_scale[b] first, or null
};

// dst [batch][P][rows][ld] (ld values a row, zeros past cols) and dst_t
// [batch][P][cols][ld_t]; either may be null.  A workgroup takes a 64 x 64
// block: reads along rows, transposes in LDS.
template <bool BF16, int P>
__global__ __launch_bounds__(256) void k_planes(Source s, uint16_t *dst, int64_t ld, uint16_t *dst_t, int64_t ld_t) {
    __shared__ uint16_t t[P][64][66];
    const int c0 = blockIdx.x * 64;
    const int64_t r0 = (int64_t)blockIdx.y * 64;
    const int b = blockIdx.z;
    const int c = c0 + (threadIdx.x & 63);
    const double ms = s.mat_scale ? s.mat_scale[b] : 1.0;
    for (int k = 0; k < 16; ++k) {
        const int rr = (threadIdx.x >> 6) + 4 * k;
        const int64_t r = r0 + rr;
        float x = 0.f;
        if (r < s.rows && c < s.cols && !(s.label && s.label[r] < 0)) {
            const int64_t at = b * s.batch + r * s.stride + c;
            x = BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(s.p)[at])
                     : reinterpret_cast<const float *>(s.p)[at];
            if (s.mat_scale) x = (float)((double)x * ms);
        }
        uint16_t h[P];
        split<P>(x, h);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (dst && r < s.rows && c < ld) dst[((int64_t)(b * P + p) * s.rows + r) * ld + c] = h[p];
            t[p][rr][threadIdx.x & 63] = h[p];
        }
    }
    if (!dst_t) return;
    __syncthreads();
    const int64_t r = r0 + (threadIdx.x & 63);
    for (int k = 0; k < 16; ++k) {
        const int cc = (threadIdx.x >> 6) + 4 * k;
        if (c0 + cc >= s.cols || r >= ld_t) continue;
#pragma unroll
        for (int p = 0; p < P; ++p)
            dst_t[((int64_t)(b * P + p) * s.cols + c0 + cc) * ld_t + r] = t[p][threadIdx.x & 63][cc];
    }
}

template <int P>
hipError_t launch(hipStream_t stream, bool bf16, const Source &s, int64_t batch, uint16_t *dst, uint16_t *dst_t) {
    const int64_t ld = gemm::padded(s.cols), ld_t = gemm::padded(s.rows);
    const dim3 grid((unsigned)(ld / 64), (unsigned)(ld_t / 64), (unsigned)batch);
    if (bf16)
        hipLaunchKernelGGL((k_planes<true, P>), grid, dim3(256), 0, stream, s, dst, ld, dst_t, ld_t);
    else
        hipLaunchKernelGGL((k_planes<false, P>), grid, dim3(256), 0, stream, s, dst, ld, dst_t, ld_t);
    return hipGetLastError();
}

inline gemm::Operand operand(const uint16_t *p, int64_t rows, int64_t k, int P) {
    const int64_t ld = gemm::padded(k);
    return {p, ld, rows * ld, P * rows * ld, (int)rows};
}

}  // namespace
}  // namespace planes
