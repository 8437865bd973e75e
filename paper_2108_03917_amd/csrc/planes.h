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

// The same for two values, packed.
template <int P>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t *h) {
    if constexpr (P == 3) {
        split3(x, y, h[0], h[1], h[2]);
    } else {
        h[0] = pack_bf16(x, y);
        if constexpr (P == 2)
            h[1] = pack_bf16(x - __uint_as_float(h[0] << 16), y - __uint_as_float(h[0] & 0xffff0000u));
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

// dst [batch][P][rows][ld] (ld values a row, zeros past cols up to a multiple of
// kPad) and dst_t [batch][P][cols][ld_t]; either may be null.  A workgroup takes
// a 64 x 64 block, 16 bytes a lane along rows on both sides, and transposes in
// LDS (rows of 33 words: the columns that a wavefront writes at once fall on
// different banks).  Bound by the bytes.
template <bool BF16, int P>
__global__ __launch_bounds__(256) void k_planes(Source s, uint16_t *dst, int64_t ld, uint16_t *dst_t, int64_t ld_t) {
    __shared__ uint32_t t[P][64][33];
    const int c0 = blockIdx.x * 64, c = c0 + 8 * (threadIdx.x & 7);
    const int64_t r0 = (int64_t)blockIdx.y * 64;
    const int b = blockIdx.z;
    const double ms = s.mat_scale ? s.mat_scale[b] : 1.0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int rr = (threadIdx.x >> 3) + 32 * k;
        const int64_t r = r0 + rr;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r < s.rows && !(s.label && s.label[r] < 0)) {
            const char *row = reinterpret_cast<const char *>(s.p) + (b * s.batch + r * s.stride) * (BF16 ? 2 : 4);
            load_row<BF16, 8>(row, c, s.cols, x);
            if (s.mat_scale)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = c + i < s.cols ? (float)((double)x[i] * ms) : 0.f;
        }
        uint32_t h[4][P];
#pragma unroll
        for (int i = 0; i < 4; ++i) split_pair<P>(x[2 * i], x[2 * i + 1], h[i]);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (dst && r < s.rows)
                *reinterpret_cast<uint4 *>(dst + ((int64_t)(b * P + p) * s.rows + r) * ld + c) =
                    make_uint4(h[0][p], h[1][p], h[2][p], h[3][p]);
            if (dst_t)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    reinterpret_cast<uint16_t *>(t[p][8 * (threadIdx.x & 7) + i])[rr] =
                        (uint16_t)(h[i >> 1][p] >> (16 * (i & 1)));
        }
    }
    if (!dst_t) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int cc = (threadIdx.x >> 3) + 32 * k, q = 4 * (threadIdx.x & 7);
        if (c0 + cc >= s.cols) continue;
#pragma unroll
        for (int p = 0; p < P; ++p)
            *reinterpret_cast<uint4 *>(dst_t + ((int64_t)(b * P + p) * s.cols + c0 + cc) * ld_t + r0 + 2 * q) =
                make_uint4(t[p][cc][q], t[p][cc][q + 1], t[p][cc][q + 2], t[p][cc][q + 3]);
    }
}

template <int P>
hipError_t launch(hipStream_t stream, bool bf16, const Source &s, int64_t batch, uint16_t *dst, uint16_t *dst_t) {
    const int64_t ld = gemm::row_length(s.cols), ld_t = gemm::row_length(s.rows);
    const dim3 grid((unsigned)(gemm::padded(s.cols) / 64), (unsigned)(gemm::padded(s.rows) / 64), (unsigned)batch);
    if (bf16)
        hipLaunchKernelGGL((k_planes<true, P>), grid, dim3(256), 0, stream, s, dst, ld, dst_t, ld_t);
    else
        hipLaunchKernelGGL((k_planes<false, P>), grid, dim3(256), 0, stream, s, dst, ld, dst_t, ld_t);
    return hipGetLastError();
}

inline gemm::Operand operand(const uint16_t *p, int64_t rows, int64_t k, int P) {
    const int64_t ld = gemm::row_length(k);
    return {p, ld, rows * ld, P * rows * ld, (int)rows};
}

}  // namespace
}  // namespace planes
