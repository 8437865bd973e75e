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

// Four lanes hold four 16-bit values each, (a.lo, a.hi, d.lo, d.hi); afterwards
// lane c holds value c of the four lanes.
__device__ __forceinline__ void transpose4(uint32_t &a, uint32_t &d) {
    const int c = threadIdx.x & 3;
    const uint32_t an = __builtin_amdgcn_mov_dpp(a, 0xB1, 0xF, 0xF, false);  // of lane c ^ 1
    const uint32_t dn = __builtin_amdgcn_mov_dpp(d, 0xB1, 0xF, 0xF, false);
    if (c & 1) {
        a = (an >> 16) | (a & 0xffff0000u);
        d = (dn >> 16) | (d & 0xffff0000u);
    } else {
        a = (a & 0xffffu) | (an << 16);
        d = (d & 0xffffu) | (dn << 16);
    }
    const uint32_t ap = __builtin_amdgcn_mov_dpp(a, 0x4E, 0xF, 0xF, false);  // of lane c ^ 2
    const uint32_t dp = __builtin_amdgcn_mov_dpp(d, 0x4E, 0xF, 0xF, false);
    if (c & 2)
        a = dp;
    else
        d = ap;
}

// What a product of two such operands is multiplied by to be the values' own.
template <int P>
constexpr float kBack = P == 3 ? kSplitBack : 1.f;

// A tile's values, packed in pairs of rows as its accumulators lie, to planes in
// both orders: at[col][row] (columns below `cols`, rows below `row_end`) and
// at_t[row][col] (rows below `rows`, columns below `col_end`); the ends are
// multiples of 8, and either matrix may be null.  They go out through LDS (BM x
// BN values), 16 bytes a lane along whole rows of the tile: stores of 8 bytes
// straight from the registers, each to another row, took 46 us more for 16384 x
// 8192 values in both orders.
template <class T, int P>
__device__ __forceinline__ void store_both(uint32_t (&pk)[T::TM][T::TN][4][2][P], const gemm::Place &at, char *lds,
                                           uint16_t *to, int64_t ld, int64_t plane, int cols, int row_end,
                                           uint16_t *to_t, int64_t ld_t, int64_t plane_t, int rows, int col_end) {
    const int lane = threadIdx.x & 63;
    const int m0 = at.tile_m * T::BM, n0 = at.tile_n * T::BN;
    const int r0 = at.row0 - m0, c0 = at.col0 - n0;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (to) {
            constexpr int CH = T::BM / 8;  // 16-byte chunks of a row
            if (p > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = c0 + 32 * j + (lane & 31), chunk = (r0 + 32 * i + 8 * q) / 8;
                        *reinterpret_cast<uint2 *>(lds + (c * CH + (chunk ^ (c & (CH - 1)))) * 16 + 8 * (lane >> 5)) =
                            make_uint2(pk[i][j][q][0][p], pk[i][j][q][1][p]);
                    }
            __syncthreads();
            uint16_t *o = to + p * plane + n0 * ld + m0;
            for (int x = threadIdx.x; x < T::BN * CH; x += T::THREADS) {
                const int c = x / CH, chunk = x % CH;
                if (n0 + c < cols && m0 + 8 * chunk < row_end)
                    *reinterpret_cast<uint4 *>(o + c * ld + 8 * chunk) =
                        *reinterpret_cast<const uint4 *>(lds + (c * CH + (chunk ^ (c & (CH - 1)))) * 16);
            }
        }
        if (to_t) {
            constexpr int CH = T::BN / 8;
            // lanes of a write hold four (eight) rows and four chunks of each
            auto key = [](int r) { return (r & (CH / 4 - 1)) * 4; };
            if (p > 0 || to) __syncthreads();
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        // lane c of four takes row c of their four columns
                        uint32_t a = pk[i][j][q][0][p], d = pk[i][j][q][1][p];
                        transpose4(a, d);
                        const int r = r0 + 32 * i + 8 * q + 4 * (lane >> 5) + (lane & 3);
                        const int c = c0 + 32 * j + (lane & 28);
                        *reinterpret_cast<uint2 *>(lds + (r * CH + ((c / 8) ^ key(r))) * 16 + 2 * (c & 4)) =
                            make_uint2(a, d);
                    }
            __syncthreads();
            uint16_t *o = to_t + p * plane_t + m0 * ld_t + n0;
            for (int x = threadIdx.x; x < T::BM * CH; x += T::THREADS) {
                const int r = x / CH, chunk = x % CH;
                if (m0 + r < rows && n0 + 8 * chunk < col_end)
                    *reinterpret_cast<uint4 *>(o + r * ld_t + 8 * chunk) =
                        *reinterpret_cast<const uint4 *>(lds + (r * CH + (chunk ^ key(r))) * 16);
            }
        }
    }
}

struct Source {
    const void *p;
    int64_t stride;   // values between rows
    int64_t batch;    // values between matrices
    int rows, cols;
    const double *mat_scale;   // every value of matrix b is multiplied by mat_scale[b] first, or null
    // rows whose label is no class are taken as zeros, whatever they hold; or null
    const int64_t *target;
    int classes;
    int64_t ignore;
    __device__ __forceinline__ bool takes(int64_t r) const {
        return !target || (target[r] != ignore && target[r] >= 0 && target[r] < classes);
    }
};

// dst [batch][P][rows][ld] (ld values a row, zeros past cols up to a multiple of
// kPad) and dst_t [batch][P][cols][ld_t]; either may be null.  A workgroup takes
// the 64 x 64 block (by, bx) of matrix b, 16 bytes a lane along rows on both sides, and transposes in
// LDS (rows of 33 words: the columns that a wavefront writes at once fall on
// different banks).  Bound by the bytes: 2048 x 8192 in bf16 to two planes in
// both orders, 34 MB in and 134 out, 30 us (5.6 TB/s).
template <int P>
struct Block {
    uint32_t t[P][64][33];
};
template <bool BF16, int P>
__device__ __forceinline__ void lay_out(const Source &s, int bx, int by, int b, uint16_t *dst, int64_t ld,
                                        uint16_t *dst_t, int64_t ld_t, Block<P> &block) {
    auto &t = block.t;
    const int c0 = bx * 64, c = c0 + 8 * (threadIdx.x & 7);
    const int64_t r0 = (int64_t)by * 64;
    const double ms = s.mat_scale ? s.mat_scale[b] : 1.0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int rr = (threadIdx.x >> 3) + 32 * k;
        const int64_t r = r0 + rr;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r < s.rows && s.takes(r)) {
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

template <bool BF16, int P>
__global__ __launch_bounds__(256) void k_planes(Source s, uint16_t *dst, int64_t ld, uint16_t *dst_t, int64_t ld_t) {
    __shared__ Block<P> block;
    lay_out<BF16, P>(s, blockIdx.x, blockIdx.y, blockIdx.z, dst, ld, dst_t, ld_t, block);
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
