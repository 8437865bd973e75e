// The orthogonalised form of a gradient matrix by Newton-Schulz steps, in
// products of the whole chip (matrices of few rows or columns: update_small.hip):
//
//   X_0 = G / (|G|_F + eps)  (transposed if it has more rows than columns)
//   S = X X^T,   X <- a X + (b S + c S S) X,
// which drives the singular values of X towards 1 and keeps its vectors.
//
// All products run on the bf16 matrix cores (gemm.h): X, S and b S + c S S are
// held as bf16 planes, two (errors of 2^-17 a value) for a bf16 result and
// three for an fp32 one, with fp32 sums.  One plane would not do: the steps
// multiply small singular values by up to a^steps (485 with the usual
// coefficients), and the roundings to 8 bits with them.
//
// X is kept in both orders, since S sums over its columns and the last product
// over its rows.  S and its square are symmetric: only tiles on and below the
// diagonal are computed, each element written to both places.  a X is part of
// the last product too: its left operand is Q = a I + b S + c S S.  The product
// Q X is not replaced by powers of S alone: a polynomial of the
// m x m matrix costs fewer operations for wide X, but squares the condition
// number, and fp32 then loses singular values below 2^-12 of the largest.
//
// Large matrices are bound by the matrix cores: a step of 2048 x 8192 with a
// bf16 result takes 375 us (190 for Q X, at 1.1 PFLOP/s of bf16 products, 103
// and 21 for S and the join of its parts, 62 for S S), of 210 at the rate of a
// large library product.  Q X holds its packed result beside the sums: 256
// registers a lane and 17 more in memory.  Small ones by the latency of a slice on a chip that
// they do not fill: 700 x 1531 in fp32, 52 us a step of 10.
#include "planes.h"
#include "update.h"

#include <type_traits>

namespace {

template <bool BF16>
__device__ __forceinline__ float value(const void *p, int64_t at) {
    return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(p)[at]) : reinterpret_cast<const float *>(p)[at];
}

// Partial sums of squares, fp64 (squares of fp32 values neither overflow nor
// vanish): a workgroup takes every gridDim.x-th run of 2048 values of a row.
template <bool BF16>
__global__ __launch_bounds__(256) void k_squares(const void *g, int m, int n, int64_t stride, int64_t batch_stride,
                                                 double *part) {
    const int b = blockIdx.y, runs = (n + 2047) / 2048;
    double s = 0.0;
    for (int64_t t = blockIdx.x; t < (int64_t)m * runs; t += gridDim.x) {
        const int64_t r = t / runs;
        float v[8];
        load_row<BF16, 8>(reinterpret_cast<const char *>(g) + (b * batch_stride + r * stride) * (BF16 ? 2 : 4),
                          (int)(t % runs) * 2048 + threadIdx.x * 8, n, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (double)v[i] * (double)v[i];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    __shared__ double red[4];
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[(int64_t)b * gridDim.x + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(256) void k_inverse_norm(const double *part, int parts, float eps, double *scale) {
    __shared__ double red[4];
    const double s = inverse_norm<256>(part + (int64_t)blockIdx.x * parts, parts, eps, red);
    if (threadIdx.x == 0) scale[blockIdx.x] = s;
}

// Zeros in the padding of rows of ld values that hold k.
__global__ __launch_bounds__(64) void k_pad(uint16_t *p, int64_t rows, int64_t k, int64_t ld) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = k + threadIdx.x; c < ld; c += 64) p[r * ld + c] = 0;
}

template <bool GB, bool OB>
__global__ __launch_bounds__(256) void k_scaled(const void *g, int m, int n, int64_t stride, int64_t batch_stride,
                                                const double *scale, void *out) {
    const int b = blockIdx.y;
    const double s = scale[b];
    for (int r = blockIdx.x; r < m; r += gridDim.x)
        for (int c = threadIdx.x; c < n; c += 256) {
            const float v = (float)((double)value<GB>(g, b * batch_stride + r * stride + c) * s);
            const int64_t at = ((int64_t)b * m + r) * n + c;
            if (OB)
                reinterpret_cast<uint16_t *>(out)[at] = (uint16_t)pack_bf16(v, 0.f);
            else
                reinterpret_cast<float *>(out)[at] = v;
        }
}

// Four consecutive values of a row of planes, and their sum.
template <int P>
__device__ __forceinline__ void load4(const uint16_t *p, int64_t plane, float *v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = 0.f;
#pragma unroll
    for (int k = P - 1; k >= 0; --k) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p + k * plane);
        v[0] += __uint_as_float(u.x << 16);
        v[1] += __uint_as_float(u.x & 0xffff0000u);
        v[2] += __uint_as_float(u.y << 16);
        v[3] += __uint_as_float(u.y & 0xffff0000u);
    }
    if (P == 3)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] *= 1.f / kSplitScale;
}

template <int P>
__device__ __forceinline__ void store4(uint16_t *p, int64_t plane, const uint16_t (&h)[4][P]) {
#pragma unroll
    for (int k = 0; k < P; ++k)
        *reinterpret_cast<uint2 *>(p + k * plane) =
            make_uint2(h[0][k] | (uint32_t)h[1][k] << 16, h[2][k] | (uint32_t)h[3][k] << 16);
}

// Epilogue of the symmetric products: S = acc, or Q = a I + b S + c acc.
template <int P>
struct Symmetric : gemm::Simple {
    const uint16_t *s;  // S for Q, or null
    uint16_t *out;      // planes [batch][P][m][ld]
    int m;
    int64_t ld;
    float a, b, c;

    template <int TM, int TN>
    __device__ __forceinline__ void direct(gemm::f32x16_t (&acc)[TM][TN], const gemm::Place &at) const {
        const int lane = threadIdx.x & 63;
        const int64_t plane = (int64_t)m * ld;
        uint16_t *o = out + at.batch * P * plane;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int col = at.col0 + 32 * j + (lane & 31);
            if (col >= m) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5);
                    if (row + 3 < col || row >= m) continue;
                    float v[4];
                    if (s) {
                        // symmetric: row `col` of S, columns row .. row + 3 (padding past m)
                        load4<P>(s + at.batch * P * plane + col * ld + row, plane, v);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            v[r] = b * v[r] + c * (acc[i][j][4 * q + r] * planes::kBack<P>) + (row + r == col ? a : 0.f);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r] * planes::kBack<P>;
                    }
                    gemm::sched_barrier();  // or the loads of all blocks come first, and spill
                    uint16_t h[4][P];
#pragma unroll
                    for (int r = 0; r < 4; ++r) planes::split<P>(v[r], h[r]);
                    const bool whole = row >= col && row + 3 < m;
                    if (whole) store4<P>(o + col * ld + row, plane, h);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row + r >= col && row + r < m)
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                o[k * plane + (row + r) * ld + col] = h[r][k];
                                if (!whole) o[k * plane + col * ld + row + r] = h[r][k];
                            }
                }
        }
    }
    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *, char *) const {
        direct<T::TM, T::TN>(acc, at);
    }
};

// Epilogue of the step's last product: both orders of the next X, or the result.
template <int P>
struct Next : gemm::Simple {
    uint16_t *nr, *nt;     // next X [batch][P][m][ldr] and X^T [batch][P][n][ldt], or null
    void *out;             // or the result [batch][m][n] ([n][m] if tall)
    bool out_bf16, tall;
    int m, n, km, kn;      // and padded
    int64_t ldr, ldt;

    template <class T>
    static constexpr int lds() { return T::BM * T::BN * 2; }

    // To the result: four rows of a column, which are next to each other if tall.
    template <int TM, int TN>
    __device__ __forceinline__ void result(gemm::f32x16_t (&acc)[TM][TN], const gemm::Place &at) const {
        const int lane = threadIdx.x & 63;
        const int64_t first = (int64_t)at.batch * m * n;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int col = at.col0 + 32 * j + (lane & 31);
            if (col >= n) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5);
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r] * planes::kBack<P>;
                    if (tall) {
                        const int64_t to = first + (int64_t)col * m + row;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m) put(to + r, v[r]);
                    } else {
                        const int64_t to = first + (int64_t)row * n + col;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m) put(to + (int64_t)r * n, v[r]);
                    }
                }
        }
    }
    __device__ __forceinline__ void put(int64_t to, float v) const {
        if (out_bf16)
            reinterpret_cast<uint16_t *>(out)[to] = (uint16_t)pack_bf16(v, 0.f);
        else
            reinterpret_cast<float *>(out)[to] = v;
    }
    // Values as planes; those past m and n, which are 0, become the padding.
    template <int TM, int TN>
    __device__ __forceinline__ void pack(gemm::f32x16_t (&acc)[TM][TN], const gemm::Place &at,
                                         uint32_t (&pk)[TM][TN][4][2][P]) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const bool on = at.col0 + 32 * j + (lane & 31) < n;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5);
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        v[r] = on && row + r < m ? acc[i][j][4 * q + r] * planes::kBack<P> : 0.f;
                    planes::split_pair<P>(v[0], v[1], pk[i][j][q][0]);
                    planes::split_pair<P>(v[2], v[3], pk[i][j][q][1]);
                }
        }
    }
    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *lds,
                                        char *) const {
        if (out) {
            result<T::TM, T::TN>(acc, at);
            return;
        }
        uint32_t pk[T::TM][T::TN][4][2][P];
        pack<T::TM, T::TN>(acc, at, pk);
        const int64_t pt = (int64_t)n * ldt, pr = (int64_t)m * ldr;
        planes::store_both<T, P>(pk, at, lds, nt + at.batch * P * pt, ldt, pt, n, km, nr + at.batch * P * pr, ldr, pr,
                                 m, kn);
    }
    template <int TM, int TN>
    __device__ __forceinline__ void direct(gemm::f32x16_t (&acc)[TM][TN], const gemm::Place &at) const {
        if (out) {
            result<TM, TN>(acc, at);
            return;
        }
        uint32_t pk[TM][TN][4][2][P];
        pack<TM, TN>(acc, at, pk);
        const int lane = threadIdx.x & 63;
        const int64_t pt = (int64_t)n * ldt, pr = (int64_t)m * ldr;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5), col = at.col0 + 32 * j + (lane & 31);
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        uint32_t lo = pk[i][j][q][0][p], hi = pk[i][j][q][1][p];
                        if (col < n && row < km)
                            *reinterpret_cast<uint2 *>(nt + (at.batch * P + p) * pt + col * ldt + row) = make_uint2(lo, hi);
                        // lane c of four takes row c of their four columns
                        planes::transpose4(lo, hi);
                        if (row + (lane & 3) < m && col - (lane & 3) < kn)
                            *reinterpret_cast<uint2 *>(nr + (at.batch * P + p) * pr + (row + (lane & 3)) * ldr + col -
                                                       (lane & 3)) = make_uint2(lo, hi);
                    }
                }
    }
};

// Tiles, the largest first (square ones for the symmetric products).  Slices
// of 64 values are read in whole 128-byte lines, but of three planes they leave
// a CU room for one workgroup: Small is for products with a tile a CU at most
// (640 x 1536 over 704 in 24 bits: 14.1 us, and 18.0 in slices of 32), Between
// for a few more (704 x 1536: 16.5 us in 144 tiles of 128 x 64, 19.2 in 264 of
// 64 x 64 in slices of 32).
template <int P, bool LOWER>
struct Tiles {
    using Large = gemm::Tile<256, 256, 2, 4, 32, 2>;
    using Middle = gemm::Tile<128, 128, 2, 2, 32, 2, 4>;
    using Between = gemm::Tile<64, 64, 2, 2, 32, 2>;
    using Small = gemm::Tile<64, 64, 2, 2, 64, 2>;
};
template <bool LOWER>
struct Tiles<3, LOWER> {
    using Middle = gemm::Tile<128, 128, 2, 2, 32, 3>;
    using Large = typename std::conditional<LOWER, Middle, gemm::Tile<256, 128, 4, 2, 32, 3>>::type;
    using Between = typename std::conditional<LOWER, gemm::Tile<64, 64, 2, 2, 32, 3>, gemm::Tile<128, 64, 4, 2, 64, 3>>::type;
    using Small = gemm::Tile<64, 64, 2, 2, 64, 3>;
};

// Which tile a product takes and the length of its contraction's parts.  The
// large tile reads the least: it is taken where there are enough of them, or
// where parts of a long contraction give enough and each is still long (S of a
// 2048 x 8192 matrix in 16 bits: 98 us in 7 parts and 20 to join them, 182 in 128 x
// 128 tiles).  Else the largest tile that keeps half the CUs busy (its square, in
// a step: 58 us in 136 tiles of 128 x 128, 66 in 528 of 64 x 64; both slower than
// alone, since the product before it has filled the caches), or the smallest, in
// parts if the contraction is long enough to pay for the launch that joins them,
// 6 us (S of a 700 x 1531 matrix in 24 bits: 16 us in 3 parts, 25 in one; its
// square, over 704: 15 either way).
struct Choice {
    int kind;
    int64_t part, parts;
    int64_t floats;  // of the parts' sums
};
template <int P, bool LOWER>
Choice choose(const lattice_dense *D, int64_t m, int64_t n, int64_t K, int64_t batch) {
    using X = Tiles<P, LOWER>;
    const int64_t cu = D->cu_count;
    const int bm[4] = {X::Large::BM, X::Middle::BM, X::Between::BM, X::Small::BM};
    const int bn[4] = {X::Large::BN, X::Middle::BN, X::Between::BN, X::Small::BN};
    auto tiles = [&](int k) { return batch * gemm::tiles_of(m, n, bm[k], bn[k], LOWER); };
    auto with = [&](int kind, int64_t splits) {
        const int64_t part = gemm::part_length(K, splits), parts = (K + part - 1) / part;
        return Choice{kind, part, parts, parts > 1 ? parts * tiles(kind) * bm[kind] * bn[kind] : 0};
    };
    if (tiles(0) * 8 >= cu * 7) return with(0, 1);
    const int64_t s = cu / tiles(0);
    if (K / s >= 1024) return with(0, s);
    if (tiles(1) * 2 >= cu) return with(1, 1);
    if (tiles(3) > cu) return with(2, 1);
    if (tiles(3) * 2 >= cu || K < 1024) return with(3, 1);
    const int64_t most = K / 256, fill = cu / tiles(3);
    return with(3, fill < most ? fill : most);
}

template <int P, bool LOWER, class E>
hipError_t product(const lattice_dense *D, const gemm::Operand &A, const gemm::Operand &B, int64_t K, int64_t batch,
                   const E &e, float *parts) {
    using X = Tiles<P, LOWER>;
    const Choice c = choose<P, LOWER>(D, A.rows, B.rows, K, batch);
    if (c.kind == 0) return gemm::launch_parts<typename X::Large>(D->stream, A, B, K, c.part, batch, LOWER, e, parts);
    if (c.kind == 1) return gemm::launch_parts<typename X::Middle>(D->stream, A, B, K, c.part, batch, LOWER, e, parts);
    if (c.kind == 2) return gemm::launch_parts<typename X::Between>(D->stream, A, B, K, c.part, batch, LOWER, e, parts);
    return gemm::launch_parts<typename X::Small>(D->stream, A, B, K, c.part, batch, LOWER, e, parts);
}

struct Plan {
    int m, n;       // of X: m <= n
    bool tall;
    int P;
    int64_t ldr, ldt;  // values between rows
    int64_t kn, km;    // n and m padded
    int64_t chunk;     // matrices taken together
    int64_t scale, part, xr[2], xt[2], s, q, sums, bytes;

    Plan(const lattice_dense *D, const UpdateArgs &a) {
        tall = a.m > a.n;
        m = tall ? a.n : a.m;
        n = tall ? a.m : a.n;
        P = a.out_bf16 ? 2 : 3;
        ldr = gemm::row_length(n);
        ldt = gemm::row_length(m);
        kn = gemm::padded(n);
        km = gemm::padded(m);
        const int64_t each = P * 2 * (2 * (m * ldr + n * ldt) + 2 * m * ldt);
        chunk = kUpdateChunk / each;
        chunk = chunk < 1 ? 1 : chunk < a.batch ? chunk : a.batch;
        ScratchLayout l;
        scale = l.take(a.batch * 8);
        part = l.take(a.batch * square_parts(a) * 8);
        if (a.steps > 0) {
            for (int i = 0; i < 2; ++i) {
                xr[i] = l.take(chunk * P * m * ldr * 2);
                xt[i] = l.take(chunk * P * n * ldt * 2);
            }
            s = l.take(chunk * P * m * ldt * 2);
            q = l.take(chunk * P * m * ldt * 2);
            int64_t floats = 0;  // of the sums of products in parts, for a whole chunk or the last
            for (int64_t b : {chunk, a.batch % chunk}) {
                if (b == 0) continue;
                const int64_t f = P == 2 ? sum_floats<2>(D, b) : sum_floats<3>(D, b);
                floats = f > floats ? f : floats;
            }
            sums = l.take(floats * 4);
        }
        bytes = l.bytes;
    }

    template <int PL>
    int64_t sum_floats(const lattice_dense *D, int64_t b) const {
        int64_t most = choose<PL, true>(D, m, m, kn, b).floats;
        const int64_t square = choose<PL, true>(D, m, m, km, b).floats, next = choose<PL, false>(D, m, n, km, b).floats;
        most = most > square ? most : square;
        return most > next ? most : next;
    }
};

template <int P>
hipError_t steps(lattice_dense *D, const UpdateArgs &a, const Plan &p) {
    char *ws = reinterpret_cast<char *>(D->ws);
    auto h = [&](int64_t at) { return reinterpret_cast<uint16_t *>(ws + at); };
    const int m = p.m, n = p.n;
    hipStream_t st = D->stream;
    const int esz = a.g_bf16 ? 2 : 4, osz = a.out_bf16 ? 2 : 4;
    float *sums = reinterpret_cast<float *>(ws + p.sums);
    // the padding, which the symmetric products leave as it is
    auto pad = [&](int64_t at, int64_t rows, int64_t k, int64_t ld) {
        if (k == ld) return hipSuccess;
        hipLaunchKernelGGL(k_pad, dim3(grid_for(rows, 1, D->cu_count)), dim3(64), 0, st, h(at), rows, k, ld);
        return hipGetLastError();
    };
    TRY(pad(p.s, p.chunk * P * m, m, p.ldt));
    TRY(pad(p.q, p.chunk * P * m, m, p.ldt));
    for (int64_t b0 = 0; b0 < a.batch; b0 += p.chunk) {
        const int64_t batch = a.batch - b0 < p.chunk ? a.batch - b0 : p.chunk;
        const planes::Source src = {reinterpret_cast<const char *>(a.g) + b0 * a.batch_stride * esz, a.row_stride,
                                    a.batch_stride, a.m, a.n,
                                    reinterpret_cast<const double *>(ws + p.scale) + b0, nullptr, 0, 0};
        TRY(planes::launch<P>(st, a.g_bf16, src, batch, h(p.tall ? p.xt[0] : p.xr[0]), h(p.tall ? p.xr[0] : p.xt[0])));
        const gemm::Operand S = planes::operand(h(p.s), m, m, P), Q = planes::operand(h(p.q), m, m, P);
        for (int i = 0; i < a.steps; ++i) {
            const int now = i & 1, next = now ^ 1;
            const gemm::Operand X = planes::operand(h(p.xr[now]), m, n, P);
            const gemm::Operand Xt = planes::operand(h(p.xt[now]), n, m, P);
            TRY((product<P, true>(D, X, X, p.kn, batch, Symmetric<P>{{}, nullptr, h(p.s), m, p.ldt, 0.f, 0.f, 0.f}, sums)));
            TRY((product<P, true>(D, S, S, p.km, batch,
                                  Symmetric<P>{{}, h(p.s), h(p.q), m, p.ldt, a.coef[0], a.coef[1], a.coef[2]}, sums)));
            const bool last = i + 1 == a.steps;
            const Next<P> e = {{}, last ? nullptr : h(p.xr[next]), last ? nullptr : h(p.xt[next]),
                               last ? reinterpret_cast<char *>(a.out) + b0 * a.m * a.n * osz : nullptr,
                               a.out_bf16, p.tall, m, n, (int)p.km, (int)p.kn, p.ldr, p.ldt};
            TRY((product<P, false>(D, Q, Xt, p.km, batch, e, sums)));
        }
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_squares(hipStream_t stream, const UpdateArgs &a, double *part) {
    const dim3 grid(square_parts(a), (unsigned)a.batch);
    if (a.g_bf16)
        hipLaunchKernelGGL(k_squares<true>, grid, dim3(256), 0, stream, a.g, a.m, a.n, a.row_stride, a.batch_stride, part);
    else
        hipLaunchKernelGGL(k_squares<false>, grid, dim3(256), 0, stream, a.g, a.m, a.n, a.row_stride, a.batch_stride, part);
    return hipGetLastError();
}

int64_t update_scratch(const lattice_dense *D, const UpdateArgs &a) {
    return update_small_covers(a) ? update_small_scratch(a) : Plan(D, a).bytes;
}

hipError_t launch_update(lattice_dense *D, const UpdateArgs &a) {
    if (update_small_covers(a)) return launch_update_small(D, a);
    const Plan p(D, a);
    char *ws = reinterpret_cast<char *>(D->ws);
    double *scale = reinterpret_cast<double *>(ws + p.scale), *part = reinterpret_cast<double *>(ws + p.part);
    TRY(launch_squares(D->stream, a, part));
    hipLaunchKernelGGL(k_inverse_norm, dim3((unsigned)a.batch), dim3(256), 0, D->stream, part, square_parts(a), a.eps,
                       scale);
    TRY(hipGetLastError());
    if (a.steps > 0) return a.out_bf16 ? steps<2>(D, a, p) : steps<3>(D, a, p);
    const dim3 rows(grid_for(a.m, 1, D->cu_count), (unsigned)a.batch);
#define GO(GB, OB) \
    hipLaunchKernelGGL((k_scaled<GB, OB>), rows, dim3(256), 0, D->stream, a.g, a.m, a.n, a.row_stride, a.batch_stride, scale, a.out)
    if (a.g_bf16 && a.out_bf16) GO(true, true);
    else if (a.g_bf16) GO(true, false);
    else if (a.out_bf16) GO(false, true);
    else GO(false, false);
#undef GO
    return hipGetLastError();
}
