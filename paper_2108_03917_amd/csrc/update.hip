// The orthogonalised form of a gradient matrix by Newton-Schulz steps:
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
// diagonal are computed, each element written to both places.  The product
// (b S + c S S) X is not replaced by powers of S alone: a polynomial of the
// m x m matrix costs fewer operations for wide X, but squares the condition
// number, and fp32 then loses singular values below 2^-12 of the largest.
#include "planes.h"

namespace {

constexpr int kNormParts = 64;                           // partial sums of squares of a matrix
constexpr int64_t kChunkBytes = (int64_t)2 << 30;        // scratch of the matrices taken together

template <bool BF16>
__device__ __forceinline__ float value(const void *p, int64_t at) {
    return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(p)[at]) : reinterpret_cast<const float *>(p)[at];
}

// Partial sums of squares, fp64 (squares of fp32 values neither overflow nor vanish).
template <bool BF16>
__global__ __launch_bounds__(256) void k_squares(const void *g, int m, int n, int64_t stride, int64_t batch_stride,
                                                 double *part) {
    const int b = blockIdx.y;
    double s = 0.0;
    for (int r = blockIdx.x; r < m; r += gridDim.x)
        for (int c = threadIdx.x; c < n; c += 256) {
            const double v = value<BF16>(g, b * batch_stride + r * stride + c);
            s += v * v;
        }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    __shared__ double red[4];
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[(int64_t)b * gridDim.x + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(64) void k_inverse_norm(const double *part, int parts, float eps, double *scale) {
    const int b = blockIdx.x;
    double s = threadIdx.x < parts ? part[(int64_t)b * parts + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if (threadIdx.x == 0) scale[b] = 1.0 / (sqrt(s) + (double)eps);
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

// Epilogue of the symmetric products: S = acc, or b S + c acc.
template <int P>
struct Symmetric : gemm::Simple {
    const uint16_t *s;  // S of which b times is added, or null
    uint16_t *out;      // planes [batch][P][m][ld]
    int m;
    int64_t ld;
    float b, c;

    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *, char *) const {
        const int lane = threadIdx.x & 63;
        const int64_t plane = (int64_t)m * ld;
        uint16_t *o = out + at.batch * P * plane;
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            const int col = at.col0 + 32 * j + (lane & 31);
            if (col >= m) continue;
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5);
                    if (row + 3 < col || row >= m) continue;
                    float v[4];
                    if (s) {
                        // symmetric: row `col` of S, columns row .. row + 3 (padding past m)
                        load4<P>(s + at.batch * P * plane + col * ld + row, plane, v);
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = b * v[r] + c * (acc[i][j][4 * q + r] * planes::kBack<P>);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r] * planes::kBack<P>;
                    }
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
};

// Epilogue of the step's last product: a X + acc, to both orders of the next X
// or to the result.
template <int P>
struct Next : gemm::Simple {
    const uint16_t *xt;    // X^T planes [batch][P][n][ldt]
    uint16_t *nr, *nt;     // next X [batch][P][m][ldr] and X^T, or null
    void *out;             // or the result [batch][m][n] ([n][m] if tall)
    bool out_bf16, tall;
    int m, n;
    int64_t ldr, ldt;
    float a;

    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *, char *) const {
        const int lane = threadIdx.x & 63;
        const int64_t pt = (int64_t)n * ldt, pr = (int64_t)m * ldr;
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            const int col = at.col0 + 32 * j + (lane & 31);
            if (col >= n) continue;
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = at.row0 + 32 * i + 8 * q + 4 * (lane >> 5);
                    if (row >= m) continue;
                    float v[4];
                    load4<P>(xt + at.batch * P * pt + col * ldt + row, pt, v);
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = a * v[r] + acc[i][j][4 * q + r] * planes::kBack<P>;
                    if (!out) {
                        uint16_t h[4][P];
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if (row + r >= m) v[r] = 0.f;  // the padding of X^T
                            planes::split<P>(v[r], h[r]);
                        }
                        store4<P>(nt + at.batch * P * pt + col * ldt + row, pt, h);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m)
#pragma unroll
                                for (int k = 0; k < P; ++k)
                                    nr[(at.batch * P + k) * pr + (row + r) * ldr + col] = h[r][k];
                        continue;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (row + r >= m) continue;
                        const int64_t to = (int64_t)at.batch * m * n +
                                           (tall ? (int64_t)col * m + row + r : (int64_t)(row + r) * n + col);
                        if (out_bf16)
                            reinterpret_cast<uint16_t *>(out)[to] = (uint16_t)pack_bf16(v[r], 0.f);
                        else
                            reinterpret_cast<float *>(out)[to] = v[r];
                    }
                }
        }
    }
};

struct Plan {
    int m, n;       // of X: m <= n
    bool tall;
    int P;
    int64_t ldr, ldt;  // values between rows
    int64_t kn, km;    // n and m padded
    int64_t chunk;     // matrices taken together
    int64_t scale, part, xr[2], xt[2], s, q, bytes;

    explicit Plan(const UpdateArgs &a) {
        tall = a.m > a.n;
        m = tall ? a.n : a.m;
        n = tall ? a.m : a.n;
        P = a.out_bf16 ? 2 : 3;
        ldr = gemm::row_length(n);
        ldt = gemm::row_length(m);
        kn = gemm::padded(n);
        km = gemm::padded(m);
        const int64_t each = P * 2 * (2 * (m * ldr + n * ldt) + 2 * m * ldt);
        chunk = kChunkBytes / each;
        chunk = chunk < 1 ? 1 : chunk < a.batch ? chunk : a.batch;
        ScratchLayout l;
        scale = l.take(a.batch * 8);
        part = l.take(a.batch * kNormParts * 8);
        if (a.steps > 0) {
            for (int i = 0; i < 2; ++i) {
                xr[i] = l.take(chunk * P * m * ldr * 2);
                xt[i] = l.take(chunk * P * n * ldt * 2);
            }
            s = l.take(chunk * P * m * ldt * 2);
            q = l.take(chunk * P * m * ldt * 2);
        }
        bytes = l.bytes;
    }
};

#define TRY(expr)                          \
    do {                                   \
        const hipError_t e_ = (expr);      \
        if (e_ != hipSuccess) return e_;   \
    } while (0)

template <int P>
struct Tiles {
    using Large = gemm::Tile<128, 128, 2, 2, 32, P>;
    using Small = gemm::Tile<64, 64, 2, 2, 32, P>;
};

// The large tile reads half as much for a product; the small one is for
// products whose large tiles would leave CUs without work.
template <int P, class E>
hipError_t product(const lattice_dense *D, const gemm::Operand &A, const gemm::Operand &B, int64_t K, int64_t batch,
                   bool lower, const E &e) {
    const int64_t tm = (A.rows + 127) / 128, tn = (B.rows + 127) / 128;
    const int64_t tiles = batch * (lower ? tm * (tm + 1) / 2 : tm * tn);
    if (tiles >= D->cu_count)
        return gemm::launch<typename Tiles<P>::Large>(D->stream, A, B, K, K, batch, lower, e);
    return gemm::launch<typename Tiles<P>::Small>(D->stream, A, B, K, K, batch, lower, e);
}

template <int P>
hipError_t steps(lattice_dense *D, const UpdateArgs &a, const Plan &p) {
    char *ws = reinterpret_cast<char *>(D->ws);
    auto h = [&](int64_t at) { return reinterpret_cast<uint16_t *>(ws + at); };
    const int m = p.m, n = p.n;
    hipStream_t st = D->stream;
    const int esz = a.g_bf16 ? 2 : 4, osz = a.out_bf16 ? 2 : 4;
    // the padding, which the products' epilogues leave as it is
    auto pad = [&](int64_t at, int64_t rows, int64_t k, int64_t ld) {
        if (k == ld) return hipSuccess;
        hipLaunchKernelGGL(k_pad, dim3(grid_for(rows, 1, D->cu_count)), dim3(64), 0, st, h(at), rows, k, ld);
        return hipGetLastError();
    };
    TRY(pad(p.xr[1], p.chunk * P * m, n, p.ldr));
    TRY(pad(p.xt[1], p.chunk * P * n, m, p.ldt));
    TRY(pad(p.s, p.chunk * P * m, m, p.ldt));
    TRY(pad(p.q, p.chunk * P * m, m, p.ldt));
    for (int64_t b0 = 0; b0 < a.batch; b0 += p.chunk) {
        const int64_t batch = a.batch - b0 < p.chunk ? a.batch - b0 : p.chunk;
        const planes::Source src = {reinterpret_cast<const char *>(a.g) + b0 * a.batch_stride * esz, a.row_stride,
                                    a.batch_stride, a.m, a.n, nullptr,
                                    reinterpret_cast<const double *>(ws + p.scale) + b0};
        TRY(planes::launch<P>(st, a.g_bf16, src, batch, h(p.tall ? p.xt[0] : p.xr[0]), h(p.tall ? p.xr[0] : p.xt[0])));
        const gemm::Operand S = planes::operand(h(p.s), m, m, P), Q = planes::operand(h(p.q), m, m, P);
        for (int i = 0; i < a.steps; ++i) {
            const int now = i & 1, next = now ^ 1;
            const gemm::Operand X = planes::operand(h(p.xr[now]), m, n, P);
            const gemm::Operand Xt = planes::operand(h(p.xt[now]), n, m, P);
            TRY((product<P>(D, X, X, p.kn, batch, true, Symmetric<P>{{}, nullptr, h(p.s), m, p.ldt, 0.f, 0.f})));
            TRY((product<P>(D, S, S, p.km, batch, true,
                            Symmetric<P>{{}, h(p.s), h(p.q), m, p.ldt, a.coef[1], a.coef[2]})));
            const bool last = i + 1 == a.steps;
            const Next<P> e = {{}, h(p.xt[now]), last ? nullptr : h(p.xr[next]), last ? nullptr : h(p.xt[next]),
                               last ? reinterpret_cast<char *>(a.out) + b0 * a.m * a.n * osz : nullptr,
                               a.out_bf16, p.tall, m, n, p.ldr, p.ldt, a.coef[0]};
            TRY((product<P>(D, Q, Xt, p.km, batch, false, e)));
        }
    }
    return hipSuccess;
}

}  // namespace

int64_t update_scratch(const lattice_dense *D, const UpdateArgs &a) {
    (void)D;
    return Plan(a).bytes;
}

hipError_t launch_update(lattice_dense *D, const UpdateArgs &a) {
    const Plan p(a);
    char *ws = reinterpret_cast<char *>(D->ws);
    double *scale = reinterpret_cast<double *>(ws + p.scale), *part = reinterpret_cast<double *>(ws + p.part);
    const int parts = a.m < kNormParts ? a.m : kNormParts;
    const dim3 grid(parts, (unsigned)a.batch);
    if (a.g_bf16)
        hipLaunchKernelGGL(k_squares<true>, grid, dim3(256), 0, D->stream, a.g, a.m, a.n, a.row_stride, a.batch_stride, part);
    else
        hipLaunchKernelGGL(k_squares<false>, grid, dim3(256), 0, D->stream, a.g, a.m, a.n, a.row_stride, a.batch_stride, part);
    hipLaunchKernelGGL(k_inverse_norm, dim3((unsigned)a.batch), dim3(64), 0, D->stream, part, parts, a.eps, scale);
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
