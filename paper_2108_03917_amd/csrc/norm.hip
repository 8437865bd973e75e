// Layer normalisation of the channels of each row, and its gradients.
//
//   mu = mean_c x_c,  v = mean_c (x_c - mu)^2,  r = 1 / sqrt(v + eps)
//   h_c = r (x_c - mu),  y_c = gamma_c h_c + beta_c
// and, with u_c = g_c gamma_c for g = dL/dy,
//   dx_c = r (u_c - mean(u) - h_c mean(u h))
//   dgamma_c = sum over rows of g_c h_c,  dbeta_c = sum over rows of g_c.
//
// A row stays in the registers of G threads (8 to 64 lanes of a wavefront, or
// a whole workgroup of 256 or 1024 threads for wide rows), NV chunks of VEC channels each, so
// that it is read once and the variance is the two-pass one.  Rows of more
// channels than a workgroup holds are read again for each pass.  Everything is
// bound by the bytes: x in and y out; g and x in and dx out.  16384 x 4096 in
// bf16: 48 us forward (5.6 TB/s, a large copy 5.2) and 80 backward (5.0 TB/s);
// 82411 x 100 in fp32: 15 (4.5 TB/s) and 23 (4.3 TB/s).
//
// The backward kernel's workgroups walk over the rows; a thread's channels are
// the same in each, and their dgamma and dbeta stay in its registers.  At the
// end a workgroup adds its row groups in LDS and writes one partial row; the
// partial rows are added in a fixed order (rowsum.h): no atomics, so two calls
// give the same bits.
#include "dense.h"
#include "rowsum.h"

namespace {

constexpr int kForward = 256;    // threads of a forward workgroup, at least
// Threads of a backward workgroup: two of 512 a CU, each a row of partial sums
// (16384 x 4096 in bf16: 80 us and 8 for the sums; one of 1024, 89 and 5).
template <int G>
constexpr int backward_threads() { return G > 512 ? G : 512; }

__device__ __forceinline__ int64_t row_count(const int32_t *counters, int64_t rows) {
    if (!counters) return rows;
    const int64_t v = counters[CNT_V];
    return v < rows ? v : rows;
}

// Sums over the G threads of a row; every one of them gets them.  For G above a
// wavefront all threads of the workgroup call it, with `red` one value for each
// wave and sum, and with another `red` in the next call: a wavefront that
// writes one again has passed the barrier of the call in between, which the
// others reach after reading it.
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *red) {
#pragma unroll
    for (int d = 1; d < (G < 64 ? G : 64); d *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], d);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) red[N * wave + k] = v[k];
        __syncthreads();
        const float *mine = red + wave / W * W * N;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += mine[N * i + k];
    }
}

// Rows that a thread has in hand at once: two where a row is one load a thread,
// for the bytes in flight.
template <int G, int NV>
constexpr int at_once() { return G <= 64 && NV == 1 ? 2 : 1; }

template <bool XB, bool YB, int G, int NV>
__global__ __launch_bounds__(G > kForward ? G : kForward) void k_norm(NormArgs a) {
    constexpr int VEC = XB || YB ? 8 : 4;
    constexpr int RPB = (G > kForward ? G : kForward) / G, U = at_once<G, NV>();
    __shared__ float red[2][16];
    const int64_t n = row_count(a.counters, a.rows);
    const int j = threadIdx.x % G;
    float ga[NV][VEC], be[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (a.gamma) load_row<false, VEC>(a.gamma, (j + k * G) * VEC, a.C, ga[k]);
        if (a.beta) load_row<false, VEC>(a.beta, (j + k * G) * VEC, a.C, be[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (!a.gamma) ga[k][i] = 1.f;
            if (!a.beta) be[k][i] = 0.f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * RPB * U;
    // every thread of the workgroup runs the same number of rounds
    for (int64_t r0 = (int64_t)blockIdx.x * RPB * U; r0 < n; r0 += step) {
        float v[U][NV][VEC];
        int64_t row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = r0 + u * RPB + threadIdx.x / G;
            const char *xr = reinterpret_cast<const char *>(a.x) + (row[u] < n ? row[u] : n - 1) * a.x_stride * (XB ? 2 : 4);
#pragma unroll
            for (int k = 0; k < NV; ++k) load_row<XB, VEC>(xr, (j + k * G) * VEC, a.C, v[u][k]);
        }
        float s[U], q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[u] += v[u][k][i];
        }
        row_sums<G, U>(s, red[0]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] /= a.C;
            q[u] = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = v[u][k][i] - s[u];
                    q[u] += (j + k * G) * VEC + i < a.C ? d * d : 0.f;
                }
        }
        row_sums<G, U>(q, red[1]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= n) continue;
            const float rs = 1.f / sqrtf(q[u] / a.C + a.eps);
            char *yr = reinterpret_cast<char *>(a.y) + row[u] * a.y_stride * (YB ? 2 : 4);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c0 = (j + k * G) * VEC;
                if (c0 >= a.C) continue;
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[u][k][i] = ga[k][i] * ((v[u][k][i] - s[u]) * rs) + be[k][i];
                store_row<YB, VEC>(yr, c0, a.C, v[u][k]);
            }
            if (j == 0) {
                if (a.mean) a.mean[row[u]] = s[u];
                if (a.rstd) a.rstd[row[u]] = rs;
            }
        }
    }
}

// Rows of more channels than a workgroup's registers hold: three reads.
template <bool XB, bool YB>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
    constexpr int VEC = XB || YB ? 8 : 4;
    __shared__ float red[2][16];
    const int64_t n = row_count(a.counters, a.rows);
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const char *xr = reinterpret_cast<const char *>(a.x) + r * a.x_stride * (XB ? 2 : 4);
        char *yr = reinterpret_cast<char *>(a.y) + r * a.y_stride * (YB ? 2 : 4);
        float v[VEC];
        float s[1] = {0.f}, q[1] = {0.f};
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<XB, VEC>(xr, c, a.C, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[0] += v[i];
        }
        row_sums<1024, 1>(s, red[0]);
        const float mu = s[0] / a.C;
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<XB, VEC>(xr, c, a.C, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) q[0] += c + i < a.C ? (v[i] - mu) * (v[i] - mu) : 0.f;
        }
        row_sums<1024, 1>(q, red[1]);
        const float rs = 1.f / sqrtf(q[0] / a.C + a.eps);
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<XB, VEC>(xr, c, a.C, v);
            float ga[VEC], be[VEC];
            if (a.gamma) load_row<false, VEC>(a.gamma, c, a.C, ga);
            if (a.beta) load_row<false, VEC>(a.beta, c, a.C, be);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float h = (v[i] - mu) * rs;
                v[i] = (a.gamma ? ga[i] * h : h) + (a.beta ? be[i] : 0.f);
            }
            store_row<YB, VEC>(yr, c, a.C, v);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rs;
        }
    }
}

// part: [2][gridDim.x][C] partial dgamma and dbeta, or null without either.
template <bool XB, bool GB, int G, int NV>
__global__ __launch_bounds__(backward_threads<G>(), 4) void k_norm_backward(NormBackwardArgs a, float *part) {
    constexpr int VEC = XB || GB ? 8 : 4;
    constexpr int THREADS = backward_threads<G>(), RPB = THREADS / G;
    constexpr int U = at_once<G, NV>();
    __shared__ float red[2][32];
    extern __shared__ float sums[];  // [RPB][G * NV * VEC]
    const int64_t n = row_count(a.counters, a.rows);
    const int j = threadIdx.x % G;
    float ga[NV][VEC], dg[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (a.gamma) load_row<false, VEC>(a.gamma, (j + k * G) * VEC, a.C, ga[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (!a.gamma) ga[k][i] = 1.f;
            dg[k][i] = db[k][i] = 0.f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * RPB * U;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB * U; r0 < n; r0 += step, turn ^= 1) {
        float g[U][NV][VEC], h[U][NV][VEC], mu[U], rs[U], s[2 * U];
        int64_t row[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = r0 + u * RPB + threadIdx.x / G;
            const int64_t r = row[u] < n ? row[u] : n - 1;
            const char *gr = reinterpret_cast<const char *>(a.g) + r * a.g_stride * (GB ? 2 : 4);
            const char *xr = reinterpret_cast<const char *>(a.x) + r * a.x_stride * (XB ? 2 : 4);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                load_row<GB, VEC>(gr, (j + k * G) * VEC, a.C, g[u][k]);
                load_row<XB, VEC>(xr, (j + k * G) * VEC, a.C, h[u][k]);
            }
            mu[u] = a.mean[r];
            rs[u] = a.rstd[r];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[2 * u] = s[2 * u + 1] = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[u][k][i] = (h[u][k][i] - mu[u]) * rs[u];
                    const float t = g[u][k][i] * ga[k][i];  // 0 past C
                    s[2 * u] += t;
                    s[2 * u + 1] += t * h[u][k][i];
                }
        }
        row_sums<G, 2 * U>(s, red[turn]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= n) continue;
            const float s1 = s[2 * u] / a.C, s2 = s[2 * u + 1] / a.C;
            char *or_ = reinterpret_cast<char *>(a.gx) + row[u] * a.gx_stride * (XB ? 2 : 4);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c0 = (j + k * G) * VEC;
                if (c0 >= a.C) continue;
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    o[i] = rs[u] * (g[u][k][i] * ga[k][i] - s1 - h[u][k][i] * s2);
                    dg[k][i] += g[u][k][i] * h[u][k][i];
                    db[k][i] += g[u][k][i];
                }
                if (a.gx) store_row<XB, VEC>(or_, c0, a.C, o);
            }
        }
    }
    if (!part) return;
    constexpr int WIDE = G * NV * VEC;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!(which ? a.grad_beta : a.grad_gamma)) continue;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                sums[(threadIdx.x / G) * WIDE + (j + k * G) * VEC + i] = which ? db[k][i] : dg[k][i];
        __syncthreads();
        float *row = part + ((int64_t)which * gridDim.x + blockIdx.x) * a.C;
        for (int c = threadIdx.x; c < a.C; c += THREADS) {
            float s = 0.f;
            for (int w = 0; w < RPB; ++w) s += sums[w * WIDE + c];
            row[c] = s;
        }
    }
}

template <bool XB, bool GB>
__global__ __launch_bounds__(1024) void k_norm_backward_long(NormBackwardArgs a) {
    constexpr int VEC = XB || GB ? 8 : 4;
    __shared__ float red[2][32];
    const int64_t n = row_count(a.counters, a.rows);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x, turn ^= 1) {
        const char *gr = reinterpret_cast<const char *>(a.g) + r * a.g_stride * (GB ? 2 : 4);
        const char *xr = reinterpret_cast<const char *>(a.x) + r * a.x_stride * (XB ? 2 : 4);
        char *or_ = reinterpret_cast<char *>(a.gx) + r * a.gx_stride * (XB ? 2 : 4);
        const float mu = a.mean[r], rs = a.rstd[r];
        float g[VEC], x[VEC], ga[VEC];
        float s[2] = {0.f, 0.f};
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<GB, VEC>(gr, c, a.C, g);
            load_row<XB, VEC>(xr, c, a.C, x);
            if (a.gamma) load_row<false, VEC>(a.gamma, c, a.C, ga);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float u = a.gamma ? g[i] * ga[i] : g[i];
                s[0] += u;
                s[1] += u * ((x[i] - mu) * rs);
            }
        }
        row_sums<1024, 2>(s, red[turn]);
        const float s1 = s[0] / a.C, s2 = s[1] / a.C;
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<GB, VEC>(gr, c, a.C, g);
            load_row<XB, VEC>(xr, c, a.C, x);
            if (a.gamma) load_row<false, VEC>(a.gamma, c, a.C, ga);
            float o[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                o[i] = rs * ((a.gamma ? g[i] * ga[i] : g[i]) - s1 - (x[i] - mu) * rs * s2);
            store_row<XB, VEC>(or_, c, a.C, o);
        }
    }
}

// dgamma and dbeta of long rows: workgroup (i, s) sums the rows s, s + S, ..
// of 256 channels.
template <bool XB, bool GB>
__global__ __launch_bounds__(256) void k_norm_params_long(NormBackwardArgs a, float *part) {
    const int64_t n = row_count(a.counters, a.rows);
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.C) return;
    float dg = 0.f, db = 0.f;
    for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const int64_t ig = r * a.g_stride + c, ix = r * a.x_stride + c;
        const float g = GB ? bf16_to_f32(reinterpret_cast<const uint16_t *>(a.g)[ig])
                           : reinterpret_cast<const float *>(a.g)[ig];
        const float x = XB ? bf16_to_f32(reinterpret_cast<const uint16_t *>(a.x)[ix])
                           : reinterpret_cast<const float *>(a.x)[ix];
        dg += g * ((x - a.mean[r]) * a.rstd[r]);
        db += g;
    }
    part[(int64_t)blockIdx.y * a.C + c] = dg;
    part[((int64_t)gridDim.y + blockIdx.y) * a.C + c] = db;
}

constexpr int kLongSplit = 256;  // partial rows of k_norm_params_long

int vec_of(bool a, bool b) { return a || b ? 8 : 4; }
int chunks_of(int C, int vec) { return (C + vec - 1) / vec; }
bool is_long(int C, int vec) { return chunks_of(C, vec) > 2048; }

// Threads a row is given, and chunks a thread: the fewest lanes that hold it.
struct Shape {
    int G, NV;
};
Shape shape_of(int C, int vec) {
    const int n = chunks_of(C, vec);
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {32, 1};
    if (n <= 64) return {64, 1};
    if (n <= 128) return {64, 2};
    if (n <= 256) return {256, 1};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {1024, 1};
    return {1024, 2};
}

#define NORM_SHAPES(X) X(8, 1) X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(256, 1) X(256, 2) X(1024, 1) X(1024, 2)

template <bool XB, bool YB>
hipError_t forward(lattice_dense *D, const NormArgs &a) {
    constexpr int VEC = XB || YB ? 8 : 4;
    if (is_long(a.C, VEC)) {
        hipLaunchKernelGGL((k_norm_long<XB, YB>), dim3(grid_for(a.rows, 1, D->cu_count, 2)), dim3(1024), 0, D->stream,
                           a);
        return hipGetLastError();
    }
    const Shape s = shape_of(a.C, VEC);
#define GO(G_, NV_)                                                                                              \
    if (s.G == G_ && s.NV == NV_) {                                                                              \
        constexpr int TB = G_ > kForward ? G_ : kForward;                                                        \
        hipLaunchKernelGGL((k_norm<XB, YB, G_, NV_>), dim3(grid_for(a.rows, TB / G_ * at_once<G_, NV_>(), D->cu_count, 2048 / TB)), \
                           dim3(TB), 0, D->stream, a);                                                           \
    }
    NORM_SHAPES(GO)
#undef GO
    return hipGetLastError();
}

unsigned backward_grid(const lattice_dense *D, int64_t rows, int rpb, int threads) {
    return grid_for(rows, rpb, D->cu_count, 1024 / threads);
}

template <bool XB, bool GB>
hipError_t backward(lattice_dense *D, const NormBackwardArgs &a) {
    constexpr int VEC = XB || GB ? 8 : 4;
    const bool params = a.grad_gamma || a.grad_beta;
    float *part = params ? reinterpret_cast<float *>(D->ws) : nullptr;
    int64_t prows = 0;
    if (is_long(a.C, VEC)) {
        if (a.gx)
            hipLaunchKernelGGL((k_norm_backward_long<XB, GB>), dim3(grid_for(a.rows, 1, D->cu_count, 2)), dim3(1024),
                               0, D->stream, a);
        // without rows there is no partial row, and the sums are zeros
        if (params && a.rows > 0) {
            prows = a.rows < kLongSplit ? a.rows : kLongSplit;
            hipLaunchKernelGGL((k_norm_params_long<XB, GB>), dim3((a.C + 255) / 256, (unsigned)prows), dim3(256), 0,
                               D->stream, a, part);
        }
    } else {
        const Shape s = shape_of(a.C, VEC);
        const int threads = s.G > 512 ? s.G : 512;
        const unsigned grid = backward_grid(D, a.rows, threads / s.G, threads);
        prows = grid;
#define GO(G_, NV_)                                                                                               \
    if (s.G == G_ && s.NV == NV_)                                                                                 \
        hipLaunchKernelGGL((k_norm_backward<XB, GB, G_, NV_>), dim3(grid), dim3(threads),                       \
                           params ? threads * NV_ * VEC * sizeof(float) : 0, D->stream, a, part);
        NORM_SHAPES(GO)
#undef GO
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !params) return e;
    const rowsum::Job jobs[2] = {{part, a.grad_gamma, prows, a.C}, {part + prows * a.C, a.grad_beta, prows, a.C}};
    return rowsum::sum_all(D->stream, jobs, 2, nullptr);
}

}  // namespace

hipError_t launch_layer_norm(lattice_dense *D, const NormArgs &a) {
    if (a.x_bf16) return a.y_bf16 ? forward<true, true>(D, a) : forward<true, false>(D, a);
    return a.y_bf16 ? forward<false, true>(D, a) : forward<false, false>(D, a);
}

// The partial rows are at most two a CU (or kLongSplit): one level of rowsum.
int64_t layer_norm_backward_scratch(const lattice_dense *D, const NormBackwardArgs &a) {
    if (!a.grad_gamma && !a.grad_beta) return 0;
    const int64_t rows = 2 * D->cu_count > kLongSplit ? 2 * D->cu_count : kLongSplit;
    return 2 * rows * a.C * (int64_t)sizeof(float);
}

hipError_t launch_layer_norm_backward(lattice_dense *D, const NormBackwardArgs &a) {
    if (a.x_bf16) return a.g_bf16 ? backward<true, true>(D, a) : backward<true, false>(D, a);
    return a.g_bf16 ? backward<false, true>(D, a) : backward<false, false>(D, a);
}
