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
// bound by the bytes: x in and y out; g and x in and dx out.
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
constexpr int kBackward = 1024;  // threads of a backward workgroup

__device__ __forceinline__ int64_t row_count(const int32_t *counters, int64_t rows) {
    if (!counters) return rows;
    const int64_t v = counters[CNT_V];
    return v < rows ? v : rows;
}

// Sum over the G threads of a row; every one of them gets it.  For G above a
// wavefront the workgroup's threads all call it: `red` holds one value a wave.
template <int G>
__device__ __forceinline__ float row_sum(float v, float *red) {
#pragma unroll
    for (int d = 1; d < (G < 64 ? G : 64); d *= 2) v += __shfl_xor(v, d);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        const float *mine = red + wave / W * W;
        v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += mine[i];
    }
    return v;
}

// Two sums at once.
template <int G>
__device__ __forceinline__ void row_sum2(float &a, float &b, float *red) {
#pragma unroll
    for (int d = 1; d < (G < 64 ? G : 64); d *= 2) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            red[2 * wave] = a;
            red[2 * wave + 1] = b;
        }
        __syncthreads();
        const float *mine = red + wave / W * W * 2;
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            a += mine[2 * i];
            b += mine[2 * i + 1];
        }
    }
}

template <bool XB, bool YB, int G, int NV>
__global__ __launch_bounds__(G > kForward ? G : kForward) void k_norm(NormArgs a) {
    constexpr int VEC = XB || YB ? 8 : 4;
    constexpr int RPB = (G > kForward ? G : kForward) / G;
    __shared__ float red[32];
    const int64_t n = row_count(a.counters, a.rows);
    const int j = threadIdx.x % G;
    const int64_t step = (int64_t)gridDim.x * RPB;
    // every thread of the workgroup runs the same number of rounds
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < n; r0 += step) {
        const int64_t r = r0 + threadIdx.x / G;
        const bool on = r < n;
        const char *xr = reinterpret_cast<const char *>(a.x) + (on ? r : n - 1) * a.x_stride * (XB ? 2 : 4);
        float v[NV][VEC];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) load_row<XB, VEC>(xr, (j + k * G) * VEC, a.C, v[k]);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[k][i];
        const float mu = row_sum<G>(s, red) / a.C;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = v[k][i] - mu;
                q += (j + k * G) * VEC + i < a.C ? d * d : 0.f;
            }
        const float rs = 1.f / sqrtf(row_sum<G>(q, red) / a.C + a.eps);
        if (!on) continue;
        char *yr = reinterpret_cast<char *>(a.y) + r * a.y_stride * (YB ? 2 : 4);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c0 = (j + k * G) * VEC;
            if (c0 >= a.C) continue;
            float ga[VEC], be[VEC];
            if (a.gamma) load_row<false, VEC>(a.gamma, c0, a.C, ga);
            if (a.beta) load_row<false, VEC>(a.beta, c0, a.C, be);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float h = (v[k][i] - mu) * rs;
                v[k][i] = (a.gamma ? ga[i] * h : h) + (a.beta ? be[i] : 0.f);
            }
            store_row<YB, VEC>(yr, c0, a.C, v[k]);
        }
        if (j == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rs;
        }
    }
}

// Rows of more channels than a workgroup's registers hold: three reads.
template <bool XB, bool YB>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
    constexpr int VEC = XB || YB ? 8 : 4;
    __shared__ float red[32];
    const int64_t n = row_count(a.counters, a.rows);
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const char *xr = reinterpret_cast<const char *>(a.x) + r * a.x_stride * (XB ? 2 : 4);
        char *yr = reinterpret_cast<char *>(a.y) + r * a.y_stride * (YB ? 2 : 4);
        float v[VEC];
        float s = 0.f;
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<XB, VEC>(xr, c, a.C, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[i];
        }
        const float mu = row_sum<1024>(s, red) / a.C;
        float q = 0.f;
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<XB, VEC>(xr, c, a.C, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) q += c + i < a.C ? (v[i] - mu) * (v[i] - mu) : 0.f;
        }
        const float rs = 1.f / sqrtf(row_sum<1024>(q, red) / a.C + a.eps);
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
__global__ __launch_bounds__(kBackward) void k_norm_backward(NormBackwardArgs a, float *part) {
    constexpr int VEC = XB || GB ? 8 : 4;
    constexpr int RPB = kBackward / G;
    __shared__ float red[64];
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
    const int64_t step = (int64_t)gridDim.x * RPB;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < n; r0 += step) {
        const int64_t r = r0 + threadIdx.x / G;
        const bool on = r < n;
        const int64_t rr = on ? r : n - 1;
        const char *gr = reinterpret_cast<const char *>(a.g) + rr * a.g_stride * (GB ? 2 : 4);
        const char *xr = reinterpret_cast<const char *>(a.x) + rr * a.x_stride * (XB ? 2 : 4);
        float g[NV][VEC], h[NV][VEC];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            load_row<GB, VEC>(gr, (j + k * G) * VEC, a.C, g[k]);
            load_row<XB, VEC>(xr, (j + k * G) * VEC, a.C, h[k]);
        }
        const float mu = a.mean[rr], rs = a.rstd[rr];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                h[k][i] = (h[k][i] - mu) * rs;
                const float u = g[k][i] * ga[k][i];  // 0 past C
                s1 += u;
                s2 += u * h[k][i];
            }
        row_sum2<G>(s1, s2, red);
        if (!on) continue;
        s1 /= a.C;
        s2 /= a.C;
        char *or_ = reinterpret_cast<char *>(a.gx) + r * a.gx_stride * (XB ? 2 : 4);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c0 = (j + k * G) * VEC;
            if (c0 >= a.C) continue;
            float o[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                o[i] = rs * (g[k][i] * ga[k][i] - s1 - h[k][i] * s2);
                dg[k][i] += g[k][i] * h[k][i];
                db[k][i] += g[k][i];
            }
            if (a.gx) store_row<XB, VEC>(or_, c0, a.C, o);
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
        for (int c = threadIdx.x; c < a.C; c += kBackward) {
            float s = 0.f;
            for (int w = 0; w < RPB; ++w) s += sums[w * WIDE + c];
            row[c] = s;
        }
    }
}

template <bool XB, bool GB>
__global__ __launch_bounds__(1024) void k_norm_backward_long(NormBackwardArgs a) {
    constexpr int VEC = XB || GB ? 8 : 4;
    __shared__ float red[64];
    const int64_t n = row_count(a.counters, a.rows);
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const char *gr = reinterpret_cast<const char *>(a.g) + r * a.g_stride * (GB ? 2 : 4);
        const char *xr = reinterpret_cast<const char *>(a.x) + r * a.x_stride * (XB ? 2 : 4);
        char *or_ = reinterpret_cast<char *>(a.gx) + r * a.gx_stride * (XB ? 2 : 4);
        const float mu = a.mean[r], rs = a.rstd[r];
        float g[VEC], x[VEC], ga[VEC];
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x * VEC; c < a.C; c += 1024 * VEC) {
            load_row<GB, VEC>(gr, c, a.C, g);
            load_row<XB, VEC>(xr, c, a.C, x);
            if (a.gamma) load_row<false, VEC>(a.gamma, c, a.C, ga);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float u = a.gamma ? g[i] * ga[i] : g[i];
                s1 += u;
                s2 += u * ((x[i] - mu) * rs);
            }
        }
        row_sum2<1024>(s1, s2, red);
        s1 /= a.C;
        s2 /= a.C;
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
        hipLaunchKernelGGL((k_norm<XB, YB, G_, NV_>), dim3(grid_for(a.rows, TB / G_, D->cu_count, 2048 / TB)), \
                           dim3(TB), 0, D->stream, a);                                                           \
    }
    NORM_SHAPES(GO)
#undef GO
    return hipGetLastError();
}

unsigned backward_grid(const lattice_dense *D, int64_t rows, int rpb) { return grid_for(rows, rpb, D->cu_count, 1); }

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
        if (params) {
            prows = a.rows < kLongSplit ? a.rows : kLongSplit;
            hipLaunchKernelGGL((k_norm_params_long<XB, GB>), dim3((a.C + 255) / 256, (unsigned)prows), dim3(256), 0,
                               D->stream, a, part);
        }
    } else {
        const Shape s = shape_of(a.C, VEC);
        const unsigned grid = backward_grid(D, a.rows, kBackward / s.G);
        prows = grid;
#define GO(G_, NV_)                                                                                               \
    if (s.G == G_ && s.NV == NV_)                                                                                 \
        hipLaunchKernelGGL((k_norm_backward<XB, GB, G_, NV_>), dim3(grid), dim3(kBackward),                       \
                           params ? kBackward * NV_ * VEC * sizeof(float) : 0, D->stream, a, part);
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

// The partial rows are at most cu_count (or kLongSplit): one level of rowsum.
int64_t layer_norm_backward_scratch(const lattice_dense *D, const NormBackwardArgs &a) {
    if (!a.grad_gamma && !a.grad_beta) return 0;
    const int64_t rows = D->cu_count > kLongSplit ? D->cu_count : kLongSplit;
    return 2 * rows * a.C * (int64_t)sizeof(float);
}

hipError_t launch_layer_norm_backward(lattice_dense *D, const NormBackwardArgs &a) {
    if (a.x_bf16) return a.g_bf16 ? backward<true, true>(D, a) : backward<true, false>(D, a);
    return a.g_bf16 ? backward<false, true>(D, a) : backward<false, false>(D, a);
}
