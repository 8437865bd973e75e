// The norm of each head's row with a gain for each channel, and the rotation of
// its channels by the row's position, for queries and keys in one launch, and
// the gradients.  With n_c = x_c r, r = 1 / sqrt(mean_c x_c^2 + eps), w_c =
// gain_c n_c, and for a pair (a, b) of channels that turns with axis j of the
// position, angle t = position_j freq_pair,
//   y_a = w_a cos t - w_b sin t,   y_b = w_b cos t + w_a sin t.
// Backward, for g = dL/dy:  u_a = g_a cos t + g_b sin t,  u_b = g_b cos t - g_a sin t
// (= dL/dw),  dgain_c = sum over rows of u_c n_c,  and with v_c = u_c gain_c
//   dx_c = r (v_c - n_c mean(v n)).
//
// Channels go in units of two: a pair that turns, or two of those that stay.  A
// lane has 4 units of a head, the same ones for each row it takes, so that their
// gain and frequency stay in registers; a group of 4 to 32 lanes has a head, and
// takes one row's heads after another, so that angles are made once a row.  An angle is
// reduced to a part of a turn in 64 bits: a position of 1e5 has 1.6e4 turns, of
// which 24 bits would leave 1e-3 of one.  Everything is bound by the bytes.
//
// dgain: each lane adds up its channels in fp32, a workgroup its groups in LDS,
// and rowsum.h the workgroups in fp64, in a fixed order.
#include "dense.h"
#include "rowsum.h"

namespace {

struct Side {  // queries or keys
    const void *x, *g;
    void *out;      // y, or dx
    int64_t x_row, x_head, g_row, g_head, out_row, out_head;
    int heads;
    const float *gain;
    float *part;    // of dgain: [workgroups][D], or null
};

struct Params {
    Side side[2];
    int64_t rows;
    int D, pairs, units;
    const void *pos;
    int64_t pos_stride;
    int integers;   // positions are int32
    int axes, end[LATTICE_ROTATE_MAX_AXES];  // pairs of the axes up to and with each
    const float *freq;
    int norm;
    float eps;
    int share;      // groups that share a row
    int64_t items;  // rows x share
};

// Channels of unit u: (a, b), -1 for none.
template <bool INTER>
__device__ __forceinline__ void channels(const Params &p, int u, int &a, int &b) {
    const int rest = p.D - 2 * p.pairs, half = (rest + 1) / 2;
    if (u < p.pairs) {
        a = INTER ? 2 * u : u;
        b = INTER ? 2 * u + 1 : u + p.pairs;
    } else {
        a = 2 * p.pairs + u - p.pairs;
        b = a + half;
        if (u >= p.units) a = b = -1;
        else if (b >= p.D) b = -1;
    }
}

template <bool BF16>
__device__ __forceinline__ float load1(const void *row, int c) {
    if (c < 0) return 0.f;
    return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(row)[c]) : reinterpret_cast<const float *>(row)[c];
}
template <bool BF16>
__device__ __forceinline__ void store1(void *row, int c, float v) {
    if (c < 0) return;
    if (BF16)
        reinterpret_cast<uint16_t *>(row)[c] = (uint16_t)pack_bf16(v, 0.f);
    else
        reinterpret_cast<float *>(row)[c] = v;
}

// Four values next to each other, at the alignment of one.
template <bool BF16>
__device__ __forceinline__ void load4(const void *row, int c, float *v) {
    if constexpr (BF16) {
        struct __attribute__((packed, aligned(2))) Two { uint32_t v[2]; };
        const Two t = *reinterpret_cast<const Two *>(reinterpret_cast<const uint16_t *>(row) + c);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[2 * i] = __uint_as_float(t.v[i] << 16);
            v[2 * i + 1] = __uint_as_float(t.v[i] & 0xffff0000u);
        }
    } else {
        const Words4 t = *reinterpret_cast<const Words4 *>(reinterpret_cast<const float *>(row) + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(t.v[i]);
    }
}
template <bool BF16>
__device__ __forceinline__ void store4(void *row, int c, const float *v) {
    if constexpr (BF16) {
        struct __attribute__((packed, aligned(2))) Two { uint32_t v[2]; };
        *reinterpret_cast<Two *>(reinterpret_cast<uint16_t *>(row) + c) = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
        *reinterpret_cast<Words4 *>(reinterpret_cast<float *>(row) + c) = {__float_as_uint(v[0]), __float_as_uint(v[1]),
                                                                            __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
}

// A lane's four units of a row: first channels in v[0..3], second in v[4..7].
template <bool BF16, bool INTER>
__device__ __forceinline__ void load_units(const Params &p, const void *row, int u0, float *v) {
    if (u0 + 4 <= p.pairs) {
        if (INTER) {
            float t[8];
            load4<BF16>(row, 2 * u0, t);
            load4<BF16>(row, 2 * u0 + 4, t + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = t[2 * i];
                v[4 + i] = t[2 * i + 1];
            }
        } else {
            load4<BF16>(row, u0, v);
            load4<BF16>(row, u0 + p.pairs, v + 4);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int a, b;
            channels<INTER>(p, u0 + i, a, b);
            v[i] = load1<BF16>(row, a);
            v[4 + i] = load1<BF16>(row, b);
        }
    }
}
template <bool BF16, bool INTER>
__device__ __forceinline__ void store_units(const Params &p, void *row, int u0, const float *v) {
    if (u0 + 4 <= p.pairs) {
        if (INTER) {
            const float t[8] = {v[0], v[4], v[1], v[5], v[2], v[6], v[3], v[7]};
            store4<BF16>(row, 2 * u0, t);
            store4<BF16>(row, 2 * u0 + 4, t + 4);
        } else {
            store4<BF16>(row, u0, v);
            store4<BF16>(row, u0 + p.pairs, v + 4);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int a, b;
            channels<INTER>(p, u0 + i, a, b);
            store1<BF16>(row, a, v[i]);
            store1<BF16>(row, b, v[4 + i]);
        }
    }
}

template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int d = 1; d < G; d *= 2) x += __shfl_xor(x, d);
    return x;
}

constexpr int kThreads = 256;
constexpr double kTurns = 0.15915494309189535;  // 1 / (2 pi)

template <bool BF16, bool INTER, int G, bool BACKWARD>
__global__ __launch_bounds__(kThreads) void k_rotate(Params p) {
    constexpr int E = BF16 ? 2 : 4, GROUPS = kThreads / G;
    const int lane = threadIdx.x % G, group = threadIdx.x / G, u0 = 4 * lane;
    // this lane's units: what they turn with
    double turns[4];
    int axis[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int u = u0 + i;
        turns[i] = u < p.pairs ? (double)p.freq[u] * kTurns : 0.0;
        axis[i] = 0;
        for (int j = 0; j + 1 < p.axes; ++j)
            if (u < p.pairs && u >= p.end[j]) axis[i] = j + 1;
    }
    float gain[2][8], sums[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int a, b;
            channels<INTER>(p, u0 + i, a, b);
            gain[s][i] = p.side[s].gain && a >= 0 ? p.side[s].gain[a] : 1.f;
            gain[s][4 + i] = p.side[s].gain && b >= 0 ? p.side[s].gain[b] : 1.f;
            sums[s][i] = sums[s][4 + i] = 0.f;
        }
    for (int64_t item = (int64_t)blockIdx.x * GROUPS + group; item < p.items; item += (int64_t)gridDim.x * GROUPS) {
        const int64_t row = p.share == 1 ? item : item / p.share;
        const int mine = (int)(item - row * p.share);
        float cs[4], sn[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = row * p.pos_stride + axis[i];
            const double x = p.integers ? (double)reinterpret_cast<const int32_t *>(p.pos)[at]
                                        : (double)reinterpret_cast<const float *>(p.pos)[at];
            const double t = x * turns[i];
            sincospif((float)(2.0 * (t - rint(t))), &sn[i], &cs[i]);
            if (u0 + i >= p.pairs) {  // also where the position is no number
                cs[i] = 1.f;
                sn[i] = 0.f;
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Side &d = p.side[s];
            for (int h = mine; h < d.heads; h += p.share) {
                const char *xr = reinterpret_cast<const char *>(d.x) + (row * d.x_row + h * d.x_head) * E;
                float x[8], y[8];
                load_units<BF16, INTER>(p, xr, u0, x);
                if (!BACKWARD) {
                    float r = 1.f;
                    if (p.norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
                        r = 1.f / sqrtf(group_sum<G>(ss) / (float)p.D + p.eps);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = x[i] * r * gain[s][i], b = x[4 + i] * r * gain[s][4 + i];
                        y[i] = a * cs[i] - b * sn[i];
                        y[4 + i] = b * cs[i] + a * sn[i];
                    }
                } else {
                    float g[8], u[8];
                    load_units<BF16, INTER>(p, reinterpret_cast<const char *>(d.g) + (row * d.g_row + h * d.g_head) * E, u0,
                                            g);
                    float ss = 0.f, vx = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        u[i] = g[i] * cs[i] + g[4 + i] * sn[i];
                        u[4 + i] = g[4 + i] * cs[i] - g[i] * sn[i];
                    }
                    if (p.norm) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            ss = fmaf(x[i], x[i], ss);
                            vx = fmaf(u[i] * gain[s][i], x[i], vx);
                        }
                        ss = group_sum<G>(ss);
                        vx = group_sum<G>(vx);
                        const float r = 1.f / sqrtf(ss / (float)p.D + p.eps), m = vx * r / (float)p.D;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float n = x[i] * r;
                            y[i] = r * (u[i] * gain[s][i] - n * m);
                            sums[s][i] = fmaf(u[i], n, sums[s][i]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = u[i];
                    }
                }
                store_units<BF16, INTER>(p, reinterpret_cast<char *>(d.out) + (row * d.out_row + h * d.out_head) * E, u0, y);
            }
        }
    }
    if (BACKWARD && (p.side[0].part || p.side[1].part)) {
        // a workgroup's groups, in their order
        __shared__ float all[2][GROUPS][8 * G];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) all[s][group][8 * lane + i] = sums[s][i];
        __syncthreads();
        for (int id = threadIdx.x; id < 2 * 8 * G; id += kThreads) {
            const int s = id / (8 * G), at = id % (8 * G), i = at & 7;
            int c[2];
            channels<INTER>(p, 4 * (at >> 3) + (i & 3), c[0], c[1]);
            const int to = i < 4 ? c[0] : c[1];
            if (to < 0 || !p.side[s].part) continue;
            float x = 0.f;
            for (int g = 0; g < GROUPS; ++g) x += all[s][g][at];
            p.side[s].part[(int64_t)blockIdx.x * p.D + to] = x;
        }
    }
}

int group_of(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32; }

Params params_of(const lattice_dense *D, const RotateArgs &a, bool backward, unsigned &grid) {
    Params p = {};
    p.side[0] = {a.q, a.grad_q, a.out_q, a.q_row, a.q_head, a.gq_row, a.gq_head, a.oq_row, a.oq_head, a.heads, a.gain_q, nullptr};
    p.side[1] = {a.k, a.grad_k, a.out_k, a.k_row, a.k_head, a.gk_row, a.gk_head, a.ok_row, a.ok_head, a.kv_heads, a.gain_k, nullptr};
    p.rows = a.rows;
    p.D = a.D;
    p.pos = a.pos;
    p.pos_stride = a.pos_stride;
    p.integers = a.integers;
    p.axes = a.axes;
    for (int i = 0; i < a.axes; ++i) p.end[i] = p.pairs += a.sections[i];
    p.units = p.pairs + (a.D - 2 * p.pairs + 1) / 2;
    p.freq = a.freq;
    p.norm = a.norm;
    p.eps = a.eps;
    // groups share a row where the rows alone are few
    const int groups = kThreads / group_of(a.D), heads = a.heads > a.kv_heads ? a.heads : a.kv_heads;
    const int64_t enough = (int64_t)4 * D->cu_count * groups;
    p.share = 1;
    while (p.share < heads && a.rows * p.share < enough) p.share *= 2;
    p.items = a.rows * p.share;
    grid = grid_for(p.items, groups, D->cu_count, backward ? 4 : 8);
    return p;
}

template <bool BF16, bool INTER, bool BACKWARD>
hipError_t launch_as(lattice_dense *D, const Params &p, unsigned grid) {
    switch (group_of(p.D)) {
        case 4: hipLaunchKernelGGL((k_rotate<BF16, INTER, 4, BACKWARD>), dim3(grid), dim3(kThreads), 0, D->stream, p); break;
        case 8: hipLaunchKernelGGL((k_rotate<BF16, INTER, 8, BACKWARD>), dim3(grid), dim3(kThreads), 0, D->stream, p); break;
        case 16: hipLaunchKernelGGL((k_rotate<BF16, INTER, 16, BACKWARD>), dim3(grid), dim3(kThreads), 0, D->stream, p); break;
        default: hipLaunchKernelGGL((k_rotate<BF16, INTER, 32, BACKWARD>), dim3(grid), dim3(kThreads), 0, D->stream, p); break;
    }
    return hipGetLastError();
}

template <bool BACKWARD>
hipError_t launch(lattice_dense *D, const RotateArgs &a, const Params &p, unsigned grid) {
    if (a.bf16) return a.interleaved ? launch_as<true, true, BACKWARD>(D, p, grid) : launch_as<true, false, BACKWARD>(D, p, grid);
    return a.interleaved ? launch_as<false, true, BACKWARD>(D, p, grid) : launch_as<false, false, BACKWARD>(D, p, grid);
}

}  // namespace

hipError_t launch_rotate(lattice_dense *D, const RotateArgs &a) {
    unsigned grid;
    const Params p = params_of(D, a, false, grid);
    return launch<false>(D, a, p, grid);
}

int64_t rotate_backward_scratch(const lattice_dense *D, const RotateArgs &a) {
    if (!a.grad_gain_q && !a.grad_gain_k) return 0;
    unsigned grid;
    params_of(D, a, true, grid);
    return (int64_t)2 * grid * a.D * 4;
}

hipError_t launch_rotate_backward(lattice_dense *D, const RotateArgs &a) {
    unsigned grid;
    Params p = params_of(D, a, true, grid);
    float *part = static_cast<float *>(D->ws);
    if (a.grad_gain_q) p.side[0].part = part;
    if (a.grad_gain_k) p.side[1].part = part + (int64_t)grid * a.D;
    const int64_t rows = a.rows > 0 ? grid : 0;
    if (a.rows > 0) TRY(launch<true>(D, a, p, grid));
    if (!a.grad_gain_q && !a.grad_gain_k) return hipSuccess;
    // at most 4 workgroups a CU: one level of sums
    const rowsum::Job jobs[2] = {{part, a.grad_gain_q, rows, a.D}, {part + (int64_t)grid * a.D, a.grad_gain_k, rows, a.D}};
    return rowsum::sum_all(D->stream, jobs, 2, nullptr);
}
