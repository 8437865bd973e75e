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
// A lane has 4 pairs, or 8 of the channels that stay, the same ones for each row it
// takes, so that their gain and frequency stay in registers; a group of 4 to 64 lanes
// has a head, and takes one row's heads after another, so that angles are made once
// a row.  An angle is
// reduced to a part of a turn in 64 bits: a position of 1e5 has 1.6e4 turns, of
// which 24 bits would leave 1e-3 of one.
//
// Everything is bound by the bytes: 16384 rows of 32 + 8 heads of 128 in bf16, 66 us
// forward (335 MB, 5.0 TB/s; a large copy 5.6) and 113 backward (503 MB, 4.5 TB/s);
// 82411 rows of 4 + 4 heads of 36 in fp32, 49 and 100 (3.9 and 2.8 TB/s: 5 of a
// group's 8 lanes have channels).  What got them there from 113 and 364 us: loads without
// a branch around them, of 4 (backward 2) heads at a time; sums by moves between lanes
// in place of LDS; addresses made for each head, which leaves room for 5 (4)
// wavefronts a SIMD (backward, fp32 rows that are not whole lanes' keep 3 or 4 vector registers
// in memory).
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
    int D, pairs;
    const void *pos;
    int64_t pos_stride;
    int integers;   // positions are int32
    int axes, end[LATTICE_ROTATE_MAX_AXES];  // pairs of the axes up to and with each
    const float *freq;
    int norm;
    float eps;
    int share, log_share;  // groups that share a row: a power of 2
    int64_t items;  // rows x share
};

// How a kernel's lanes take their values, four at a time: all there are (WHOLE), the
// last ones of a row fewer (TAILS), or one by one (ONES, rows of fewer than four).
enum Mode { WHOLE, TAILS, ONES };

// Addresses are kept as numbers, hidden from the compiler when they are made: it would
// otherwise keep one for each of a lane's values from head to head, in 100 registers.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2), aligned(2)));
template <class T>
using global = __attribute__((address_space(1))) T;
__device__ __forceinline__ uint64_t address(const void *p, int64_t bytes) {
    uint64_t a = reinterpret_cast<uint64_t>(p) + (uint64_t)bytes;
    asm("" : "+v"(a));
    return a;
}

// Values c .. c + n - 1 of a row of D as they are stored, with zeros after them.
template <bool BF16>
struct Four {
    uint32_t w[BF16 ? 2 : 4];
};
template <bool BF16, Mode MODE>
__device__ __forceinline__ Four<BF16> load4(uint64_t row, int c, int n, int D) {
    Four<BF16> r;
    if constexpr (MODE == ONES) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) r.w[i] = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) {
                if (BF16)
                    r.w[i / 2] |= (uint32_t) * (const global<uint16_t> *)(row + (c + i) * 2) << (16 * (i & 1));
                else
                    r.w[i] = *(const global<uint32_t> *)(row + (c + i) * 4);
            }
        return r;
    } else {
        // four that lie in the row, moved to their places; no branch, so that the loads of all
        // heads are under way before the first is waited for
        const int from = MODE == WHOLE || c <= D - 4 ? c : D - 4, k = c - from;
        if constexpr (BF16) {
            const u32x2_t t = *(const global<u32x2_t> *)(row + (uint32_t)from * 2);
            if (MODE == WHOLE) {
                r.w[0] = t.x, r.w[1] = t.y;
            } else {
                uint64_t x = (uint64_t)t.y << 32 | t.x;
                x = n <= 0 ? 0 : (x >> (16 * (k & 3))) & (~(uint64_t)0 >> (64 - 16 * n));
                r.w[0] = (uint32_t)x, r.w[1] = (uint32_t)(x >> 32);
            }
        } else {
            u32x4_t t = *(const global<u32x4_t> *)(row + (uint32_t)from * 4);
            if (MODE == TAILS) {
                if (k & 1) t = u32x4_t{t.y, t.z, t.w, 0};
                if (k & 2) t = u32x4_t{t.z, t.w, 0, 0};
            }
            r.w[0] = t.x, r.w[1] = t.y, r.w[2] = t.z, r.w[3] = t.w;
            if (MODE == TAILS)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= n) r.w[i] = 0;
        }
        return r;
    }
}
template <bool BF16>
__device__ __forceinline__ void widen(const Four<BF16> &r, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = __uint_as_float(!BF16 ? r.w[BF16 ? 0 : i] : (i & 1) ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
}
template <bool BF16, Mode MODE>
__device__ __forceinline__ void store4(uint64_t row, int c, int n, const float *v) {
    if (MODE == WHOLE || (MODE == TAILS && n == 4)) {
        if constexpr (BF16)
            *(global<u32x2_t> *)(row + (uint32_t)c * 2) = u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else
            *(global<u32x4_t> *)(row + (uint32_t)c * 4) = u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]),
                                                                  __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) {
                if (BF16)
                    *(global<uint16_t> *)(row + (uint32_t)(c + i) * 2) = (uint16_t)pack_bf16(v[i], 0.f);
                else
                    *(global<float> *)(row + (uint32_t)(c + i) * 4) = v[i];
            }
    }
}

// What a lane has of a row: n[0] channels from c[0] and n[1] from c[1] on, up to 4
// each.  Lanes with pairs come first (four pairs each), then those with channels
// that stay.
struct Share {
    int c[2], n[2];
    int pair0, pairs;
};
template <bool INTER>
__device__ __forceinline__ Share share_of(const Params &p, int lane) {
    const int turning = (p.pairs + 3) / 4;
    Share s;
    int left[2];
    if (lane < turning) {
        s.pair0 = 4 * lane;
        s.pairs = p.pairs - s.pair0 < 4 ? p.pairs - s.pair0 : 4;
        s.c[0] = INTER ? 2 * s.pair0 : s.pair0;
        s.c[1] = INTER ? 2 * s.pair0 + 4 : s.pair0 + p.pairs;
        left[0] = INTER ? 2 * s.pairs : s.pairs;
        left[1] = INTER ? 2 * s.pairs - 4 : s.pairs;
    } else {
        s.pair0 = s.pairs = 0;
        s.c[0] = 2 * p.pairs + 8 * (lane - turning);
        s.c[1] = s.c[0] + 4;
        left[0] = p.D - s.c[0];
        left[1] = p.D - s.c[1];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) s.n[i] = left[i] < 0 ? 0 : left[i] > 4 ? 4 : left[i];
    return s;
}

// Turn the pairs of x by the angles, or back.
template <bool INTER, bool BACK>
__device__ __forceinline__ void turn(const float (&x)[8], const float (&cs)[4], const float (&sn)[4], float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = INTER ? 2 * i : i, b = INTER ? 2 * i + 1 : 4 + i;
        const float s = BACK ? -sn[i] : sn[i];
        y[a] = x[a] * cs[i] - x[b] * s;
        y[b] = x[b] * cs[i] + x[a] * s;
    }
}

// Sum over the G lanes of a group, the same in each: lanes 1, 2 away, then mirrored
// in 8 and 16, then 16 and 32 away.  Moves between lanes of a row of 16 are part of
// the addition; through LDS (shuffles) a sum took 8 round trips of it.
template <int CTRL>
__device__ __forceinline__ float plus_moved(float x) {
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float group_sum(float x) {
    x = plus_moved<0xb1>(x);   // quad_perm 1 0 3 2
    x = plus_moved<0x4e>(x);   // quad_perm 2 3 0 1
    if (G > 4) x = plus_moved<0x141>(x);   // row_half_mirror
    if (G > 8) x = plus_moved<0x140>(x);   // row_mirror
    if (G > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (G > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// 1 / sqrt(x): the hardware's, which is off by a unit in the last place and takes no
// subnormal x, and a Newton step; infinity for 0 and 0 for infinity, as they come.
__device__ __forceinline__ float inverse_root(float x) {
    const bool small = x < 1e-30f;
    const float y = small ? x * 1.2676506e30f : x;  // 2^100
    const float r = __builtin_amdgcn_rsqf(y), e = fmaf(-y * r, r, 1.f);
    const float z = e == e ? fmaf(0.5f * r, e, r) : r;
    return small ? z * 1.1258999e15f : z;           // 2^50
}

// Sums of squares, and of products with a gradient, that lose nothing in fp32: their terms that
// count are normal numbers, and none overflows.  Others (of values from about 1e18 on or, without
// eps, below 1e-15) are made again from the row times a power of two, in a branch that few rows
// take: the mean of the squares is 2^-98 to 2^116 there, for values from 2^-149 to 2^128.  The branch
// for each head costs the rows that do not take it 1 us of 48 forward and 1 of 99 backward (fp32, the
// sizes above); one branch for the heads side by side keeps their values and cost 17 of 66 in
// bf16.  Where all gradients are zero the backward pass takes 3 us longer.
__device__ __forceinline__ bool holds(float sum) { return sum >= 0x1p-100f && sum <= 0x1p120f; }
// The root of that power of two.
__device__ __forceinline__ float half_scale_for(float mean) {
    return mean > 0x1p120f ? 0x1p-35f : mean < 0x1p-100f ? 0x1p50f : 1.f;
}

// Sine and cosine of `turns` whole turns: the part of a turn (exact in 64 bits),
// its nearest quarter, and in the eighth of a turn about that the Taylor series
// about 0, whose first terms left out are below 2^-27.
__device__ __forceinline__ void sin_cos(double turns, float &sn, float &cs) {
    const float t = (float)(turns - rint(turns));
    const float quarter = rintf(4.f * t), y = fmaf(quarter, -0.25f, t) * 6.283185307179586f, z = y * y;
    const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), 1.f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
    const int q = (int)quarter;
    const float a = q & 1 ? c : s, b = q & 1 ? s : c;
    sn = q & 2 ? -a : a;
    cs = (q + 1) & 2 ? -b : b;
    if (t != t) sn = cs = t;
}

constexpr int kThreads = 256;
constexpr double kTurns = 0.15915494309189535;  // 1 / (2 pi)

template <bool BF16, bool INTER, int G, Mode MODE, bool BACKWARD>
__global__ __launch_bounds__(kThreads, 4) void k_rotate(Params p) {
    constexpr int E = BF16 ? 2 : 4, GROUPS = kThreads / G;
    // what a lane's pairs turn with, and the gains of its channels in the order of its
    // values (registers are few)
    __shared__ double turns[4 * G];
    __shared__ int axes[4 * G];
    __shared__ __attribute__((aligned(16))) float gains[2][8 * G];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const Share own = share_of<INTER>(p, lane);
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t item = (int64_t)blockIdx.x * GROUPS + group;

    // U heads' values at a time, so that enough loads are under way
    constexpr int U = BACKWARD ? 2 : 4;
    Four<BF16> xs[U][2], gs[BACKWARD ? U : 1][2];
    auto fetch = [&](int s, int64_t row, int h) {
        const Side &d = p.side[s];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int at = h + k * p.share < d.heads ? h + k * p.share : h;
            const uint64_t xr = address(d.x, (row * d.x_row + at * d.x_head) * E);
#pragma unroll
            for (int i = 0; i < 2; ++i) xs[k][i] = load4<BF16, MODE>(xr, own.c[i], own.n[i], p.D);
            if (BACKWARD) {
                const uint64_t gr = address(d.g, (row * d.g_row + at * d.g_head) * E);
#pragma unroll
                for (int i = 0; i < 2; ++i) gs[k][i] = load4<BF16, MODE>(gr, own.c[i], own.n[i], p.D);
            }
        }
    };

    if (group == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = own.pair0 + i;
            int axis = 0;
            for (int j = 0; j + 1 < p.axes; ++j)
                if (i < own.pairs && pair >= p.end[j]) axis = j + 1;
            turns[4 * lane + i] = i < own.pairs ? (double)p.freq[pair] * kTurns : 0.0;
            axes[4 * lane + i] = axis;
        }
    if (group < 2) {
        const float *gain = p.side[group].gain;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            gains[group][8 * lane + i] = gain && (i & 3) < own.n[i / 4] ? gain[own.c[i / 4] + (i & 3)] : 1.f;
    }
    __syncthreads();
    float sums[2][8];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[s][i] = 0.f;
    const float of_all = 1.f / (float)p.D;
    for (; item < p.items; item += step) {
        const int64_t row = item >> p.log_share;
        const int mine = (int)item & (p.share - 1);
        fetch(0, row, mine);  // every share has one of the queries' heads
        float cs[4], sn[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cs[i] = 1.f;
            sn[i] = 0.f;
            if (i < own.pairs) {
                const int64_t at = row * p.pos_stride + axes[4 * lane + i];
                const double x = p.integers ? (double)reinterpret_cast<const int32_t *>(p.pos)[at]
                                            : (double)reinterpret_cast<const float *>(p.pos)[at];
                sin_cos(x * turns[4 * lane + i], sn[i], cs[i]);
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Side &d = p.side[s];
#pragma unroll 1
            for (int h0 = mine; h0 < d.heads; h0 += U * p.share) {
                if (s > 0 || h0 > mine) fetch(s, row, h0);
                float gain[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 t = *reinterpret_cast<const float4 *>(&gains[s][8 * lane + i]);
                    gain[i] = t.x, gain[i + 1] = t.y, gain[i + 2] = t.z, gain[i + 3] = t.w;
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int h = h0 + k * p.share;
                    if (h >= d.heads) break;
                    float x[8], y[8];
                    widen<BF16>(xs[k][0], x);
                    widen<BF16>(xs[k][1], x + 4);
                    if (!BACKWARD) {
                        float ss = 0.f, w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
                        float r = 1.f;
                        if (p.norm) {
                            const float mean = group_sum<G>(ss) * of_all + p.eps;
                            r = inverse_root(mean);
                            if (!holds(mean)) {  // the same for a group's lanes
                                const float h = half_scale_for(mean), f = h * h;
                                ss = 0.f;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    x[i] *= f;
                                    ss = fmaf(x[i], x[i], ss);
                                }
                                r = inverse_root(group_sum<G>(ss) * of_all + p.eps * f * f);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = x[i] * r * gain[i];
                        turn<INTER, false>(w, cs, sn, y);
                    } else {
                        float g[8], u[8];
                        widen<BF16>(gs[k][0], g);
                        widen<BF16>(gs[k][1], g + 4);
                        turn<INTER, true>(g, cs, sn, u);
                        if (p.norm) {
                            float ss = 0.f, vx = 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                ss = fmaf(x[i], x[i], ss);
                                vx = fmaf(u[i] * gain[i], x[i], vx);
                            }
                            ss = group_sum<G>(ss);
                            vx = group_sum<G>(vx);
                            const float mean = ss * of_all + p.eps;
                            float r = inverse_root(mean), m = vx * r * of_all, h = 1.f;
                            if (!holds(mean) || !holds(fabsf(vx))) {  // also gradients of zero
                                h = half_scale_for(mean);
                                ss = vx = 0.f;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    x[i] *= h * h;
                                    ss = fmaf(x[i], x[i], ss);
                                }
                                r = inverse_root(group_sum<G>(ss) * of_all + p.eps * (h * h) * (h * h));
                                const float part = r * of_all;  // (a mean's parts: their sum may overflow)
#pragma unroll
                                for (int i = 0; i < 8; ++i) vx = fmaf(u[i] * gain[i], x[i] * part, vx);
                                m = group_sum<G>(vx);
                            }
                            // r h h is 1 / sqrt(mean), which need be no normal number
                            const float rh = r * h;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float n = x[i] * r;
                                y[i] = rh * (u[i] * gain[i] - n * m) * h;
                                sums[s][i] = fmaf(u[i], n, sums[s][i]);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) y[i] = u[i];
                        }
                    }
                    const uint64_t to = address(d.out, (row * d.out_row + h * d.out_head) * E);
#pragma unroll
                    for (int i = 0; i < 2; ++i) store4<BF16, MODE>(to, own.c[i], own.n[i], y + 4 * i);
                }
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
            const Share of = share_of<INTER>(p, at >> 3);
            if ((i & 3) >= of.n[i / 4] || !p.side[s].part) continue;
            float x = 0.f;
            for (int g = 0; g < GROUPS; ++g) x += all[s][g][at];
            p.side[s].part[(int64_t)blockIdx.x * p.D + of.c[i / 4] + (i & 3)] = x;
        }
    }
}

// Lanes of a head's row.
int group_of(int D, int pairs) {
    const int lanes = (pairs + 3) / 4 + (D - 2 * pairs + 7) / 8;
    return lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64;
}

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
    p.freq = a.freq;
    p.norm = a.norm;
    p.eps = a.eps;
    // Groups share a row, of which each makes the angles, where the rows alone are few
    // for the 4 workgroups of a CU, but one row and head each; every share has a query.
    const int groups = kThreads / group_of(a.D, p.pairs);
    const int64_t resident = (int64_t)4 * D->cu_count * groups;
    p.share = 1;
    while (2 * p.share <= a.heads && (a.rows * p.share < resident || (a.rows * p.share < 4 * resident && a.heads >= 8 * p.share)))
        p.share = 1 << ++p.log_share;
    p.items = a.rows * p.share;
    // Forward a group has one item, up to 2^14 workgroups a CU: 2^30 threads (the runtime
    // refuses 2^32).
    grid = grid_for(p.items, groups, D->cu_count, backward ? 4 : 1 << 14);
    return p;
}

template <bool BF16, bool INTER, bool BACKWARD, Mode MODE>
hipError_t launch_as(lattice_dense *D, const Params &p, unsigned grid) {
    const int g = MODE == ONES ? 4 : group_of(p.D, p.pairs);  // a row of three has two lanes at most
    const dim3 blocks(grid), threads(kThreads);
    if (g == 4) {
        hipLaunchKernelGGL((k_rotate<BF16, INTER, 4, MODE, BACKWARD>), blocks, threads, 0, D->stream, p);
    } else if constexpr (MODE != ONES) {
        if (g == 8)
            hipLaunchKernelGGL((k_rotate<BF16, INTER, 8, MODE, BACKWARD>), blocks, threads, 0, D->stream, p);
        else if (g == 16)
            hipLaunchKernelGGL((k_rotate<BF16, INTER, 16, MODE, BACKWARD>), blocks, threads, 0, D->stream, p);
        else if (g == 32)
            hipLaunchKernelGGL((k_rotate<BF16, INTER, 32, MODE, BACKWARD>), blocks, threads, 0, D->stream, p);
        else if constexpr (MODE == TAILS)
            hipLaunchKernelGGL((k_rotate<BF16, INTER, 64, MODE, BACKWARD>), blocks, threads, 0, D->stream, p);
    }
    return hipGetLastError();
}

template <bool BF16, bool INTER, bool BACKWARD>
hipError_t launch_mode(lattice_dense *D, const Params &p, unsigned grid) {
    if (p.D < 4) return launch_as<BF16, INTER, BACKWARD, ONES>(D, p, grid);
    // every lane of a group has eight values: no lane past them, no row's end inside
    if (p.pairs % 4 == 0 && (p.D - 2 * p.pairs) % 8 == 0 && p.D == 8 * group_of(p.D, p.pairs))
        return launch_as<BF16, INTER, BACKWARD, WHOLE>(D, p, grid);
    return launch_as<BF16, INTER, BACKWARD, TAILS>(D, p, grid);
}

template <bool BACKWARD>
hipError_t launch(lattice_dense *D, const RotateArgs &a, const Params &p, unsigned grid) {
    if (a.bf16) return a.interleaved ? launch_mode<true, true, BACKWARD>(D, p, grid) : launch_mode<true, false, BACKWARD>(D, p, grid);
    return a.interleaved ? launch_mode<false, true, BACKWARD>(D, p, grid) : launch_mode<false, false, BACKWARD>(D, p, grid);
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
