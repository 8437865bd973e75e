// The classifier loss and its gradients for few classes and channels (the
// labels of a segmentation), in one pass over the rows: see loss.hip for the
// formulas and for everything larger.
//
// A workgroup of four wavefronts takes 64 rows at a time, 16 a wavefront, with
// all of w in LDS.  Per wavefront, with rows x of the block and lane (i, q) =
// (lane % 16, lane / 16):
//   z^T = w x^T        lane (i, q) gets classes 16 t + 4 q + r of row i, so the
//                      softmax of a row is over registers and four lanes
//   G = p - [k = t]    stays in those registers as an operand of
//   dx^T = w^T G^T     (the classes in the order that the lanes hold them)
// and through LDS, over the workgroup's 64 rows,
//   dw += G^T x        each wavefront a quarter of the channels, in registers
//                      from the first block to the last.
// So x is read once and dx written once, which is what bounds it on large
// clouds; a workgroup's dw, db and loss go out once, as one row of partial
// sums, and k_fused_join adds the rows in a fixed order in fp64.
//
// fp32 operands are multiplied on the fp32 matrix cores (16x16x4: exact
// products), bf16 ones on the bf16 ones (16x16x32), where a value of G is the sum
// of two bf16 (16 bits): rounded to one, the gradients' error against 64 bits was
// 2.1e-3, of which the rounding of the stored result alone makes 1.7e-3.  The
// second one costs 2% (103889 x 128 with 20 classes: 30.6 and 31.3 us a call) to 13%
// (100000 x 128 with 100: 77 and 87).
//
// 537211 x 64 with 20 classes in fp32: 91 us (3.0 TB/s of x and dx; the fp32
// matrix cores, half busy, and the exponentials do not hide all of it).
// 103889 x 128 with 20 classes in bf16: 25 us (2.1 TB/s) in three workgroups a CU,
// which its 135 registers a lane and its 47 KB of LDS both allow: 1624 blocks
// are 2.1 rounds of them and take 3, and the transposed parts go to LDS two bytes a
// lane at a time.  The next block's rows are read while a block is multiplied.
#include "planes.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRows = 64;           // rows of a block
constexpr int kCounts = 256;        // partial counts of rows with a label
constexpr int kParts = 2;           // bf16 that a value of G is the sum of
// Those of them whose transposed matrices are in LDS at a time: one after the
// other where room for both would leave a CU one workgroup instead of two (100000
// x 256 with 20 classes in bf16: 49 us, 56 at once).
__host__ __device__ constexpr int parts_at_once(int KT, int CT4) { return KT == 2 && CT4 == 4 ? 1 : kParts; }
constexpr int64_t kCountHere = 8192;  // up to so many rows every workgroup counts them itself

__device__ __forceinline__ f32x4_t mfma4(float a, float b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma32(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}

struct FusedArgs {
    LossArgs a;
    const int32_t *count;  // partial counts, or null: count here
    float *part;           // [gridDim.x][K C + K + 1]
    int32_t *status;
};

__device__ __forceinline__ bool has_label(int64_t t, int K, int64_t ignore) { return t != ignore && t >= 0 && t < K; }

// Rows with a label (of all N), for every thread of the workgroup.
__device__ __forceinline__ int64_t labelled(const FusedArgs &f, int64_t *red) {
    int64_t n = 0;
    if (f.count) {
        n = f.count[threadIdx.x];
    } else {
        for (int64_t i = threadIdx.x; i < f.a.N; i += 256) n += has_label(f.a.target[i], f.a.K, f.a.ignore);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

// Softmax of a row whose logits lie in the registers of four lanes (q = 0..3),
// class 16 t + 4 q + r in z[t][r]: turns them into G and returns the row's
// loss.  Without a label G is 0 and so is the loss.
template <int KT>
__device__ __forceinline__ float softmax(f32x4_t (&z)[KT], int label, bool has) {
    const int q = (threadIdx.x & 63) >> 4;
    float top = -INFINITY, picked = 0.f;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            top = fmaxf(top, z[t][r]);
            picked = 16 * t + 4 * q + r == label ? z[t][r] : picked;
        }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float ref = top == -INFINITY ? 0.f : top;
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            z[t][r] = __expf(z[t][r] - ref);
            s += z[t][r];
        }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    // the three lanes without the label's class add 0
    picked += __shfl_xor(picked, 16);
    picked += __shfl_xor(picked, 32);
    const float inv = 1.f / s;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float p = z[t][r] * inv - (16 * t + 4 * q + r == label ? 1.f : 0.f);
            z[t][r] = has ? p : 0.f;
        }
    return has ? top + logf(s) - picked : 0.f;
}

// Adds a value over the 16 lanes of a quarter wavefront.
__device__ __forceinline__ float sum16(float v) {
#pragma unroll
    for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// What both kernels do at the end: the workgroup's row of partial sums.
template <int KT, int CT4, bool GRAD>
__device__ __forceinline__ void write_part(const FusedArgs &f, const f32x4_t (&dw)[CT4][KT], f32x4_t (&db)[KT],
                                           double loss, float factor, float *red) {
    const LossArgs &a = f.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    float *row = f.part + (int64_t)blockIdx.x * ((int64_t)a.K * a.C + a.K + 1);
    if (GRAD && a.grad_w) {
#pragma unroll
        for (int c = 0; c < CT4; ++c)
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int k = 16 * t + 4 * q + r, ch = 16 * (wave + 4 * c) + i;
                    if (k < a.K && ch < a.C) row[(int64_t)k * a.C + ch] = dw[c][t][r] * factor;
                }
    }
    __syncthreads();
    if (GRAD && a.grad_bias) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float s = sum16(db[t][r]);
                if (i == 0) red[wave * KT * 16 + 16 * t + 4 * q + r] = s;
            }
        __syncthreads();
        for (int k = threadIdx.x; k < a.K; k += 256) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) s += red[w * KT * 16 + k];
            row[(int64_t)a.K * a.C + k] = s * factor;
        }
    }
    // the lanes of a quarter hold their rows' losses (those of q > 0 are copies)
    if (q > 0) loss = 0.0;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) loss += __shfl_xor(loss, d);
    double *dred = reinterpret_cast<double *>(red);
    __syncthreads();
    if (lane == 0) dred[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0)
        row[(int64_t)a.K * a.C + a.K] = (float)((dred[0] + dred[1] + dred[2] + dred[3]) * (double)factor);
}

// LDS layouts.  Rows of w and x are padded so that 16 rows read at one 16-byte
// chunk, and four rows read at 16 consecutive words, hit different banks.
struct Lds32 {
    int cp, ws, xs, gs;
    __host__ __device__ Lds32(int C, int KT) : cp((C + 15) / 16 * 16), ws(cp + 4), xs(cp + 20), gs(KT * 16 + 20) {}
    __host__ __device__ int floats(int KT, bool grad) const {
        return KT * 16 * (ws + 1) + (grad ? kRows * (xs + gs) : 0) + 4 * KT * 16 + 16;
    }
};

template <int KT, int CT4, bool GRAD>
__global__ __launch_bounds__(256) void k_fused_f32(FusedArgs f) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const LossArgs &a = f.a;
    const Lds32 L(a.C, KT);
    float *W = lds, *B = W + KT * 16 * L.ws, *red = B + KT * 16, *X = red + 4 * KT * 16 + 16, *G = X + kRows * L.xs;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int ct = L.cp / 16;
    {
        // a row of w by as many threads as it has values, up to 64
        const int wide = L.cp < 64 ? (L.cp <= 16 ? 16 : 32) : 64, c0 = threadIdx.x & (wide - 1);
        for (int c = c0; c < L.cp; c += wide)
#pragma unroll 4
            for (int k = threadIdx.x / wide; k < KT * 16; k += 256 / wide)
                W[k * L.ws + c] = k < a.K && c < a.C ? reinterpret_cast<const float *>(a.w)[k * a.w_stride + c] : 0.f;
    }
    for (int k = threadIdx.x; k < KT * 16; k += 256) B[k] = k < a.K ? (a.bias ? a.bias[k] : 0.f) : -INFINITY;
    float factor = 1.f;
    if (a.mean) {
        const int64_t n = labelled(f, reinterpret_cast<int64_t *>(red));
        factor = n > 0 ? (float)(1.0 / (double)n) : 0.f;
    }
    __syncthreads();
    f32x4_t dw[CT4][KT], db[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        db[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CT4; ++c) dw[c][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    double loss = 0.0;
    bool bad = false;
    // A block's rows are read while the one before it is worked on, into the
    // registers that its logits have just freed.
    float x[CT4 * 4][4];
    int64_t target;
    auto read = [&](int64_t p) {
        const float *xr = reinterpret_cast<const float *>(a.x) + (p < a.N ? p : a.N - 1) * a.x_stride;
#pragma unroll
        for (int t = 0; t < CT4 * 4; ++t) load_row<false, 4>(xr, 16 * t + 4 * q, a.C, x[t]);
        target = p < a.N ? a.target[p] : a.ignore;
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    if ((int64_t)blockIdx.x * kRows < a.N) read((int64_t)blockIdx.x * kRows + 16 * wave + i);
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.N; r0 += step) {
        const int64_t p = r0 + 16 * wave + i;
        const bool has = has_label(target, a.K, a.ignore);
        bad |= !has && target != a.ignore;
        const int label = has ? (int)target : -1;
        f32x4_t z[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) z[t] = *reinterpret_cast<const f32x4_t *>(B + 16 * t + 4 * q);
#pragma unroll
        for (int t = 0; t < CT4 * 4; ++t) {
            if (t >= ct) continue;
            float4 v = make_float4(x[t][0], x[t][1], x[t][2], x[t][3]);
            // whatever a row without a label holds
            if (!has) v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (GRAD) *reinterpret_cast<float4 *>(X + (16 * wave + i) * L.xs + 16 * t + 4 * q) = v;
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                const float4 w = *reinterpret_cast<const float4 *>(W + (16 * k + i) * L.ws + 16 * t + 4 * q);
                z[k] = mfma4(w.x, v.x, z[k]);
                z[k] = mfma4(w.y, v.y, z[k]);
                z[k] = mfma4(w.z, v.z, z[k]);
                z[k] = mfma4(w.w, v.w, z[k]);
            }
        }
        if (r0 + step < a.N) read(p + step);
        const float l = softmax<KT>(z, label, has);
        loss += l;
        if (a.rows && q == 0 && p < a.N) a.rows[p] = l;
        if (!GRAD) continue;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            db[k] += z[k];
            *reinterpret_cast<f32x4_t *>(G + (16 * wave + i) * L.gs + 16 * k + 4 * q) = z[k];
        }
        if (a.grad_x) {
            float *gr = reinterpret_cast<float *>(a.grad_x) + p * a.C;
#pragma unroll
            for (int c = 0; c < CT4 * 4; ++c) {
                if (c >= ct) continue;
                f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        o = mfma4(W[(16 * k + 4 * q + r) * L.ws + 16 * c + i], z[k][r], o);
                const float v[4] = {o[0] * factor, o[1] * factor, o[2] * factor, o[3] * factor};
                if (p < a.N) store_row<false, 4>(gr, 16 * c + 4 * q, a.C, v);
            }
        }
        if (!a.grad_w) continue;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CT4; ++c) {
            if (wave + 4 * c >= ct) continue;
#pragma unroll 4
            for (int s = 0; s < kRows / 4; ++s) {
                const float v = X[(4 * s + q) * L.xs + 16 * (wave + 4 * c) + i];
#pragma unroll
                for (int k = 0; k < KT; ++k) dw[c][k] = mfma4(G[(4 * s + q) * L.gs + 16 * k + i], v, dw[c][k]);
            }
        }
        __syncthreads();
    }
    if (bad) atomicOr(f.status, DENSE_ST_LABEL);
    write_part<KT, CT4, GRAD>(f, dw, db, loss, factor, red);
}

// bf16: classes are held in pairs of 16 (u), a lane's eight being 32 u + 4 q +
// {0..3} and 32 u + 16 + 4 q + {0..3}: V holds w^T with its classes in that
// order.  Gt and Xt are G^T and x^T of the block.
struct Lds16 {
    int cp, ws, vs;
    static constexpr int rs = kRows + 8;
    __host__ __device__ Lds16(int C, int KT) : cp((C + 31) / 32 * 32), ws(cp + 8), vs(KT * 16 + 8) {}
    // in bytes: w, V, G^T and x^T, biases and the sums
    __host__ __device__ int bytes(int KT, int CT4, bool grad) const {
        return 2 * KT * 16 * ws + (grad ? 2 * cp * vs + 2 * (parts_at_once(KT, CT4) * KT * 16 + cp) * rs : 0) +
               4 * (5 * KT * 16 + 16);
    }
};

template <int KT, int CT4, bool GRAD>
__global__ __launch_bounds__(256) void k_fused_bf16(FusedArgs f) {
    extern __shared__ __attribute__((aligned(16))) uint16_t lds16[];
    const LossArgs &a = f.a;
    const Lds16 L(a.C, KT);
    constexpr int HELD = parts_at_once(KT, CT4);
    uint16_t *W = lds16, *V = W + KT * 16 * L.ws;
    uint16_t *Gt = V + (GRAD ? L.cp * L.vs : 0), *Xt = Gt + (GRAD ? HELD * KT * 16 * L.rs : 0);
    float *B = reinterpret_cast<float *>(Xt + (GRAD ? L.cp * L.rs : 0)), *red = B + KT * 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int ct = (a.C + 15) / 16, cs = L.cp / 32;
    {
        const int wide = L.cp < 64 ? 32 : 64, c0 = threadIdx.x & (wide - 1);
        for (int c = c0; c < L.cp; c += wide)
#pragma unroll 4
            for (int k = threadIdx.x / wide; k < KT * 16; k += 256 / wide) {
                const uint16_t v = k < a.K && c < a.C ? reinterpret_cast<const uint16_t *>(a.w)[k * a.w_stride + c] : 0;
                W[k * L.ws + c] = v;
                // class 32 u + 16 h + 4 j + r lies at 32 u + 8 j + 4 h + r
                if (GRAD) V[c * L.vs + (k & ~31) + ((k >> 2) & 3) * 8 + ((k >> 4) & 1) * 4 + (k & 3)] = v;
            }
    }
    for (int k = threadIdx.x; k < KT * 16; k += 256) B[k] = k < a.K ? (a.bias ? a.bias[k] : 0.f) : -INFINITY;
    float factor = 1.f;
    if (a.mean) {
        const int64_t n = labelled(f, reinterpret_cast<int64_t *>(red));
        factor = n > 0 ? (float)(1.0 / (double)n) : 0.f;
    }
    __syncthreads();
    f32x4_t dw[CT4][KT], db[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        db[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CT4; ++c) dw[c][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    double loss = 0.0;
    bool bad = false;
    // A block's rows are read while the one before it is worked on, into the
    // registers that its logits have just freed.
    Raw<true, 8> x[CT4 * 2];
    int64_t target;
    auto read = [&](int64_t p) {
        const uint16_t *xr = reinterpret_cast<const uint16_t *>(a.x) + (p < a.N ? p : a.N - 1) * a.x_stride;
#pragma unroll
        for (int t = 0; t < CT4 * 2; ++t) load_raw<true, 8>(xr, 32 * t + 8 * q, a.C, x[t]);
        target = p < a.N ? a.target[p] : a.ignore;
    };
    const int64_t step = (int64_t)gridDim.x * kRows;
    if ((int64_t)blockIdx.x * kRows < a.N) read((int64_t)blockIdx.x * kRows + 16 * wave + i);
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.N; r0 += step) {
        const int64_t p = r0 + 16 * wave + i;
        const bool has = has_label(target, a.K, a.ignore);
        bad |= !has && target != a.ignore;
        const int label = has ? (int)target : -1;
        f32x4_t z[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) z[t] = *reinterpret_cast<const f32x4_t *>(B + 16 * t + 4 * q);
#pragma unroll
        for (int t = 0; t < CT4 * 2; ++t) {
            if (t >= cs) continue;
            // whatever a row without a label holds
            const u32x4_t v = has ? u32x4_t{x[t].w[0], x[t].w[1], x[t].w[2], x[t].w[3]} : u32x4_t{0, 0, 0, 0};
            if (GRAD)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    Xt[(32 * t + 8 * q + j) * L.rs + 16 * wave + i] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
#pragma unroll
            for (int k = 0; k < KT; ++k)
                z[k] = mfma32(*reinterpret_cast<const u32x4_t *>(W + (16 * k + i) * L.ws + 32 * t + 8 * q), v, z[k]);
        }
        if (r0 + step < a.N) read(p + step);
        const float l = softmax<KT>(z, label, has);
        loss += l;
        if (a.rows && q == 0 && p < a.N) a.rows[p] = l;
        if (!GRAD) continue;
        u32x4_t g[kParts][KT / 2];
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            db[k] += z[k];
            uint32_t lo[kParts], hi[kParts];
            planes::split_pair<kParts>(z[k][0], z[k][1], lo);
            planes::split_pair<kParts>(z[k][2], z[k][3], hi);
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                g[p][k / 2][2 * (k & 1)] = lo[p];
                g[p][k / 2][2 * (k & 1) + 1] = hi[p];
            }
        }
        // parts `first` on of G^T
        auto transposed = [&](int first) {
#pragma unroll
            for (int p = 0; p < HELD; ++p)
#pragma unroll
                for (int k = 0; k < KT; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        Gt[(16 * (KT * p + k) + 4 * q + r) * L.rs + 16 * wave + i] =
                            (uint16_t)(g[first + p][k / 2][2 * (k & 1) + (r >> 1)] >> (16 * (r & 1)));
        };
        if (a.grad_w) transposed(kParts - HELD);
        if (a.grad_x) {
            uint16_t *gr = reinterpret_cast<uint16_t *>(a.grad_x) + p * a.C;
#pragma unroll
            for (int c = 0; c < CT4 * 4; ++c) {
                if (c >= ct) continue;
                f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < KT / 2; ++u) {
                    const u32x4_t v = *reinterpret_cast<const u32x4_t *>(V + (16 * c + i) * L.vs + 32 * u + 8 * q);
#pragma unroll
                    for (int p = kParts - 1; p >= 0; --p) o = mfma32(v, g[p][u], o);
                }
                const int c0 = 16 * c + 4 * q;
                if (p >= a.N) continue;
                const uint32_t lo = pack_bf16(o[0] * factor, o[1] * factor), hi = pack_bf16(o[2] * factor, o[3] * factor);
                if (c0 + 4 <= a.C) {
                    struct __attribute__((packed, aligned(2))) Two { uint32_t v[2]; };
                    *reinterpret_cast<Two *>(gr + c0) = Two{{lo, hi}};
                } else {
#pragma unroll
                    for (int j = 0; j < 3; ++j)
                        if (c0 + j < a.C) gr[c0 + j] = (uint16_t)((j < 2 ? lo : hi) >> (16 * (j & 1)));
                }
            }
        }
        if (!a.grad_w) continue;
#pragma unroll
        for (int first = kParts - HELD; first >= 0; first -= HELD) {  // the smaller parts first
            if (first != kParts - HELD) transposed(first);
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CT4; ++c) {
                if (wave + 4 * c >= ct) continue;
#pragma unroll
                for (int s = 0; s < kRows / 32; ++s) {
                    const u32x4_t v =
                        *reinterpret_cast<const u32x4_t *>(Xt + (16 * (wave + 4 * c) + i) * L.rs + 32 * s + 8 * q);
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int p = HELD - 1; p >= 0; --p)
                            dw[c][k] = mfma32(*reinterpret_cast<const u32x4_t *>(
                                                  Gt + (16 * (KT * p + k) + i) * L.rs + 32 * s + 8 * q),
                                              v, dw[c][k]);
                }
            }
            __syncthreads();
        }
    }
    if (bad) atomicOr(f.status, DENSE_ST_LABEL);
    write_part<KT, CT4, GRAD>(f, dw, db, loss, factor, red);
}

// Rows with a label, per workgroup.
__global__ __launch_bounds__(256) void k_fused_count(const int64_t *__restrict__ target, int64_t N, int K,
                                                     int64_t ignore, int32_t *count) {
    int n = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N; i += (int64_t)gridDim.x * 256)
        n += has_label(target[i], K, ignore);
    __shared__ int red[4];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) count[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// Column sums of the partial rows: dw, db, loss.  A workgroup takes 16 columns,
// 64 threads each, in fp64.
template <bool BF16>
__global__ __launch_bounds__(1024) void k_fused_join(const float *__restrict__ part, int rows, int64_t nw, int K,
                                                     void *grad_w, float *grad_bias, float *loss, int64_t first) {
    __shared__ double red[1024];
    const int64_t n = nw + K + 1;
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t j = first + (int64_t)blockIdx.x * 16 + c;
    double s = 0.0;
    if (j < n)
        for (int r = g; r < rows; r += 64) s += (double)part[(int64_t)r * n + j];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int h = 32; h > 0; h /= 2) {
        if (g < h) red[threadIdx.x] += red[threadIdx.x + h * 16];
        __syncthreads();
    }
    if (g > 0 || j >= n) return;
    const float v = (float)red[threadIdx.x];
    if (j < nw) {
        if (!grad_w) return;
        if (BF16)
            reinterpret_cast<uint16_t *>(grad_w)[j] = (uint16_t)pack_bf16(v, 0.f);
        else
            reinterpret_cast<float *>(grad_w)[j] = v;
    } else if (j < nw + K) {
        if (grad_bias) grad_bias[j - nw] = v;
    } else {
        *loss = v;
    }
}

int class_tiles(bool bf16, int K) { return K <= 16 && !bf16 ? 1 : K <= 32 ? 2 : K <= 64 ? 4 : 8; }
int channel_groups(int C) { return C <= 64 ? 1 : C <= 128 ? 2 : 4; }

int lds_bytes(const LossArgs &a) {
    const int KT = class_tiles(a.bf16, a.K);
    return a.bf16 ? Lds16(a.C, KT).bytes(KT, channel_groups(a.C), a.any_grad())
                  : Lds32(a.C, KT).floats(KT, a.any_grad()) * 4;
}

unsigned fused_grid(const lattice_dense *D, const LossArgs &a) {
    // as many workgroups as are resident at once
    int per_cu = 160 * 1024 / lds_bytes(a);
    if (per_cu > 4) per_cu = 4;
    return grid_for(a.N, kRows, D->cu_count, per_cu);
}

#define FUSED_SHAPES(X) \
    X(1, 1) X(1, 2) X(1, 4) X(2, 1) X(2, 2) X(2, 4) X(4, 1) X(4, 2) X(4, 4) X(8, 1) X(8, 2)

template <int KT, int CT4, bool GRAD>
hipError_t launch_shape(lattice_dense *D, const FusedArgs &f, unsigned grid) {
    const int lds = lds_bytes(f.a);
    // bf16 classes go in pairs of 16
    constexpr int KB = KT < 2 ? 2 : KT;
    const void *fn = f.a.bf16 ? reinterpret_cast<const void *>(&k_fused_bf16<KB, CT4, GRAD>)
                              : reinterpret_cast<const void *>(&k_fused_f32<KT, CT4, GRAD>);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    if (f.a.bf16)
        hipLaunchKernelGGL((k_fused_bf16<KB, CT4, GRAD>), dim3(grid), dim3(256), lds, D->stream, f);
    else
        hipLaunchKernelGGL((k_fused_f32<KT, CT4, GRAD>), dim3(grid), dim3(256), lds, D->stream, f);
    return hipGetLastError();
}

}  // namespace

// Up to 128 classes and 256 channels (not both), whose w, and for gradients a
// block's rows, fit into LDS.
bool loss_fused_covers(const LossArgs &a) {
    if (a.K > 128 || a.C > 256) return false;
    if (class_tiles(a.bf16, a.K) * channel_groups(a.C) > 16) return false;
    return lds_bytes(a) <= 160 * 1024;
}

int64_t loss_fused_scratch(const lattice_dense *D, const LossArgs &a) {
    return kCounts * 4 + (int64_t)fused_grid(D, a) * ((int64_t)a.K * a.C + a.K + 1) * 4;
}

hipError_t launch_loss_fused(lattice_dense *D, const LossArgs &a) {
    FusedArgs f = {a, nullptr, reinterpret_cast<float *>(reinterpret_cast<char *>(D->ws) + kCounts * 4), D->status};
    if (a.mean && a.N > kCountHere) {
        int32_t *count = reinterpret_cast<int32_t *>(D->ws);
        hipLaunchKernelGGL(k_fused_count, dim3(kCounts), dim3(256), 0, D->stream, a.target, a.N, a.K, a.ignore, count);
        f.count = count;
    }
    const unsigned grid = fused_grid(D, a);
    const int KT = class_tiles(a.bf16, a.K), CT4 = channel_groups(a.C);
    hipError_t e = hipSuccess;
#define GO(KT_, CT4_)             \
    if (KT == KT_ && CT4 == CT4_) \
        e = a.any_grad() ? launch_shape<KT_, CT4_, true>(D, f, grid) : launch_shape<KT_, CT4_, false>(D, f, grid);
    FUSED_SHAPES(GO)
#undef GO
    if (e != hipSuccess) return e;
    // without gradients only the last column was written
    const int64_t nw = (int64_t)a.K * a.C, n = nw + a.K + 1;
    const int64_t first = a.grad_w ? 0 : a.grad_bias ? nw : n - 1;
    const dim3 blocks((unsigned)((n - first + 15) / 16));
    if (a.bf16)
        hipLaunchKernelGGL(k_fused_join<true>, blocks, dim3(1024), 0, D->stream, f.part, (int)grid, nw, a.K, a.grad_w,
                           a.grad_bias, a.loss, first);
    else
        hipLaunchKernelGGL(k_fused_join<false>, blocks, dim3(1024), 0, D->stream, f.part, (int)grid, nw, a.K, a.grad_w,
                           a.grad_bias, a.loss, first);
    return hipGetLastError();
}
