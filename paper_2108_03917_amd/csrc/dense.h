// Declarations shared by the dense operators (dense.hip: the host side;
// norm.hip, loss.hip, update.hip: the kernels).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

// In the launchers: pass a failure on.
#define TRY(expr)                          \
    do {                                   \
        const hipError_t e_ = (expr);      \
        if (e_ != hipSuccess) return e_;   \
    } while (0)

// Device status bits of a lattice_dense.
enum : int { DENSE_ST_LABEL = 1 };

// Scratch that a larger one has replaced while a graph may still use it.
struct KeptScratch {
    void *p;
    KeptScratch *next;
};

struct lattice_dense {
    int device = 0;
    hipStream_t stream = nullptr;
    int cu_count = 256;
    void *ws = nullptr;  // scratch of the operators, grown on demand
    int64_t ws_bytes = 0;
    bool split_gradients = false;  // d loss / dz of bf16 operands in 16 bits
    bool ws_captured = false;     // a call with this scratch was captured
    KeptScratch *kept = nullptr;  // freed with the handle
    int32_t *status = nullptr;       // device
    int32_t *host_status = nullptr;  // pinned
    char err[512] = {0};
};

// Offsets of the parts of an operator's scratch, each aligned to 256 bytes.
struct ScratchLayout {
    int64_t bytes = 0;
    int64_t take(int64_t n) {
        const int64_t at = bytes;
        bytes += (n + 255) & ~(int64_t)255;
        return at;
    }
};

// norm.hip
struct NormArgs {
    const int32_t *counters;  // of the lattice whose vertices the rows are, or null
    int64_t rows;
    int C;
    float eps;
    const void *x;
    int64_t x_stride;
    bool x_bf16;
    const float *gamma, *beta;
    void *y;
    int64_t y_stride;
    bool y_bf16;
    float *mean, *rstd;
};
hipError_t launch_layer_norm(lattice_dense *D, const NormArgs &a);

struct NormBackwardArgs {
    const int32_t *counters;
    int64_t rows;
    int C;
    const void *g;
    int64_t g_stride;
    bool g_bf16;
    const void *x;
    int64_t x_stride;
    bool x_bf16;
    const float *mean, *rstd, *gamma;
    void *gx;
    int64_t gx_stride;
    float *grad_gamma, *grad_beta;
};
int64_t layer_norm_backward_scratch(const lattice_dense *D, const NormBackwardArgs &a);
hipError_t launch_layer_norm_backward(lattice_dense *D, const NormBackwardArgs &a);

// loss.hip
struct LossArgs {
    bool bf16;  // storage of x, w and their gradients
    int64_t N;
    int C;
    const void *x;
    int64_t x_stride;
    const void *w;
    int K;
    int64_t w_stride;
    const float *bias;
    const int64_t *target;
    int64_t ignore;
    bool mean;
    float *loss, *rows;
    void *grad_x, *grad_w;
    float *grad_bias;
    bool split;  // bf16: G in two planes, where it is not anyway
    bool any_grad() const { return grad_x || grad_w || grad_bias; }
};
int64_t loss_scratch(const lattice_dense *D, const LossArgs &a);
hipError_t launch_loss(lattice_dense *D, const LossArgs &a);

// loss_fused.hip: few classes and channels
bool loss_fused_covers(const LossArgs &a);
int64_t loss_fused_scratch(const lattice_dense *D, const LossArgs &a);
hipError_t launch_loss_fused(lattice_dense *D, const LossArgs &a);

// update.hip
struct UpdateArgs {
    const void *g;
    bool g_bf16;
    int64_t batch;
    int m, n;
    int64_t batch_stride, row_stride;
    int steps;
    float coef[3];
    float eps;
    void *out;
    bool out_bf16;
};
int64_t update_scratch(const lattice_dense *D, const UpdateArgs &a);
hipError_t launch_update(lattice_dense *D, const UpdateArgs &a);

// Sixteen or fewer bytes of consecutive values, at the alignment of one value.
struct __attribute__((packed, aligned(4))) Words4 { uint32_t v[4]; };
struct __attribute__((packed, aligned(2))) Halves8 { uint32_t v[4]; };

// Eight or four consecutive channels of a row as they are stored.
template <bool BF16, int VEC>
struct Raw {
    static_assert(BF16 ? VEC == 8 : VEC == 4 || VEC == 8, "channels per load");
    uint32_t w[BF16 ? 4 : VEC];
};

// Channels c0.. of a row of C channels; those past C are 0.  A row may start at
// any multiple of its element's size: the vector loads of this chip take any
// such address.
template <bool BF16, int VEC>
__device__ __forceinline__ void load_raw(const void *row, int c0, int C, Raw<BF16, VEC> &u) {
    constexpr int WORDS = BF16 ? 4 : VEC;
    if (c0 + VEC <= C) {
        if constexpr (BF16) {
            const Halves8 t = *reinterpret_cast<const Halves8 *>(reinterpret_cast<const uint16_t *>(row) + c0);
#pragma unroll
            for (int i = 0; i < 4; ++i) u.w[i] = t.v[i];
        } else {
#pragma unroll
            for (int h = 0; h < VEC / 4; ++h) {
                const Words4 t = *reinterpret_cast<const Words4 *>(reinterpret_cast<const float *>(row) + c0 + 4 * h);
#pragma unroll
                for (int i = 0; i < 4; ++i) u.w[4 * h + i] = t.v[i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            u.w[i] = 0;
            if (BF16) {
                if (c0 + 2 * i < C) u.w[i] = reinterpret_cast<const uint16_t *>(row)[c0 + 2 * i];
                if (c0 + 2 * i + 1 < C) u.w[i] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c0 + 2 * i + 1] << 16;
            } else {
                if (c0 + i < C) u.w[i] = reinterpret_cast<const uint32_t *>(row)[c0 + i];
            }
        }
    }
}
template <bool BF16, int VEC>
__device__ __forceinline__ void unpack(const Raw<BF16, VEC> &u, float *v) {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        v[i] = __uint_as_float(!BF16 ? u.w[BF16 ? 0 : i] : (i & 1) ? u.w[i / 2] & 0xffff0000u : u.w[i / 2] << 16);
}

// The same as fp32.
template <bool BF16, int VEC>
__device__ __forceinline__ void load_row(const void *row, int c0, int C, float *v) {
    Raw<BF16, VEC> u;
    load_raw<BF16, VEC>(row, c0, C, u);
    unpack<BF16, VEC>(u, v);
}

// The reverse: values rounded to nearest even where the row is bf16.
template <bool BF16, int VEC>
__device__ __forceinline__ void store_row(void *row, int c0, int C, const float *v) {
    if (c0 + VEC <= C) {
        if constexpr (BF16) {
            Halves8 u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u.v[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<Halves8 *>(reinterpret_cast<uint16_t *>(row) + c0) = u;
        } else {
#pragma unroll
            for (int h = 0; h < VEC / 4; ++h) {
                Words4 u;
#pragma unroll
                for (int i = 0; i < 4; ++i) u.v[i] = __float_as_uint(v[4 * h + i]);
                *reinterpret_cast<Words4 *>(reinterpret_cast<float *>(row) + c0 + 4 * h) = u;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (c0 + i < C) {
                if (BF16)
                    reinterpret_cast<uint16_t *>(row)[c0 + i] = (uint16_t)pack_bf16(v[i], 0.f);
                else
                    reinterpret_cast<float *>(row)[c0 + i] = v[i];
            }
    }
}
