// Products of two matrices whose rows hold the contraction index next to each
// other, D[i][j] = sum_k A[i][k] B[j][k], on the bf16 matrix cores: the part
// that the loss (loss.hip) and the update (update.hip) share.
//
// An operand is P planes of bf16 whose sum is its value: one for values that
// are bf16, two (the upper 16 bits of a product's operands, errors below 2^-16)
// or three (24 bits, as exact as fp32) for fp32 ones.  Of the products of two
// sums the largest are taken: 1 of 1, 3 of 4, 6 of 9; sums are fp32.
//
// A workgroup computes a BM x BN tile.  Operand slices of BK values a row go
// from memory straight into LDS (16 bytes a lane), one slice ahead of the one
// that is multiplied, and from there as 16-byte reads into
// v_mfma_f32_32x32x16_bf16.  16-byte chunks of the rows are XOR-swizzled so
// that 16 consecutive rows read at one chunk index hit 16 different 16-byte
// bank groups.
//
// The caller's matrices are padded: a row holds a multiple of 64 values with
// zeros after its K.  Rows past an operand's last are not read (the last one
// stands in, and the epilogue drops what comes of it).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

// Each source file that includes this gets its own copy of the kernels.
namespace gemm {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kPad = 64;  // rows of operands hold a multiple of this many values
inline int64_t padded(int64_t k) { return (k + kPad - 1) / kPad * kPad; }

// bf16 planes [P][rows][ld] of each of a batch.  ld < kMaxLd: offsets within a
// tile are 32 bits.
constexpr int64_t kMaxLd = (int64_t)1 << 23;
struct Operand {
    const uint16_t *p;
    int64_t ld, plane, batch;
    int rows;
};

struct Shape {
    int K;         // contraction length, a multiple of kPad
    int k_split;   // the part of it that one of gridDim.y takes, a multiple of kPad
    int tiles_m, tiles_n;
    bool lower;    // square and symmetric: only tiles with tile_m >= tile_n
};

template <int BM_, int BN_, int WM_, int WN_, int BK_, int P_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, P = P_;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 blocks of a wavefront
    static constexpr int CPR = BK / 8;                          // 16-byte chunks of a row of a slice
    static constexpr int SLICE = P * (BM + BN) * CPR * 16;      // bytes
    static constexpr int STAGES = 2;
    static constexpr int LDS = STAGES * SLICE;
    static constexpr int INSTR = P * (BM + BN) * CPR / 64;      // direct loads of a slice, one per wavefront each
    static constexpr int DMA = INSTR / NW;
    static constexpr int RPI = 64 / CPR;                        // rows of one such load
    static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "wavefront blocks");
    static_assert(INSTR % NW == 0 && BM % RPI == 0 && BN % RPI == 0, "direct loads");
    static_assert((BK == 64 || BK == 32) && kPad % BK == 0, "slice");
    static_assert(LDS <= 160 * 1024, "LDS");
    __device__ static __forceinline__ int key(int row) { return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }
};

// 16 bytes a lane from memory to 1024 bytes of LDS.
__device__ __forceinline__ void dma16(const void *src, char *lds_wave_base) {
    __builtin_amdgcn_global_load_lds(src, (lds_void *)lds_wave_base, 16, 0, 0);
}
// Wait for this wavefront's memory operations, then the workgroup barrier.
__device__ __forceinline__ void drain_and_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Where a wavefront's accumulators lie: register e of block (i, j) of lane l is
// row  row0 + 32 i + 8 (e / 4) + 4 (l / 32) + e % 4, column col0 + 32 j + l % 32.
struct Place {
    int row0, col0;  // of this wavefront's blocks
    int tile_m, tile_n, split, batch;
};

__device__ __forceinline__ int acc_row(int e) { return 8 * (e >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (e & 3); }

// Tile of workgroup b: consecutive workgroups of an XCD take the tiles of a
// band of 8 tile rows, so that its L2 holds the operands they share.
__device__ __forceinline__ void tile_of(const Shape &s, int64_t b, int &tm, int &tn) {
    if (s.lower) {  // row r has r + 1 tiles
        int r = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
        while ((int64_t)(r + 1) * (r + 2) / 2 <= b) ++r;
        while ((int64_t)r * (r + 1) / 2 > b) --r;
        tm = r;
        tn = (int)(b - (int64_t)r * (r + 1) / 2);
        return;
    }
    const int band = 8;
    const int per = band * s.tiles_n;
    const int first = (int)(b / per) * band;
    const int high = s.tiles_m - first < band ? s.tiles_m - first : band;
    const int in = (int)(b % per);
    tm = first + in % high;
    tn = in / high;
}

template <class T, class Epilogue>
__global__ __launch_bounds__(T::THREADS) void k_gemm(Operand A, Operand B, Shape s, Epilogue epi) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = wave_index();
    Place at;
    tile_of(s, xcd_order(blockIdx.x, gridDim.x), at.tile_m, at.tile_n);
    at.split = blockIdx.y;
    at.batch = blockIdx.z;
    const int m0 = at.tile_m * T::BM, n0 = at.tile_n * T::BN;
    const int wm = wave / T::WN, wn = wave % T::WN;
    at.row0 = m0 + wm * 32 * T::TM;
    at.col0 = n0 + wn * 32 * T::TN;
    const int k0 = blockIdx.y * s.k_split;
    const int k1 = k0 + s.k_split < s.K ? k0 + s.k_split : s.K;

    // This wavefront's direct loads: load d brings RPI rows of one plane of A
    // or B.  Lane l's 16 bytes land at chunk l of the load's 1024 bytes; it
    // reads the chunk that the swizzle puts there.
    const char *base[T::DMA];
    uint32_t off[T::DMA];
#pragma unroll
    for (int d = 0; d < T::DMA; ++d) {
        const int instr = wave + T::NW * d;
        const int plane = instr / ((T::BM + T::BN) / T::RPI);
        const int r0 = instr % ((T::BM + T::BN) / T::RPI) * T::RPI;  // row of the plane's BM + BN
        const bool is_b = r0 >= T::BM;
        const Operand &o = is_b ? B : A;
        const int first = is_b ? n0 : m0;
        int r = r0 + lane / T::CPR;
        const int chunk = (lane % T::CPR) ^ T::key(r);
        r -= is_b ? T::BM : 0;
        if (first + r > o.rows - 1) r = o.rows - 1 - first;
        base[d] = reinterpret_cast<const char *>(o.p + at.batch * o.batch + plane * o.plane + (int64_t)first * o.ld + k0);
        off[d] = (uint32_t)r * (uint32_t)(o.ld * 2) + chunk * 16;
    }
    auto issue = [&](int buf, int step) {
#pragma unroll
        for (int d = 0; d < T::DMA; ++d)
            dma16(base[d] + (int64_t)step * (T::BK * 2) + off[d], lds + buf * T::SLICE + (wave + T::NW * d) * 1024);
    };

    f32x16_t acc[T::TM][T::TN];
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int steps = (k1 - k0) / T::BK;
    const int ar = wm * 32 * T::TM + (lane & 31), br = T::BM + wn * 32 * T::TN + (lane & 31);
    issue(0, 0);
    for (int step = 0; step < steps; ++step) {
        // this slice is there, and the other buffer is read no more
        drain_and_barrier();
        if (step + 1 < steps) issue((step + 1) & 1, step + 1);
        const char *slice = lds + (step & 1) * T::SLICE;
#pragma unroll
        for (int kk = 0; kk < T::BK / 16; ++kk) {
            bf16x8_t a[T::P][T::TM], b[T::P][T::TN];
            const int chunk = 2 * kk + (lane >> 5);
#pragma unroll
            for (int p = 0; p < T::P; ++p) {
                const char *plane = slice + p * (T::BM + T::BN) * T::CPR * 16;
#pragma unroll
                for (int i = 0; i < T::TM; ++i)
                    a[p][i] = *reinterpret_cast<const bf16x8_t *>(
                        plane + ((ar + 32 * i) * T::CPR + (chunk ^ T::key(ar + 32 * i))) * 16);
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
                    b[p][j] = *reinterpret_cast<const bf16x8_t *>(
                        plane + ((br + 32 * j) * T::CPR + (chunk ^ T::key(br + 32 * j))) * 16);
            }
            // the smaller products first
#pragma unroll
            for (int t = T::P - 1; t >= 0; --t)
#pragma unroll
                for (int p = 0; p <= t; ++p)
#pragma unroll
                    for (int i = 0; i < T::TM; ++i)
#pragma unroll
                        for (int j = 0; j < T::TN; ++j)
                            acc[i][j] = mfma(a[p][i], b[t - p][j], acc[i][j]);
        }
    }
    // the epilogue may use the slices' LDS
    drain_and_barrier();
    epi.template run<T>(acc, at, lds);
}

template <class T, class Epilogue>
hipError_t launch(hipStream_t stream, const Operand &A, const Operand &B, int64_t K, int64_t k_split, int64_t batch,
                  bool lower, const Epilogue &epi) {
    if (A.rows <= 0 || B.rows <= 0 || batch <= 0) return hipSuccess;
    Shape s;
    s.K = (int)K;
    s.k_split = (int)k_split;
    s.tiles_m = (A.rows + T::BM - 1) / T::BM;
    s.tiles_n = (B.rows + T::BN - 1) / T::BN;
    s.lower = lower;
    const int64_t tiles = lower ? (int64_t)s.tiles_m * (s.tiles_m + 1) / 2 : (int64_t)s.tiles_m * s.tiles_n;
    const int64_t parts = (K + s.k_split - 1) / s.k_split;
    constexpr int LDS = T::LDS > Epilogue::template lds<T>() ? T::LDS : Epilogue::template lds<T>();
    if (LDS > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_gemm<T, Epilogue>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_gemm<T, Epilogue>), dim3((unsigned)tiles, (unsigned)parts, (unsigned)batch), dim3(T::THREADS),
                       LDS, stream, A, B, s, epi);
    return hipGetLastError();
}

// The length of a part when a contraction of K is cut into at most `splits`.
inline int64_t part_length(int64_t K, int64_t splits) { return padded((K + splits - 1) / splits); }

}  // namespace
}  // namespace gemm
