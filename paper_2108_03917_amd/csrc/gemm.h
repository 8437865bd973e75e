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
// from memory straight into LDS (16 bytes a lane), STAGES - 1 slices ahead of
// the one that is multiplied, and from there as 16-byte reads into
// v_mfma_f32_32x32x16_bf16.  16-byte chunks of the rows are XOR-swizzled so
// that 16 consecutive rows read at one chunk index hit 16 different 16-byte
// bank groups.
//
// 8192 x 65536 over 1024 in bf16 with the loss's statistics in the epilogue:
// 1.0 ms, 1.1 PFLOP/s (a plain library product 1.6): reading the fragments and
// issuing the direct loads share the slots of the matrix instructions.
//
// The caller's matrices are padded: a row holds a multiple of 64 values with
// zeros after its K.  Rows past an operand's last are not read (the last one
// stands in, and the epilogue drops what comes of it).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

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
// Values from row to row of an operand laid out here: a row more than a
// multiple of 1 KB long is left out of step by 128 bytes, since rows at such
// distances fall on the same memory channels (a product with rows 128 KB apart
// took 338 us, see loss.hip, and 278 with this).
inline int64_t row_length(int64_t k) { return padded(k) % 512 == 0 ? padded(k) + 64 : padded(k); }

// bf16 planes [P][rows][ld] of each of a batch.  ld < kMaxLd: offsets within a
// tile are 32 bits.
constexpr int64_t kMaxLd = (int64_t)1 << 22;
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

template <int BM_, int BN_, int WM_, int WN_, int BK_, int P_, int STAGES_ = 2>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, P = P_;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 blocks of a wavefront
    static constexpr int CPR = BK / 8;                          // 16-byte chunks of a row of a slice
    static constexpr int SLICE = P * (BM + BN) * CPR * 16;      // bytes
    static constexpr int STAGES = STAGES_;
    static constexpr int LDS = STAGES * SLICE;
    static constexpr int RPI = 64 / CPR;                        // rows of a wavefront's direct load
    static constexpr int DMA_A = BM / RPI / NW, DMA_B = BN / RPI / NW;  // its loads of one plane's slice
    static constexpr int DMA = P * (DMA_A + DMA_B);
    static constexpr int PRODUCTS = P * (P + 1) / 2 * TM * TN, READS = P * (TM + TN);  // of 16 values
    static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "wavefront blocks");
    static_assert(BM % (RPI * NW) == 0 && BN % (RPI * NW) == 0, "direct loads");
    static_assert((BK == 64 || BK == 32) && kPad % BK == 0 && STAGES >= 2, "slice");
    static_assert(LDS <= 160 * 1024, "LDS");
    __device__ static __forceinline__ int key(int row) { return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }
};

typedef __amdgpu_buffer_rsrc_t rsrc_t;
// The 4 GiB from p on.
__device__ __forceinline__ rsrc_t buffer(const void *p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, -1, 0x00020000);
}
// 16 bytes a lane from memory (lane offset v, common offset s) to 1024 bytes of LDS.
__device__ __forceinline__ void dma16(rsrc_t from, uint32_t v, uint32_t s, char *lds_wave_base) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)lds_wave_base, 16, v, s, 0, 0);
}
// Wait until at most N of this wavefront's loads from memory are outstanding,
// and none of its LDS operations, then the workgroup barrier.
template <int N>
__device__ __forceinline__ void wait_and_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ __forceinline__ void sched_barrier() { __builtin_amdgcn_sched_barrier(0); }
// Orders what lies between two sched_barriers: the LDS reads among the first
// half of the products, so that they are done when the next ones want them, and
// the direct loads among the second, so that the matrix core never waits for a
// run of either to be issued.
template <int PRODUCTS, int READS, int LOADS, int I = 0>
__device__ __forceinline__ void interleave() {
    if constexpr (I < PRODUCTS) {
        constexpr int H = PRODUCTS / 2;
        constexpr int r = I < H ? (I + 1) * READS / H - I * READS / H : 0;
        constexpr int l = I < H ? 0 : (I + 1 - H) * LOADS / (PRODUCTS - H) - (I - H) * LOADS / (PRODUCTS - H);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
        if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x020, l, 0);
        interleave<PRODUCTS, READS, LOADS, I + 1>();
    }
}
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

// Workgroups go round robin to the eight XCDs: those of one XCD take consecutive
// tiles, also where the tiles are no multiple of eight.
__device__ __forceinline__ int64_t tile_order(int64_t b, int64_t n) {
    const int64_t x = b % 8, left = n % 8;
    return x * (n / 8) + (x < left ? x : left) + b / 8;
}

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

// An epilogue that wants nothing but the accumulators.
struct Simple {
    template <class T>
    static constexpr int lds() { return 0; }
    template <class T>
    static constexpr int extra() { return 0; }
    template <class T>
    __device__ __forceinline__ void begin(const Place &, char *) const {}
    // the accumulators start as zeros
    template <class T>
    __device__ __forceinline__ void init(f32x16_t (&)[T::TM][T::TN], const Place &) const {}
};

// LDS of the slices, which the epilogue may use after them.
template <class T, class Epilogue>
constexpr int room() { return T::LDS > Epilogue::template lds<T>() ? T::LDS : Epilogue::template lds<T>(); }

template <class T, class Epilogue>
__global__ __launch_bounds__(T::THREADS) void k_gemm(Operand A, Operand B, Shape s, Epilogue epi) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63;
    const int wave = wave_index();
    Place at;
    tile_of(s, tile_order(blockIdx.x, gridDim.x), at.tile_m, at.tile_n);
    at.split = blockIdx.y;
    at.batch = blockIdx.z;
    const int m0 = at.tile_m * T::BM, n0 = at.tile_n * T::BN;
    const int wm = wave / T::WN, wn = wave % T::WN;
    at.row0 = m0 + wm * 32 * T::TM;
    at.col0 = n0 + wn * 32 * T::TN;
    const int k0 = blockIdx.y * s.k_split;
    const int k1 = k0 + s.k_split < s.K ? k0 + s.k_split : s.K;

    // This wavefront's direct loads of a slice: load d of an operand brings RPI
    // rows of one of its planes.  Lane l's 16 bytes land at chunk l of the
    // load's 1024 bytes; it reads the chunk that the swizzle puts there.
    constexpr int DA = T::DMA_A, DB = T::DMA_B;
    uint32_t off_a[DA], off_b[DB];
    auto offset = [&](const Operand &o, int first, int r, int row) {
        const int chunk = (lane % T::CPR) ^ T::key(r);
        const int last = o.rows - 1 - first;
        return (uint32_t)(row < last ? row : last) * (uint32_t)(o.ld * 2) + chunk * 16;
    };
#pragma unroll
    for (int d = 0; d < DA; ++d) {
        const int row = (wave + T::NW * d) * T::RPI + lane / T::CPR;
        off_a[d] = offset(A, m0, row, row);
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int row = (wave + T::NW * d) * T::RPI + lane / T::CPR;
        off_b[d] = offset(B, n0, T::BM + row, row);
    }
    rsrc_t from_a[T::P], from_b[T::P];
#pragma unroll
    for (int p = 0; p < T::P; ++p) {
        from_a[p] = buffer(A.p + at.batch * A.batch + p * A.plane + (int64_t)m0 * A.ld);
        from_b[p] = buffer(B.p + at.batch * B.batch + p * B.plane + (int64_t)n0 * B.ld);
    }
    auto issue = [&](int buf, int step) {
        const uint32_t k = (uint32_t)(k0 + step * T::BK) * 2;
#pragma unroll
        for (int p = 0; p < T::P; ++p) {
            char *to = lds + buf * T::SLICE + p * (T::BM + T::BN) * T::CPR * 16 + wave * 1024;
#pragma unroll
            for (int d = 0; d < DA; ++d) dma16(from_a[p], off_a[d], k, to + T::NW * d * 1024);
#pragma unroll
            for (int d = 0; d < DB; ++d) dma16(from_b[p], off_b[d], k, to + T::BM * T::CPR * 16 + T::NW * d * 1024);
        }
    };

    // what the epilogue wants in LDS, loaded while the products go on
    constexpr int ROOM = room<T, Epilogue>();
    epi.template begin<T>(at, lds + ROOM);

    f32x16_t acc[T::TM][T::TN];
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    epi.template init<T>(acc, at);

    // Of three planes the products other than the largest have sums of their own,
    // added at the end: each addition of a small one to the large sum would round
    // that once more (an update of 1255 x 1504 in fp32 was off by 3.6e-6 so, and is by
    // 1.8e-6; plain fp32 products make 2.5e-6; 820 us either way).
    constexpr bool APART = T::P == 3;
    f32x16_t low[APART ? T::TM : 1][APART ? T::TN : 1];
    if constexpr (APART)
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) low[i][j][e] = 0.f;

    const int steps = (k1 - k0) / T::BK;
    const int ar = wm * 32 * T::TM + (lane & 31), br = T::BM + wn * 32 * T::TN + (lane & 31);
    constexpr int KK = T::BK / 16;
    // Operand fragments are read one 16-value step ahead of the products that
    // use them, in two register sets, also across the slices: the barrier
    // after which the next slice may be read and this one's buffer filled again
    // comes before the products of a slice's last step.
    bf16x8_t a[2][T::P][T::TM], b[2][T::P][T::TN];
    auto read = [&](const char *slice, int kk, int set) {
        const int chunk = 2 * kk + (lane >> 5);
#pragma unroll
        for (int p = 0; p < T::P; ++p) {
            const char *plane = slice + p * (T::BM + T::BN) * T::CPR * 16;
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
                a[set][p][i] = *reinterpret_cast<const bf16x8_t *>(
                    plane + ((ar + 32 * i) * T::CPR + (chunk ^ T::key(ar + 32 * i))) * 16);
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
                b[set][p][j] = *reinterpret_cast<const bf16x8_t *>(
                    plane + ((br + 32 * j) * T::CPR + (chunk ^ T::key(br + 32 * j))) * 16);
        }
    };
    auto multiply = [&](int set) {  // the smaller products first
#pragma unroll
        for (int t = T::P - 1; t >= 0; --t)
#pragma unroll
            for (int p = 0; p <= t; ++p)
#pragma unroll
                for (int i = 0; i < T::TM; ++i)
#pragma unroll
                    for (int j = 0; j < T::TN; ++j) {
                        f32x16_t &to = APART && t > 0 ? low[i][j] : acc[i][j];
                        to = mfma(a[set][p][i], b[set][t - p][j], to);
                    }
    };
#pragma unroll
    for (int t = 0; t < T::STAGES; ++t)
        if (t < steps) issue(t, t);
    if (steps >= T::STAGES)
        wait_and_barrier<(T::STAGES - 1) * T::DMA>();
    else
        wait_and_barrier<0>();
    read(lds, 0, 0);
    int buf = 0;
    // One slice; its last step's products come after the switch to the next
    // one.  MORE: a slice is left to be loaded into this one's buffer; NEXT:
    // there is a next one.
    auto slice = [&](int step, auto more, auto next) {
        constexpr bool MORE = decltype(more)::value, NEXT = decltype(next)::value;
        const char *at_ = lds + buf * T::SLICE;
        const int after = buf + 1 == T::STAGES ? 0 : buf + 1;
#pragma unroll
        for (int kk = 0; kk < KK - 1; ++kk) {
            read(at_, kk + 1, (kk + 1) & 1);
            multiply(kk & 1);
            interleave<T::PRODUCTS, T::READS, 0>();
            sched_barrier();
        }
        if constexpr (NEXT) {
            // the next slice is there (the ones after it may be on their way),
            // and no wavefront reads this one any more
            wait_and_barrier<MORE ? (T::STAGES - 2) * T::DMA : 0>();
            read(lds + after * T::SLICE, 0, 0);
            if constexpr (MORE) issue(buf, step + T::STAGES);
        }
        multiply((KK - 1) & 1);
        interleave<T::PRODUCTS, NEXT ? T::READS : 0, MORE ? T::DMA : 0>();
        sched_barrier();
        buf = after;
    };
    int step = 0;
    for (; step + T::STAGES < steps; ++step) slice(step, std::true_type{}, std::true_type{});
    for (; step + 1 < steps; ++step) slice(step, std::false_type{}, std::true_type{});
    slice(step, std::false_type{}, std::false_type{});
    if constexpr (APART)
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j) acc[i][j] += low[i][j];
    // the epilogue may use the slices' LDS
    wait_and_barrier<0>();
    epi.template run<T>(acc, at, lds, lds + ROOM);
}

// Allow a kernel more than 64 KB of LDS, once on each device.
inline hipError_t allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

inline int64_t tiles_of(int64_t m, int64_t n, int bm, int bn, bool lower) {
    const int64_t tm = (m + bm - 1) / bm, tn = (n + bn - 1) / bn;
    return lower ? tm * (tm + 1) / 2 : tm * tn;
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
    const int64_t tiles = tiles_of(A.rows, B.rows, T::BM, T::BN, lower);
    const int64_t parts = (K + s.k_split - 1) / s.k_split;
    constexpr int LDS = room<T, Epilogue>() + Epilogue::template extra<T>();
    static_assert(LDS <= 160 * 1024, "LDS");
    if (LDS > 64 * 1024) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_lds(reinterpret_cast<const void *>(&k_gemm<T, Epilogue>), LDS, done);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_gemm<T, Epilogue>), dim3((unsigned)tiles, (unsigned)parts, (unsigned)batch), dim3(T::THREADS),
                       LDS, stream, A, B, s, epi);
    return hipGetLastError();
}

// The length of a part when a contraction of K is cut into at most `splits`.
inline int64_t part_length(int64_t K, int64_t splits) { return padded((K + splits - 1) / splits); }

// A product whose contraction is cut into parts: the parts' accumulators, 16
// bytes a lane, and the launch that adds them and goes on with the epilogue.
struct Store : Simple {
    float *out;  // [batch][parts][tiles][accumulators / 4][threads][4]
    Shape s;
    int parts;

    Store(float *out, const Shape &s, int parts) : out(out), s(s), parts(parts) {}

    template <class T>
    __device__ __forceinline__ int64_t place(const Place &at, int part) const {
        const int64_t tiles = s.lower ? (int64_t)s.tiles_m * (s.tiles_m + 1) / 2 : (int64_t)s.tiles_m * s.tiles_n;
        const int64_t tile = s.lower ? (int64_t)at.tile_m * (at.tile_m + 1) / 2 + at.tile_n
                                     : (int64_t)at.tile_m * s.tiles_n + at.tile_n;
        return (((int64_t)at.batch * parts + part) * tiles + tile) * (T::BM * T::BN) + threadIdx.x * 4;
    }
    template <class T>
    __device__ __forceinline__ void run(f32x16_t (&acc)[T::TM][T::TN], const Place &at, char *, char *) const {
        float *o = out + place<T>(at, at.split);
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4 *>(o + ((i * T::TN + j) * 4 + q) * T::THREADS * 4) =
                        make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    }
};

// Accumulators that an epilogue stored with Store (in one part), and another
// epilogue for them.
template <class T, class Epilogue>
__global__ __launch_bounds__(T::THREADS) void k_gemm_again(Store stored, Epilogue epi) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Place at;
    tile_of(stored.s, tile_order(blockIdx.x, gridDim.x), at.tile_m, at.tile_n);
    at.split = at.batch = 0;
    const int wave = wave_index();
    at.row0 = at.tile_m * T::BM + wave / T::WN * 32 * T::TM;
    at.col0 = at.tile_n * T::BN + wave % T::WN * 32 * T::TN;
    constexpr int ROOM = Epilogue::template lds<T>();
    epi.template begin<T>(at, lds + ROOM);
    f32x16_t acc[T::TM][T::TN];
    const float *from = stored.out + stored.template place<T>(at, 0);
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(from + ((i * T::TN + j) * 4 + q) * T::THREADS * 4);
                acc[i][j][4 * q] = v.x;
                acc[i][j][4 * q + 1] = v.y;
                acc[i][j][4 * q + 2] = v.z;
                acc[i][j][4 * q + 3] = v.w;
            }
    __syncthreads();
    epi.template run<T>(acc, at, lds, lds + ROOM);
}

template <class T, class Epilogue>
hipError_t launch_again(hipStream_t stream, const Store &stored, const Epilogue &epi) {
    constexpr int LDS = Epilogue::template lds<T>() + Epilogue::template extra<T>();
    static_assert(LDS <= 160 * 1024, "LDS");
    if (LDS > 64 * 1024) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_lds(reinterpret_cast<const void *>(&k_gemm_again<T, Epilogue>), LDS, done);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((k_gemm_again<T, Epilogue>), dim3((unsigned)(stored.s.tiles_m * stored.s.tiles_n)),
                       dim3(T::THREADS), LDS, stream, stored, epi);
    return hipGetLastError();
}

// A workgroup joins one row of 32 x 32 blocks of each wavefront (gridDim.y of
// them), so that a few large tiles still give many workgroups.
template <class T, class Epilogue>
__global__ __launch_bounds__(T::THREADS) void k_gemm_join(Store parts, Epilogue epi) {
    Place at;
    tile_of(parts.s, tile_order(blockIdx.x, gridDim.x), at.tile_m, at.tile_n);
    at.split = 0;
    at.batch = blockIdx.z;
    const int wave = wave_index(), i = blockIdx.y;
    at.row0 = at.tile_m * T::BM + wave / T::WN * 32 * T::TM + 32 * i;
    at.col0 = at.tile_n * T::BN + wave % T::WN * 32 * T::TN;
    f32x16_t acc[1][T::TN];
#pragma unroll
    for (int j = 0; j < T::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[0][j][e] = 0.f;
#pragma unroll 2
    for (int k = 0; k < parts.parts; ++k) {
        const float *from = parts.out + parts.template place<T>(at, k);
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(from + ((i * T::TN + j) * 4 + q) * T::THREADS * 4);
                acc[0][j][4 * q] += v.x;
                acc[0][j][4 * q + 1] += v.y;
                acc[0][j][4 * q + 2] += v.z;
                acc[0][j][4 * q + 3] += v.w;
            }
    }
    epi.template direct<1, T::TN>(acc, at);
}

// The product with its contraction in parts of k_part, by way of `parts`
// (parts x batch x tiles x BM x BN floats) if there is more than one.
template <class T, class Epilogue>
hipError_t launch_parts(hipStream_t stream, const Operand &A, const Operand &B, int64_t K, int64_t k_part,
                        int64_t batch, bool lower, const Epilogue &epi, float *parts) {
    const int n = (int)((K + k_part - 1) / k_part);
    if (n <= 1) return launch<T>(stream, A, B, K, K, batch, lower, epi);
    const Shape s = {(int)K, (int)k_part, (A.rows + T::BM - 1) / T::BM, (B.rows + T::BN - 1) / T::BN, lower};
    const Store store(parts, s, n);
    const hipError_t e = launch<T>(stream, A, B, K, k_part, batch, lower, store);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_gemm_join<T, Epilogue>), dim3((unsigned)tiles_of(A.rows, B.rows, T::BM, T::BN, lower), T::TM, (unsigned)batch),
                       dim3(T::THREADS), 0, stream, store, epi);
    return hipGetLastError();
}

}  // namespace
}  // namespace gemm
