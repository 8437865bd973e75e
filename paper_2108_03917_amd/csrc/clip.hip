// The norm over all values of many tensors, and the tensors scaled so that it is
// at most a given one:
//   norm = sqrt(sum over all values of x^2),  y = x min(1, most / (norm + eps)).
//
// Few values (up to kFew): one launch of one workgroup, which keeps them in registers
// (42000 values in six tensors: 9.6 us, two launches 7.5, but 2 us less of the host's time, which
// is what such a call takes: 11.4 us, 13.1).
// Otherwise two passes, each over all tensors at once: the first leaves each workgroup's sum of
// squares, in fp64 (fp32 squares overflow from 1.8e19 and vanish below 1e-23), the second adds
// these in a fixed order, in each workgroup, and scales.  Bound by the bytes, one read and
// another read and a write of everything; the second pass goes backwards, so that what
// the first read last is still in the memory-side cache.  400 million bf16 values in 48
// tensors: 154 us (5.2 TB/s) and 287 (5.6); 30 million fp32 in 60: 21 and 40.
//
// A launch takes 64 tensors.  More take two for each 64, and every workgroup that scales adds up the
// sums of all: 1e8 fp32 values take 236 us in 48 tensors (5.1 TB/s), 259 in 65, 350 in 300 and
// 712 in 1000 (1.7 TB/s), 1e9 in 1000 3300 (3.6 TB/s).
#include "dense.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTensors = 64;         // of a launch: their table goes with its arguments, a tensor a lane
constexpr int64_t kChunk = 16384;    // values that a workgroup takes at a time
constexpr int kFewThreads = 1024, kPieces = 8;     // of a wavefront
constexpr int64_t kPiece = 512, kFew = kFewThreads / 64 * kPieces * kPiece;

struct Tensor {
    const void *in;
    void *out;
    int64_t n;
    int64_t first;  // chunk; bit 62: `in` is bf16, bit 61: `out` is
};
constexpr int64_t kIn16 = (int64_t)1 << 62, kOut16 = (int64_t)1 << 61, kFirst = kOut16 - 1;

struct Table {
    Tensor t[kTensors];
    int count;
    int64_t chunks;
};

// The table in a wavefront's lanes, and a chunk's tensor out of it: a search in memory
// took as long as a chunk (six steps of a load each).
struct Lanes {
    Tensor mine;
    int64_t first;  // of a lane without a tensor: behind all chunks
    __device__ __forceinline__ explicit Lanes(const Table &table) {
        const int lane = threadIdx.x & 63;
        mine = table.t[lane < table.count ? lane : 0];
        first = lane < table.count ? mine.first & kFirst : kFirst;
    }
    __device__ __forceinline__ static uint64_t from_lane(uint64_t x, int lane) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), lane) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, lane);
    }
    __device__ __forceinline__ Tensor of(int64_t chunk) const {
        const int i = __popcll(__ballot(first <= chunk)) - 1;
        Tensor t;
        t.in = reinterpret_cast<const void *>(from_lane(reinterpret_cast<uint64_t>(mine.in), i));
        t.out = reinterpret_cast<void *>(from_lane(reinterpret_cast<uint64_t>(mine.out), i));
        t.n = (int64_t)from_lane((uint64_t)mine.n, i);
        t.first = (int64_t)from_lane((uint64_t)mine.first, i);
        return t;
    }
};

// Sum of a double over the workgroup, the same in each thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double red[THREADS / 64];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) x += red[w];
    return x;
}

template <bool BF16>
__device__ __forceinline__ double squares(const void *in, int64_t lo, int64_t hi) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int64_t i = lo + threadIdx.x * 8;
    for (; i + 8 <= hi; i += kThreads * 8) {
        float v[8];
        load_row<BF16, 8>(reinterpret_cast<const char *>(in) + i * (BF16 ? 2 : 4), 0, 8, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k & 3] = fma((double)v[k], (double)v[k], s[k & 3]);
    }
    for (int k = 0; i + k < hi && k < 8; ++k) {
        const double v = BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(in)[i + k])
                              : reinterpret_cast<const float *>(in)[i + k];
        s[0] = fma(v, v, s[0]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__device__ __forceinline__ double squares(const Tensor &t, int64_t lo, int64_t hi) {
    return t.first & kIn16 ? squares<true>(t.in, lo, hi) : squares<false>(t.in, lo, hi);
}

__global__ __launch_bounds__(kThreads) void k_squares(Table table, double *sums) {
    const Lanes lanes(table);
    double s = 0.0;
    for (int64_t c = blockIdx.x; c < table.chunks; c += gridDim.x) {
        const Tensor t = lanes.of(c);
        const int64_t lo = (c - (t.first & kFirst)) * kChunk, hi = lo + kChunk < t.n ? lo + kChunk : t.n;
        s += squares(t, lo, hi);
    }
    s = block_sum<kThreads>(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// What a norm scales by, f 2^e: a norm that is no number makes every value none, unless there is
// no largest norm; zeros stay zeros without eps too.  The power of two is there for factors that
// are no normal fp32 numbers, of norms up to 1e47.
struct Factor {
    float f;
    int e;
    __device__ __forceinline__ Factor(double norm, float most, float eps) : f(1.f), e(0) {
        const double q = (double)most / (norm + (double)eps);
        if (q > 1.0 || norm == 0.0 || most == INFINITY) return;
        if (q > 0.0 && q < 0x1p-100) e = ilogb(q) + 1;  // f <= 1: no product overflows
        f = (float)ldexp(q, -e);
    }
    __device__ __forceinline__ bool one() const { return f == 1.f && e == 0; }
    __device__ __forceinline__ float times(float v) const { return ldexpf(v * f, e); }
};

template <bool IN16, bool OUT16>
__device__ __forceinline__ void scale(const void *in, void *out, int64_t lo, int64_t hi, const Factor &f) {
    int64_t i = lo + threadIdx.x * 8;
    for (; i + 8 <= hi; i += kThreads * 8) {
        float v[8];
        load_row<IN16, 8>(reinterpret_cast<const char *>(in) + i * (IN16 ? 2 : 4), 0, 8, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = f.times(v[k]);
        store_row<OUT16, 8>(reinterpret_cast<char *>(out) + i * (OUT16 ? 2 : 4), 0, 8, v);
    }
    for (int k = 0; i + k < hi && k < 8; ++k) {
        const float v = f.times(IN16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(in)[i + k])
                                     : reinterpret_cast<const float *>(in)[i + k]);
        if (OUT16)
            reinterpret_cast<uint16_t *>(out)[i + k] = (uint16_t)pack_bf16(v, 0.f);
        else
            reinterpret_cast<float *>(out)[i + k] = v;
    }
}

__device__ __forceinline__ void scale(const Tensor &t, int64_t lo, int64_t hi, const Factor &f) {
    const bool in16 = t.first & kIn16, out16 = t.first & kOut16;
    if (in16 && out16)
        scale<true, true>(t.in, t.out, lo, hi, f);
    else if (in16)
        scale<true, false>(t.in, t.out, lo, hi, f);
    else if (out16)
        scale<false, true>(t.in, t.out, lo, hi, f);
    else
        scale<false, false>(t.in, t.out, lo, hi, f);
}

__global__ __launch_bounds__(kThreads) void k_scale(Table table, const double *sums, int parts, float most, float eps,
                                                    float *norm) {
    const Lanes lanes(table);
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += sums[i];
    const double all = sqrt(block_sum<kThreads>(s));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
    const Factor f(all, most, eps);
    for (int64_t c = table.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const Tensor t = lanes.of(c);
        if (f.one() && t.in == t.out) continue;
        const int64_t lo = (c - (t.first & kFirst)) * kChunk, hi = lo + kChunk < t.n ? lo + kChunk : t.n;
        scale(t, lo, hi, f);
    }
}

// Up to 16 x kPieces pieces of 512 values, of which a wavefront keeps every 16th.
__global__ __launch_bounds__(kFewThreads) void k_few(Table table, float most, float eps, float *norm) {
    constexpr int WAVES = kFewThreads / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Lanes lanes(table);
    // as they are stored; nothing is made of them before all are under way
    uint32_t w[kPieces][8];
    bool half[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const int64_t c = wave + k * WAVES;
        half[k] = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[k][i] = 0;
        if (c >= table.chunks) continue;
        const Tensor t = lanes.of(c);
        const int64_t lo = (c - (t.first & kFirst)) * kPiece, at = lo + lane * 8;
        half[k] = t.first & kIn16;
        if (lo + kPiece <= t.n) {
            if (half[k]) {
                Raw<true, 8> u;
                load_raw<true, 8>(reinterpret_cast<const uint16_t *>(t.in) + at, 0, 8, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[k][i] = u.w[i];
            } else {
                Raw<false, 8> u;
                load_raw<false, 8>(reinterpret_cast<const float *>(t.in) + at, 0, 8, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[k][i] = u.w[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i < t.n) {
                    if (half[k])
                        w[k][i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(t.in)[at + i] << (16 * (i & 1));
                    else
                        w[k][i] = reinterpret_cast<const uint32_t *>(t.in)[at + i];
                }
        }
    }
    float v[kPieces][8];
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[k][i] = __uint_as_float(!half[k] ? w[k][i] : (i & 1) ? w[k][i / 2] & 0xffff0000u : w[k][i / 2] << 16);
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fma((double)v[k][i], (double)v[k][i], s);
    const double all = sqrt(block_sum<kFewThreads>(s));
    if (threadIdx.x == 0) *norm = (float)all;
    const Factor f(all, most, eps);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const int64_t c = wave + k * WAVES;
        if (c >= table.chunks) continue;
        const Tensor t = lanes.of(c);
        const int64_t at = (c - (t.first & kFirst)) * kPiece + lane * 8;
        const int left = t.n - at < 8 ? (int)(t.n - at) : 8;
        if (left <= 0 || (f.one() && t.in == t.out)) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = f.times(v[k][i]);
        if (t.first & kOut16)
            store_row<true, 8>(reinterpret_cast<uint16_t *>(t.out) + at, 0, left, v[k]);
        else
            store_row<false, 8>(reinterpret_cast<float *>(t.out) + at, 0, left, v[k]);
    }
}

// The tensors from `at` on that a launch takes; those without values are passed over.
int fill(const ClipArgs &a, int at, int64_t chunk, Table &table) {
    table.count = 0;
    table.chunks = 0;
    for (; at < a.count && table.count < kTensors; ++at) {
        if (a.n[at] <= 0) continue;
        table.t[table.count++] = {a.in[at], a.out[at], a.n[at],
                                  table.chunks | (a.in_type[at] == LATTICE_BF16 ? kIn16 : 0) |
                                      (a.out_type[at] == LATTICE_BF16 ? kOut16 : 0)};
        table.chunks += (a.n[at] + chunk - 1) / chunk;
    }
    return at;
}

unsigned grid_of(const lattice_dense *D, const Table &table) {
    const int64_t most = (int64_t)8 * D->cu_count;
    return (unsigned)(table.chunks < most ? table.chunks : most);
}

// Whether one workgroup takes them.
bool few(const ClipArgs &a) {
    int64_t pieces = 0;
    int count = 0;
    for (int i = 0; i < a.count; ++i) {
        pieces += (a.n[i] + kPiece - 1) / kPiece;
        count += a.n[i] > 0;
        if (pieces * kPiece > kFew || count > kTensors) return false;
    }
    return true;
}

}  // namespace

int64_t clip_scratch(const lattice_dense *D, const ClipArgs &a) {
    Table table;
    if (few(a)) return 0;
    int64_t parts = 0;
    for (int at = 0; at < a.count;) {
        at = fill(a, at, kChunk, table);
        parts += grid_of(D, table);
    }
    return parts * 8;
}

hipError_t launch_clip(lattice_dense *D, const ClipArgs &a) {
    Table table;
    if (few(a)) {
        fill(a, 0, kPiece, table);
        hipLaunchKernelGGL(k_few, dim3(1), dim3(kFewThreads), 0, D->stream, table, a.most, a.eps, a.norm);
        return hipGetLastError();
    }
    double *sums = static_cast<double *>(D->ws);
    int parts = 0;
    for (int at = 0; at < a.count;) {
        at = fill(a, at, kChunk, table);
        const unsigned grid = grid_of(D, table);
        if (!grid) continue;
        hipLaunchKernelGGL(k_squares, dim3(grid), dim3(kThreads), 0, D->stream, table, sums + parts);
        TRY(hipGetLastError());
        parts += (int)grid;
    }
    bool first = true;
    for (int at = 0; at < a.count;) {
        at = fill(a, at, kChunk, table);
        const unsigned grid = grid_of(D, table);
        if (!grid) continue;
        hipLaunchKernelGGL(k_scale, dim3(grid), dim3(kThreads), 0, D->stream, table, sums, parts, a.most, a.eps,
                           first ? a.norm : nullptr);
        TRY(hipGetLastError());
        first = false;
    }
    return hipSuccess;
}
