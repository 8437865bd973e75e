// The norm over all values of many tensors, and the tensors scaled so that it is
// at most a given one:
//   norm = sqrt(sum over all values of x^2),  y = x min(1, most / (norm + eps)).
//
// Few values (up to kFew): one launch of one workgroup, which reads them twice.  Otherwise
// two passes, each over all tensors at once: the first leaves each workgroup's sum of
// squares, in fp64 (fp32 squares overflow from 1.8e19 and vanish below 1e-23), the second adds
// these in a fixed order, in each workgroup, and scales.  Bound by the bytes, one read and
// another read and a write of everything; the second pass goes backwards, so that what
// the first read last is still in the memory-side cache.
#include "dense.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTensors = 80;         // of a launch: their table goes with its arguments
constexpr int64_t kChunk = 16384;    // values that a workgroup takes at a time
constexpr int64_t kFew = 65536;
constexpr int kFewThreads = 1024;

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

// The tensor of a chunk.
__device__ __forceinline__ int tensor_of(const Table &table, int64_t chunk) {
    int lo = 0, hi = table.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((table.t[mid].first & kFirst) <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

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

template <bool BF16, int THREADS>
__device__ __forceinline__ double squares(const void *in, int64_t lo, int64_t hi) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    int64_t i = lo + threadIdx.x * 8;
    for (; i + 8 <= hi; i += THREADS * 8) {
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

template <int THREADS>
__device__ __forceinline__ double squares(const Tensor &t, int64_t lo, int64_t hi) {
    return t.first & kIn16 ? squares<true, THREADS>(t.in, lo, hi) : squares<false, THREADS>(t.in, lo, hi);
}

__global__ __launch_bounds__(kThreads) void k_squares(Table table, double *sums) {
    double s = 0.0;
    for (int64_t c = blockIdx.x; c < table.chunks; c += gridDim.x) {
        const Tensor &t = table.t[tensor_of(table, c)];
        const int64_t lo = (c - (t.first & kFirst)) * kChunk, hi = lo + kChunk < t.n ? lo + kChunk : t.n;
        s += squares<kThreads>(t, lo, hi);
    }
    s = block_sum<kThreads>(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <bool IN16, bool OUT16, int THREADS>
__device__ __forceinline__ void scale(const void *in, void *out, int64_t lo, int64_t hi, float f) {
    int64_t i = lo + threadIdx.x * 8;
    for (; i + 8 <= hi; i += THREADS * 8) {
        float v[8];
        load_row<IN16, 8>(reinterpret_cast<const char *>(in) + i * (IN16 ? 2 : 4), 0, 8, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= f;
        store_row<OUT16, 8>(reinterpret_cast<char *>(out) + i * (OUT16 ? 2 : 4), 0, 8, v);
    }
    for (int k = 0; i + k < hi && k < 8; ++k) {
        const float v = f * (IN16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(in)[i + k])
                                  : reinterpret_cast<const float *>(in)[i + k]);
        if (OUT16)
            reinterpret_cast<uint16_t *>(out)[i + k] = (uint16_t)pack_bf16(v, 0.f);
        else
            reinterpret_cast<float *>(out)[i + k] = v;
    }
}

template <int THREADS>
__device__ __forceinline__ void scale(const Tensor &t, int64_t lo, int64_t hi, float f) {
    const bool in16 = t.first & kIn16, out16 = t.first & kOut16;
    if (in16 && out16)
        scale<true, true, THREADS>(t.in, t.out, lo, hi, f);
    else if (in16)
        scale<true, false, THREADS>(t.in, t.out, lo, hi, f);
    else if (out16)
        scale<false, true, THREADS>(t.in, t.out, lo, hi, f);
    else
        scale<false, false, THREADS>(t.in, t.out, lo, hi, f);
}

// What a norm scales by: a norm that is no number makes every value none; zeros stay
// zeros without eps too.
__device__ __forceinline__ float factor(double norm, float most, float eps) {
    const double q = (double)most / (norm + (double)eps);
    return q > 1.0 || norm == 0.0 ? 1.f : (float)q;
}

__global__ __launch_bounds__(kThreads) void k_scale(Table table, const double *sums, int parts, float most, float eps,
                                                    float *norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += sums[i];
    const double all = sqrt(block_sum<kThreads>(s));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
    const float f = factor(all, most, eps);
    for (int64_t c = table.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const Tensor &t = table.t[tensor_of(table, c)];
        if (f == 1.f && t.in == t.out) continue;
        const int64_t lo = (c - (t.first & kFirst)) * kChunk, hi = lo + kChunk < t.n ? lo + kChunk : t.n;
        scale<kThreads>(t, lo, hi, f);
    }
}

__global__ __launch_bounds__(kFewThreads) void k_few(Table table, float most, float eps, float *norm) {
    double s = 0.0;
    for (int i = 0; i < table.count; ++i) s += squares<kFewThreads>(table.t[i], 0, table.t[i].n);
    const double all = sqrt(block_sum<kFewThreads>(s));
    if (threadIdx.x == 0) *norm = (float)all;
    const float f = factor(all, most, eps);
    for (int i = 0; i < table.count; ++i) {
        const Tensor &t = table.t[i];
        if (f != 1.f || t.in != t.out) scale<kFewThreads>(t, 0, t.n, f);
    }
}

// The tensors from `at` on that a launch takes; those without values are passed over.
int fill(const ClipArgs &a, int at, Table &table) {
    table.count = 0;
    table.chunks = 0;
    for (; at < a.count && table.count < kTensors; ++at) {
        if (a.n[at] <= 0) continue;
        table.t[table.count++] = {a.in[at], a.out[at], a.n[at],
                                  table.chunks | (a.in_type[at] == LATTICE_BF16 ? kIn16 : 0) |
                                      (a.out_type[at] == LATTICE_BF16 ? kOut16 : 0)};
        table.chunks += (a.n[at] + kChunk - 1) / kChunk;
    }
    return at;
}

unsigned grid_of(const lattice_dense *D, const Table &table) {
    const int64_t most = (int64_t)8 * D->cu_count;
    return (unsigned)(table.chunks < most ? table.chunks : most);
}

// Whether one workgroup takes them.
bool few(const ClipArgs &a) {
    int64_t all = 0;
    int count = 0;
    for (int i = 0; i < a.count; ++i) {
        all += a.n[i];
        count += a.n[i] > 0;
        if (all > kFew || count > kTensors) return false;
    }
    return true;
}

}  // namespace

int64_t clip_scratch(const lattice_dense *D, const ClipArgs &a) {
    Table table;
    if (few(a)) return 0;
    int64_t parts = 0;
    for (int at = 0; at < a.count;) {
        at = fill(a, at, table);
        parts += grid_of(D, table);
    }
    return parts * 8;
}

hipError_t launch_clip(lattice_dense *D, const ClipArgs &a) {
    Table table;
    if (few(a)) {
        fill(a, 0, table);
        hipLaunchKernelGGL(k_few, dim3(1), dim3(kFewThreads), 0, D->stream, table, a.most, a.eps, a.norm);
        return hipGetLastError();
    }
    double *sums = static_cast<double *>(D->ws);
    int parts = 0;
    for (int at = 0; at < a.count;) {
        at = fill(a, at, table);
        const unsigned grid = grid_of(D, table);
        if (!grid) continue;
        hipLaunchKernelGGL(k_squares, dim3(grid), dim3(kThreads), 0, D->stream, table, sums + parts);
        TRY(hipGetLastError());
        parts += (int)grid;
    }
    bool first = true;
    for (int at = 0; at < a.count || first;) {
        at = fill(a, at, table);
        const unsigned grid = grid_of(D, table);
        if (!grid && !(first && at >= a.count)) continue;
        // one workgroup without tensors still leaves the norm
        hipLaunchKernelGGL(k_scale, dim3(grid ? grid : 1), dim3(kThreads), 0, D->stream, table, sums, parts, a.most, a.eps,
                           first ? a.norm : nullptr);
        TRY(hipGetLastError());
        first = false;
    }
    return hipSuccess;
}
