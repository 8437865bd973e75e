// The orthogonalised update (formulas: update.hip) of matrices with at most 128
// rows or columns: one launch a step.
//
// X (m <= n) is cut into slabs of 64 columns, one workgroup each.  A step's
// launch first adds up the slabs' parts of S = X X^T (m x m), forms Q = a I + b S
// + c S S in LDS, the same in every workgroup of a matrix, then its slab's
// X <- Q X, and the slab's part of the next S.  So nothing but X, in fp32,
// and the parts of S go through memory between launches, and a step of a 64 x
// 576 matrix takes one launch instead of three products that would each keep a
// few CUs busy.  Where the parts are many or large they are added by a launch of
// their own (k_small_sum), since every workgroup would read all of them.
//
// Products as in gemm.h: operands in LDS as bf16 planes, two for a bf16 result
// and three for an fp32 one, v_mfma_f32_32x32x16_bf16, fp32 sums.
//
// Bound by the chain of a step's three products in one workgroup: 64 x 576 in
// fp32 takes 9 us a step (9 workgroups), twelve of 128 x 1152 take 19 (216 of
// them) and 4.7 for the sums of the parts.
#include "planes.h"
#include "update.h"

namespace {

using gemm::bf16x8_t;
using gemm::f32x16_t;

constexpr int kSlab = 64;  // columns of X that a workgroup takes

// m is padded to MT = 64 or 128 rows, and a wavefront takes rows 32 (w / 2) on.
template <int MT_, int P_>
struct Small {
    static constexpr int MT = MT_, P = P_;
    static constexpr int THREADS = MT * 4;
    static constexpr int TS = MT / 64;  // blocks of 32 columns of an m x m product that a wavefront takes
    static constexpr int S_BYTES = P * MT * MT * 2, X_BYTES = P * kSlab * MT * 2;
    static constexpr int LDS = S_BYTES + X_BYTES;
    static_assert(LDS + 2048 <= 160 * 1024, "LDS");
};

// Address of 16-byte chunk c of row r of plane p of a matrix [rows][W] in LDS:
// swizzled so that 16 rows read at one chunk hit 16 different bank groups.
template <int W>
__device__ __forceinline__ int at_chunk(int rows, int p, int r, int c) {
    constexpr int CH = W / 8;
    const int key = CH == 16 ? r & 15 : (r >> 1) & 7;
    return ((p * rows + r) * CH + (c ^ key)) * 16;
}

// acc[j] += A[row0 ..][k] B[col0 + 32 j ..][k] over k < W, both [rows][W] planes in LDS.
template <int P, int W, int TN>
__device__ __forceinline__ void product(const char *A, int rows_a, int row0, const char *B, int rows_b, int col0,
                                        f32x16_t (&acc)[TN]) {
    const int lane = threadIdx.x & 63;
    // the next step's operands are read before this one's products
    bf16x8_t a[2][P], b[2][P][TN];
    auto read = [&](int kk) {
        const int c = 2 * kk + (lane >> 5), r = lane & 31;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            a[kk & 1][p] = *reinterpret_cast<const bf16x8_t *>(A + at_chunk<W>(rows_a, p, row0 + r, c));
#pragma unroll
            for (int j = 0; j < TN; ++j)
                b[kk & 1][p][j] = *reinterpret_cast<const bf16x8_t *>(B + at_chunk<W>(rows_b, p, col0 + 32 * j + r, c));
        }
    };
    read(0);
#pragma unroll
    for (int kk = 0; kk < W / 16; ++kk) {
        if (kk + 1 < W / 16) read(kk + 1);
#pragma unroll
        for (int t = P - 1; t >= 0; --t)  // the smaller products first
#pragma unroll
            for (int p = 0; p <= t; ++p)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[j] = gemm::mfma(a[kk & 1][p], b[kk & 1][t - p][j], acc[j]);
        gemm::sched_barrier();
    }
}

template <int TN>
__device__ __forceinline__ void clear(f32x16_t (&acc)[TN]) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
}

// Four consecutive values of a row (half a chunk) to their place in the planes.
template <int P, int W>
__device__ __forceinline__ void put4(char *to, int rows, int r, int c, const float *v) {
    uint32_t lo[P], hi[P];
    planes::split_pair<P>(v[0], v[1], lo);
    planes::split_pair<P>(v[2], v[3], hi);
#pragma unroll
    for (int p = 0; p < P; ++p)
        *reinterpret_cast<uint2 *>(to + at_chunk<W>(rows, p, r, c / 8) + 2 * (c & 4)) = make_uint2(lo[p], hi[p]);
}

// The values that put4 put there.
template <int P, int W>
__device__ __forceinline__ void get4(const char *from, int rows, int r, int c, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = 0.f;
#pragma unroll
    for (int p = P - 1; p >= 0; --p) {
        const uint2 u = *reinterpret_cast<const uint2 *>(from + at_chunk<W>(rows, p, r, c / 8) + 2 * (c & 4));
        v[0] += __uint_as_float(u.x << 16);
        v[1] += __uint_as_float(u.x & 0xffff0000u);
        v[2] += __uint_as_float(u.y << 16);
        v[3] += __uint_as_float(u.y & 0xffff0000u);
    }
    if (P == 3)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= 1.f / kSplitScale;
}

// The slab's part of S from its X in LDS, [MT][kSlab].
template <class Z>
__device__ __forceinline__ void write_part(const char *X, float *part) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row0 = 32 * (wave / 2), col0 = 32 * Z::TS * (wave % 2);
    f32x16_t acc[Z::TS];
    clear(acc);
    product<Z::P, kSlab, Z::TS>(X, Z::MT, row0, X, Z::MT, col0, acc);
#pragma unroll
    for (int j = 0; j < Z::TS; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            part[(row0 + gemm::acc_row(e)) * Z::MT + col0 + 32 * j + (lane & 31)] = acc[j][e] * planes::kBack<Z::P>;
}

struct SmallArgs {
    UpdateArgs a;
    int m, n, slabs;  // of X: m <= n
    bool tall;
    const double *squares;  // [batch][parts], or null: add them up here
    int parts;
    float *x;               // X^T [batch][n][MT]
    const float *gram;      // parts of S [batch][slabs][MT][MT]
    float *next;            // the next S's
    const float *s;         // S [batch][MT][MT] already added up, or null
    int64_t first;          // matrix of the whole call that the first here is
};

// X_0 = g / (|g| + eps), and the first parts of S.
template <class Z, bool GB>
__global__ __launch_bounds__(Z::THREADS) void k_small_first(SmallArgs f) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ double red[Z::THREADS / 64];
    const int b = blockIdx.y, c0 = blockIdx.x * kSlab;
    const char *g = reinterpret_cast<const char *>(f.a.g) + (f.first + b) * f.a.batch_stride * (GB ? 2 : 4);
    const int64_t row_bytes = f.a.row_stride * (GB ? 2 : 4);
    double scale;
    if (f.squares) {
        scale = inverse_norm<Z::THREADS>(f.squares + (int64_t)b * f.parts, f.parts, f.a.eps, red);
    } else {
        double s = 0.0;
        const int chunks = (f.a.n + 7) / 8;
        for (int t = threadIdx.x; t < f.a.m * chunks; t += Z::THREADS) {
            float v[8];
            load_row<GB, 8>(g + t / chunks * row_bytes, t % chunks * 8, f.a.n, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += (double)v[i] * (double)v[i];
        }
        scale = inverse_norm<Z::THREADS>(s, f.a.eps, red);
    }
    float *x = f.x + ((int64_t)b * f.n + c0) * Z::MT;
    // chunks of 8 values along g's rows: rows of X, or its columns if tall
    const int rows = f.tall ? kSlab : Z::MT, chunks = (f.tall ? Z::MT : kSlab) / 8;
    for (int t = threadIdx.x; t < rows * chunks; t += Z::THREADS) {
        const int r = t / chunks, c = t % chunks * 8;  // in the slab
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const int gr = f.tall ? c0 + r : r, gc = f.tall ? c : c0 + c;
        if (gr < f.a.m) load_row<GB, 8>(g + gr * row_bytes, gc, f.a.n, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // what lies past the matrix stays 0, whatever the scale
            v[i] = gr < f.a.m && gc + i < f.a.n ? (float)((double)v[i] * scale) : 0.f;
            const int row = f.tall ? c + i : r, col = f.tall ? r : c + i;
            if (c0 + col < f.n) x[(int64_t)col * Z::MT + row] = v[i];
            if (f.tall) {
                uint16_t h[Z::P];
                planes::split<Z::P>(v[i], h);
#pragma unroll
                for (int p = 0; p < Z::P; ++p)
                    *reinterpret_cast<uint16_t *>(lds + at_chunk<kSlab>(Z::MT, p, row, col / 8) + 2 * (col & 7)) = h[p];
            }
        }
        if (!f.tall) {
            put4<Z::P, kSlab>(lds, Z::MT, r, c, v);
            put4<Z::P, kSlab>(lds, Z::MT, r, c + 4, v + 4);
        }
    }
    __syncthreads();
    write_part<Z>(lds, f.next + ((int64_t)b * f.slabs + blockIdx.x) * Z::MT * Z::MT);
}

// S from its parts.
__global__ __launch_bounds__(256) void k_small_sum(const float *gram, int slabs, int size, float *s) {
    const int64_t b = blockIdx.y;
    const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const float *p = gram + b * slabs * size + i;
#pragma unroll 8
    for (int k = 0; k < slabs; ++k) {
        const float4 u = *reinterpret_cast<const float4 *>(p + (int64_t)k * size);
        v.x += u.x;
        v.y += u.y;
        v.z += u.z;
        v.w += u.w;
    }
    *reinterpret_cast<float4 *>(s + b * size + i) = v;
}

// One step; the last one writes the result.
template <class Z, bool LAST>
__global__ __launch_bounds__(Z::THREADS) void k_small_step(SmallArgs f) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    char *S = lds, *X = lds + Z::S_BYTES;
    const int b = blockIdx.y, c0 = blockIdx.x * kSlab;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int SIZE = Z::MT * Z::MT;
    float *x = f.x + ((int64_t)b * f.n + c0) * Z::MT;
    // the slab's X^T, columns past n as zeros
    constexpr int XV = kSlab * Z::MT / 4 / Z::THREADS;
    float4 xv[XV];
#pragma unroll
    for (int i = 0; i < XV; ++i) {
        const int t = threadIdx.x + Z::THREADS * i, col = t / (Z::MT / 4);
        xv[i] = c0 + col < f.n ? reinterpret_cast<const float4 *>(x)[t] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // S, as planes
    constexpr int SV = SIZE / 4 / Z::THREADS;
    const float4 *from = reinterpret_cast<const float4 *>(f.s ? f.s + (int64_t)b * SIZE : f.gram + (int64_t)b * f.slabs * SIZE);
    const int parts = f.s ? 1 : f.slabs;
    float4 sv[SV];
#pragma unroll
    for (int i = 0; i < SV; ++i) sv[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int k = 0; k < parts; ++k)
#pragma unroll
        for (int i = 0; i < SV; ++i) {
            const float4 u = from[k * (SIZE / 4) + threadIdx.x + Z::THREADS * i];
            sv[i].x += u.x;
            sv[i].y += u.y;
            sv[i].z += u.z;
            sv[i].w += u.w;
        }
#pragma unroll
    for (int i = 0; i < SV; ++i) {
        const int t = threadIdx.x + Z::THREADS * i;
        const float v[4] = {sv[i].x, sv[i].y, sv[i].z, sv[i].w};
        put4<Z::P, Z::MT>(S, Z::MT, t / (Z::MT / 4), t % (Z::MT / 4) * 4, v);
    }
#pragma unroll
    for (int i = 0; i < XV; ++i) {
        const int t = threadIdx.x + Z::THREADS * i;
        const float v[4] = {xv[i].x, xv[i].y, xv[i].z, xv[i].w};
        put4<Z::P, Z::MT>(X, kSlab, t / (Z::MT / 4), t % (Z::MT / 4) * 4, v);
    }
    __syncthreads();
    {
        // Q = a I + b S + c S S over S's place, once all have read S
        const int row0 = 32 * (wave / 2), col0 = 32 * Z::TS * (wave % 2);
        f32x16_t acc[Z::TS];
        clear(acc);
        product<Z::P, Z::MT, Z::TS>(S, Z::MT, row0, S, Z::MT, col0, acc);
        float q[Z::TS][4][4];
#pragma unroll
        for (int j = 0; j < Z::TS; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // S is symmetric: its row `col`, four columns from `row` on
                const int row = row0 + 8 * g + 4 * (lane >> 5), col = col0 + 32 * j + (lane & 31);
                float v[4];
                get4<Z::P, Z::MT>(S, Z::MT, col, row, v);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    q[j][g][r] = f.a.coef[1] * v[r] + f.a.coef[2] * (acc[j][4 * g + r] * planes::kBack<Z::P>) +
                                 (row + r == col ? f.a.coef[0] : 0.f);
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < Z::TS; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                put4<Z::P, Z::MT>(S, Z::MT, col0 + 32 * j + (lane & 31), row0 + 8 * g + 4 * (lane >> 5), q[j][g]);
    }
    __syncthreads();
    const int row0 = 32 * (wave / 2), col = 32 * (wave % 2) + (lane & 31);
    float xn[4][4];
    {
        f32x16_t acc[1];
        clear(acc);
        product<Z::P, Z::MT, 1>(S, Z::MT, row0, X, kSlab, 32 * (wave % 2), acc);
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) xn[g][r] = acc[0][4 * g + r] * planes::kBack<Z::P>;
    }
    if constexpr (LAST) {
        if (c0 + col >= f.n) return;
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = row0 + 8 * g + 4 * (lane >> 5) + r;
                if (row >= f.m) continue;
                const int64_t to = (f.first + b) * (int64_t)f.m * f.n +
                                   (f.tall ? (int64_t)(c0 + col) * f.m + row : (int64_t)row * f.n + c0 + col);
                if (f.a.out_bf16)
                    reinterpret_cast<uint16_t *>(f.a.out)[to] = (uint16_t)pack_bf16(xn[g][r], 0.f);
                else
                    reinterpret_cast<float *>(f.a.out)[to] = xn[g][r];
            }
    } else {
        __syncthreads();  // X^T has been read
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int row = row0 + 8 * g + 4 * (lane >> 5);
            if (c0 + col < f.n)
                *reinterpret_cast<float4 *>(x + (int64_t)col * Z::MT + row) =
                    make_float4(xn[g][0], xn[g][1], xn[g][2], xn[g][3]);
            // X in the order that sums over its columns: lane c of four takes
            // row c of their four columns
            uint32_t lo[Z::P], hi[Z::P];
            planes::split_pair<Z::P>(xn[g][0], xn[g][1], lo);
            planes::split_pair<Z::P>(xn[g][2], xn[g][3], hi);
#pragma unroll
            for (int p = 0; p < Z::P; ++p) {
                planes::transpose4(lo[p], hi[p]);
                const int c = col & ~3;
                *reinterpret_cast<uint2 *>(X + at_chunk<kSlab>(Z::MT, p, row + (lane & 3), c / 8) + 2 * (c & 4)) =
                    make_uint2(lo[p], hi[p]);
            }
        }
        __syncthreads();
        write_part<Z>(X, f.next + ((int64_t)b * f.slabs + blockIdx.x) * SIZE);
    }
}

// Parts of S of up to so many bytes are added by every workgroup itself.
constexpr int64_t kSumHere = 256 * 1024;
// So are the squares of a matrix of up to so many bytes: a launch of their own
// takes 6 us, reading 144 KB by every workgroup 2.
constexpr int64_t kNormHere = 256 * 1024;

struct Layout {
    int m, n, MT, slabs;
    bool tall, sum_here, norm_here;
    int64_t chunk;
    int64_t squares, x, gram[2], s, bytes;

    explicit Layout(const UpdateArgs &a) {
        tall = a.m > a.n;
        m = tall ? a.n : a.m;
        n = tall ? a.m : a.n;
        MT = m <= 64 ? 64 : 128;
        slabs = (n + kSlab - 1) / kSlab;
        const int64_t size = (int64_t)MT * MT * 4;
        sum_here = slabs * size <= kSumHere;
        norm_here = (int64_t)m * n * (a.g_bf16 ? 2 : 4) <= kNormHere;
        const int64_t each = (int64_t)n * MT * 4 + 2 * slabs * size + size;
        chunk = kUpdateChunk / each;
        chunk = chunk < 1 ? 1 : chunk < a.batch ? chunk : a.batch;
        ScratchLayout l;
        squares = l.take(a.batch * square_parts(a) * 8);
        x = l.take(chunk * n * MT * 4);
        for (int i = 0; i < 2; ++i) gram[i] = l.take(chunk * slabs * size);
        s = l.take(chunk * size);
        bytes = l.bytes;
    }
};

template <class Z>
hipError_t run(lattice_dense *D, const UpdateArgs &a, const Layout &l) {
    char *ws = reinterpret_cast<char *>(D->ws);
    hipStream_t st = D->stream;
    if (Z::LDS > 64 * 1024) {
        static std::atomic<uint64_t> done[2];
        TRY(gemm::allow_lds(reinterpret_cast<const void *>(&k_small_step<Z, true>), Z::LDS, done[0]));
        TRY(gemm::allow_lds(reinterpret_cast<const void *>(&k_small_step<Z, false>), Z::LDS, done[1]));
    }
    double *squares = l.norm_here ? nullptr : reinterpret_cast<double *>(ws + l.squares);
    if (squares) TRY(launch_squares(st, a, squares));
    const int parts = square_parts(a);
    for (int64_t b0 = 0; b0 < a.batch; b0 += l.chunk) {
        const int64_t batch = a.batch - b0 < l.chunk ? a.batch - b0 : l.chunk;
        const dim3 grid(l.slabs, (unsigned)batch);
        SmallArgs f = {a, l.m, l.n, l.slabs, l.tall, squares ? squares + b0 * parts : nullptr, parts, reinterpret_cast<float *>(ws + l.x),
                       nullptr, reinterpret_cast<float *>(ws + l.gram[0]), nullptr, b0};
        if (a.g_bf16)
            hipLaunchKernelGGL((k_small_first<Z, true>), grid, dim3(Z::THREADS), Z::X_BYTES, st, f);
        else
            hipLaunchKernelGGL((k_small_first<Z, false>), grid, dim3(Z::THREADS), Z::X_BYTES, st, f);
        TRY(hipGetLastError());
        for (int i = 0; i < a.steps; ++i) {
            // a step reads all parts while it writes its own: two sets
            f.gram = f.next;
            f.next = reinterpret_cast<float *>(ws + l.gram[(i + 1) & 1]);
            if (!l.sum_here) {
                float *s = reinterpret_cast<float *>(ws + l.s);
                hipLaunchKernelGGL(k_small_sum, dim3(Z::MT * Z::MT / 1024, (unsigned)batch), dim3(256), 0, st,
                                   f.gram, l.slabs, Z::MT * Z::MT, s);
                f.s = s;
            }
            if (i + 1 < a.steps)
                hipLaunchKernelGGL((k_small_step<Z, false>), grid, dim3(Z::THREADS), Z::LDS, st, f);
            else
                hipLaunchKernelGGL((k_small_step<Z, true>), grid, dim3(Z::THREADS), Z::LDS, st, f);
            TRY(hipGetLastError());
        }
    }
    return hipSuccess;
}

}  // namespace

bool update_small_covers(const UpdateArgs &a) { return a.steps > 0 && (a.m <= 128 || a.n <= 128); }

int64_t update_small_scratch(const UpdateArgs &a) { return Layout(a).bytes; }

hipError_t launch_update_small(lattice_dense *D, const UpdateArgs &a) {
    const Layout l(a);
    if (l.MT == 64) return a.out_bf16 ? run<Small<64, 2>>(D, a, l) : run<Small<64, 3>>(D, a, l);
    return a.out_bf16 ? run<Small<128, 2>>(D, a, l) : run<Small<128, 3>>(D, a, l);
}
