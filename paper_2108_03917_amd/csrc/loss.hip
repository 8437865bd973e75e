// The linear classifier with softmax cross entropy, and its gradients, with no
// more than a piece of the logits in memory at a time.
//
//   z_ik = x_i . w_k + b_k,   lse_i = log sum_k exp z_ik,   l_i = lse_i - z_it (t = target_i)
//   L = sum_i s l_i,  s = 1, or 1 / (rows with a label);  rows without a label count for nothing
//   G_ik = exp(z_ik - lse_i) - [k = t],   dx = s G w,   dw = s G^T x,   db_k = s sum_i G_ik.
//
// Rows are taken in pieces, and for the gradients classes too.  For a piece of
// rows a first product passes over all classes and keeps, per tile of classes,
// the running maximum and sum of each row; these are joined to lse.  Then, per
// piece of classes, the logits are computed again, G is formed from them in the
// product's epilogue, in both orders, and multiplied with w and x.  The
// second product of the logits costs a third more operations than the gradients
// need; where it would cost more than writing and reading the logits of a piece
// of rows (fp32 operands, whose products are six each, from 192 channels on),
// pieces are cut to a gigabyte of logits, or to 256 rows if these have more, and
// they are kept till G is formed (so a small problem's logits are all in memory;
// both passes over 1848 x 18928 logits of 245 channels: 265 us kept, 308 again;
// of 192 channels 229 and 248, of 128 200 and 207).
//
// The products run on the bf16 matrix cores (gemm.h): bf16 operands as they
// are, fp32 ones as three planes.  For bf16 gradients G is rounded to bf16 (a
// relative 2^-8 of each term at most, random in sign, as the gradients' own
// rounding is; s is left out of it, or the entries near -s of all rows would be off by
// the same part), or held in two planes if the caller asks for that: dx and dw are
// then two products each.  dx against 64 bits, and the time of a call, with one
// plane and with two, where the rounding of the stored dx alone makes 1.66e-3:
// 8192 x 1024 x 65536 1.66e-3 and 1.66e-3, 4.5 and 7.7 ms; 2048 x 512 x 5000
// 1.69e-3 and 1.65e-3, 122 and 188 us; 100000 x 64 x 200 1.90e-3 and 1.66e-3, 150
// and 212 us.  For fp32 gradients G is in three planes.  The bias gradient is
// summed from G before any rounding.  Sums are fp32, joined in a fixed order.
//
// With gradients the matrix cores bound it: 8192 rows, 65536 classes of 1024
// channels in bf16 take 4.4 ms (1.0 PFLOP/s of 8 N C K operations): the first
// pass 1.0, G 1.4, dx 1.1 and dw 0.95.  The loss alone of few rows is bound by
// the bytes of w: 64 x 1024 x 32768 in bf16 15 us in the product (4.4 TB/s).
#include "planes.h"
#include "rowsum.h"

namespace {

constexpr int kCounts = 256;          // partial counts of rows with a label
constexpr int64_t kMaxPiece = 65536;  // rows of a piece
constexpr int64_t kPieceBytes = (int64_t)512 << 20;  // of G in both orders
constexpr int64_t kKeep = (int64_t)1 << 30;          // of kept logits
// Pieces of rows whose bias gradients are held apart before they are added up
// (each time rounded to fp32 once): with room for all of them the scratch would
// grow with the rows.
constexpr int64_t kHeld = 64;

__device__ __forceinline__ int label_of(int64_t t, int K, int64_t ignore) {
    return t != ignore && t >= 0 && t < K ? (int)t : -1;
}

// What is laid out before the first piece: of w, and of the piece's rows.
struct Layout {
    planes::Source s;
    uint16_t *dst, *dst_t;
    int64_t ld, ld_t;
    int bx, blocks;  // blocks a row of them, and in all
};

// Everything before the first product, in one launch.  The first kCounts
// workgroups: rows with a label, counted per workgroup (a label that is neither
// a class nor `ignore` sets the status), the first piece's labels, and the
// classes' biases, zeros without any and -inf from K on, so that the classes that
// fill up the last tile have no share.  The others: the operands' planes.
template <bool BF16, int P>
__global__ __launch_bounds__(256) void k_begin(const int64_t *__restrict__ target, int64_t N, int n, int K,
                                               int64_t ignore, int32_t *count, int32_t *status, int32_t *label,
                                               const float *bias, int Kp, float *padded_bias, Layout w, Layout x) {
    __shared__ planes::Block<P> block;
    int at_ = (int)blockIdx.x - kCounts;
    if (at_ >= 0) {
        const Layout &l = at_ < w.blocks ? w : x;
        at_ -= at_ < w.blocks ? 0 : w.blocks;
        planes::lay_out<BF16, P>(l.s, at_ % l.bx, at_ / l.bx, 0, l.dst, l.ld, l.dst_t, l.ld_t, block);
        return;
    }
    int c = 0, bad = 0;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)kCounts * 256;
    for (int64_t i = at; i < N; i += step) {
        const int64_t t = target[i];
        const int l = label_of(t, K, ignore);
        c += l >= 0;
        bad |= l < 0 && t != ignore;
        if (i < n) label[i] = l;
    }
    for (int64_t k = at; k < Kp; k += step) padded_bias[k] = k < K ? (bias ? bias[k] : 0.f) : -INFINITY;
    if (bad) atomicOr(status, DENSE_ST_LABEL);
    int *red = reinterpret_cast<int *>(&block);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) c += __shfl_xor(c, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) count[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// The factor s of the rows with a label.  Called by whole wavefronts.
__device__ __forceinline__ float row_factor(const int32_t *count, bool mean) {
    if (!mean) return 1.f;
    int64_t n = 0;
    for (int i = threadIdx.x & 63; i < kCounts; i += 64) n += count[i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    return n > 0 ? (float)(1.0 / (double)n) : 0.f;
}

constexpr int kNoLabel = -(1 << 30);

// What the epilogues need of a piece's rows.
struct Rows {
    const int32_t *label;  // class, or -1 for a row without one
    const float *lse;
    int n;
};

// The labels of a later piece's rows.
__global__ __launch_bounds__(256) void k_labels(const int64_t *__restrict__ target, int n, int K, int64_t ignore,
                                                int32_t *label) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) label[i] = label_of(target[i], K, ignore);
}

// Epilogue of the first pass (rows of the product are classes, columns the
// piece's rows): maximum and sum of exponentials per tile and row, and the
// logit of the label.
template <int P>
struct Stats : gemm::Simple {
    const float *bias;  // padded
    const int32_t *label;
    int n;
    float2 *stats;      // [tiles of classes][n]
    float *picked;      // [n]
    gemm::Store kept;   // keeps the accumulators if it has somewhere to

    template <class T>
    static constexpr int lds() { return T::WM * T::BN * 8; }
    template <class T>
    static constexpr int extra() { return (T::BM + T::BN) * 4; }

    // the tile's biases and labels
    template <class T>
    __device__ __forceinline__ void begin(const gemm::Place &at, char *own) const {
        float *b = reinterpret_cast<float *>(own);
        for (int x = threadIdx.x; x < T::BM + T::BN; x += T::THREADS) {
            const int col = at.tile_n * T::BN + x - T::BM;
            if (x < T::BM)
                b[x] = bias[at.tile_m * T::BM + x];
            else
                reinterpret_cast<int32_t *>(b)[x] = col < n ? label[col] : -1;
        }
    }

    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *lds,
                                        const char *own) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int wm = wave / T::WN;
        if (kept.out) kept.template run<T>(acc, at, nullptr, nullptr);
        const float *own_bias = reinterpret_cast<const float *>(own) + at.row0 - at.tile_m * T::BM;
        const int32_t *own_label = reinterpret_cast<const int32_t *>(own) + T::BM + at.col0 - at.tile_n * T::BN;
        float2 *part = reinterpret_cast<float2 *>(lds);
        float4 bb[T::TM][4];
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                bb[i][q] = *reinterpret_cast<const float4 *>(own_bias + 32 * i + 8 * q + 4 * (lane >> 5));
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            const int col = at.col0 + 32 * j + (lane & 31);
            const int t = own_label[32 * j + (lane & 31)] - at.row0;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float4 b4 = bb[i][e >> 2];
                    const float b = (e & 3) == 0 ? b4.x : (e & 3) == 1 ? b4.y : (e & 3) == 2 ? b4.z : b4.w;
                    const float z = acc[i][j][e] * planes::kBack<P> + b;
                    acc[i][j][e] = z;
                    top = fmaxf(top, z);
                }
            if (__any(t >= 0 && t < 32 * T::TM)) {  // few wavefronts hold a row's label
#pragma unroll
                for (int i = 0; i < T::TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * i + gemm::acc_row(e) == t) picked[col] = acc[i][j][e];
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float ref = top == -INFINITY ? 0.f : top;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < T::TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) s += __expf(acc[i][j][e] - ref);
            s += __shfl_xor(s, 32);
            if (lane < 32) part[wm * T::BN + col - at.tile_n * T::BN] = make_float2(top, s);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < T::BN; c += T::THREADS) {
            const int col = at.tile_n * T::BN + c;
            if (col >= n) continue;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < T::WM; ++w) top = fmaxf(top, part[w * T::BN + c].x);
            const float ref = top == -INFINITY ? 0.f : top;
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < T::WM; ++w) s += part[w * T::BN + c].y * __expf(part[w * T::BN + c].x - ref);
            stats[(int64_t)at.tile_m * n + col] = make_float2(top, s);
        }
    }
};

// Joins the tiles' statistics to lse, and the rows' losses; one partial sum of
// the losses a workgroup, in fp64.  Q threads a row share its tiles: few where
// there are rows enough.  Also writes the factor s.
template <int Q>
__global__ __launch_bounds__(256) void k_lse(const float2 *__restrict__ stats, int tiles, int n,
                                             const float *__restrict__ picked, const int32_t *__restrict__ label,
                                             float *lse, float *rows, double *part, const int32_t *count, bool mean,
                                             float *factor) {
    if (blockIdx.x == 0 && threadIdx.x < 64) {
        const float s = row_factor(count, mean);
        if (threadIdx.x == 0) *factor = s;
    }
    const int i = blockIdx.x * (256 / Q) + threadIdx.x / Q, q = threadIdx.x % Q;
    double l = 0.0;
    if (i < n) {
        float top = -INFINITY, s = 0.f;
        for (int t = q; t < tiles; t += Q) {
            const float2 v = stats[(int64_t)t * n + i];
            const float m = fmaxf(top, v.x);
            const float ref = m == -INFINITY ? 0.f : m;
            s = s * __expf(top - ref) + v.y * __expf(v.x - ref);
            top = m;
        }
#pragma unroll
        for (int d = 1; d < Q; d *= 2) {
            const float top2 = __shfl_xor(top, d), s2 = __shfl_xor(s, d);
            const float m = fmaxf(top, top2);
            const float ref = m == -INFINITY ? 0.f : m;
            s = s * __expf(top - ref) + s2 * __expf(top2 - ref);
            top = m;
        }
        const float v = top + logf(s);
        if (q == 0) {
            const float one = label[i] >= 0 ? v - picked[i] : 0.f;
            lse[i] = v;
            if (rows) rows[i] = one;
            l = one;
        }
    }
    __shared__ double red[4];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = l;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// The loss from the workgroups' partial sums.
__global__ __launch_bounds__(256) void k_total(const double *__restrict__ part, int64_t n, const int32_t *count,
                                               bool mean, float *loss) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) s += part[i];
    int64_t c = 0;
    for (int i = threadIdx.x; i < kCounts; i += 256) c += count[i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        s += __shfl_xor(s, d);
        c += __shfl_xor(c, d);
    }
    __shared__ double red[4];
    __shared__ int64_t cred[4];
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6] = s;
        cred[threadIdx.x >> 6] = c;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = red[0] + red[1] + red[2] + red[3];
        c = cred[0] + cred[1] + cred[2] + cred[3];
        *loss = (float)(mean ? (c > 0 ? s / (double)c : 0.0) : s);
    }
}

// The value of lane (this one ^ D).
template <int D>
__device__ __forceinline__ float from_lane(float v) {
    if constexpr (D == 1)
        return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xF, 0xF, false));
    else if constexpr (D == 2)
        return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xF, 0xF, false));
    else
        return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), D << 10 | 0x1f));
}

// Sums of 16 values over 32 lanes each (the two halves of a wavefront apart):
// returns which of them this lane gets, in sum[0].
__device__ __forceinline__ int sum32(float (&sum)[16]) {
    const int lane = threadIdx.x & 63;
    int which = 0;
    auto round = [&](auto half, auto dist) {
        constexpr int h = decltype(half)::value, d = decltype(dist)::value;
        const bool up = lane & d;
        which += up ? h : 0;
#pragma unroll
        for (int e = 0; e < h; ++e) {
            const float keep = up ? sum[e + h] : sum[e], give = up ? sum[e] : sum[e + h];
            sum[e] = keep + from_lane<d>(give);
        }
    };
    using std::integral_constant;
    round(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    round(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    round(integral_constant<int, 2>{}, integral_constant<int, 4>{});
    round(integral_constant<int, 1>{}, integral_constant<int, 8>{});
    sum[0] += from_lane<16>(sum[0]);
    return which;
}

// Epilogue of the second pass over a piece of classes: G in both orders, in PG
// planes, and partial sums of its columns.
template <int P, int PG>
struct Grad : gemm::Simple {
    const float *bias;  // padded, of the piece's first class on
    Rows rows;
    int class0;         // of the piece
    int K, Kp, np;      // classes of the piece, classes and rows padded
    int64_t ldg, ldt;   // values between the rows of g and of gt
    uint16_t *g;        // [PG][n][ldg], classes up to Kp written, or null
    uint16_t *gt;       // [PG][K][ldt], rows up to np written, or null
    float *pbias;       // [tiles of rows * WN][K], or null
    const float *factor;

    template <class T>
    static constexpr int lds() { return T::BM * T::BN * 2; }
    template <class T>
    static constexpr int extra() { return (T::BM + 2 * T::BN) * 4; }

    // the tile's biases, labels (counted from the tile's first class; far below
    // 0 without one) and lse
    template <class T>
    __device__ __forceinline__ void begin(const gemm::Place &at, char *own) const {
        float *b = reinterpret_cast<float *>(own);
        for (int x = threadIdx.x; x < T::BM + T::BN; x += T::THREADS) {
            const int c = x - T::BM, col = at.tile_n * T::BN + c;
            if (c < 0) {
                b[x] = bias[at.tile_m * T::BM + x];
            } else {
                const int l = col < rows.n ? rows.label[col] : -1;
                reinterpret_cast<int32_t *>(b)[x] = l < 0 ? kNoLabel : l - class0 - at.tile_m * T::BM;
                b[x + T::BN] = col < rows.n ? rows.lse[col] : 0.f;
            }
        }
    }

    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *lds,
                                        const char *own) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int n = rows.n;
        const int m0 = at.tile_m * T::BM, n0 = at.tile_n * T::BN;
        const int r0 = at.row0 - m0, c0 = at.col0 - n0;
        const float *own_bias = reinterpret_cast<const float *>(own) + r0;
        const float *own_cols = reinterpret_cast<const float *>(own) + T::BM + c0;
        int t[T::TN];  // label, counted from the wavefront's first class
        bool on[T::TN];
        float lse[T::TN];
        bool here = false;
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            const int l = __float_as_int(own_cols[32 * j + (lane & 31)]);
            on[j] = l != kNoLabel;
            t[j] = l - r0;
            here |= t[j] >= 0 && t[j] < 32 * T::TM;
            lse[j] = own_cols[T::BN + 32 * j + (lane & 31)];
        }
        const bool labels = __any(here);  // few wavefronts hold a row's label
        const float f = pbias ? *factor : 0.f;
        uint32_t pk[T::TM][T::TN][4][2][PG];  // four classes of a row, twice two
#pragma unroll
        for (int i = 0; i < T::TM; ++i) {
            float sum[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] = 0.f;
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = 32 * i + 8 * q + 4 * (lane >> 5);
                    const float4 b4 = *reinterpret_cast<const float4 *>(own_bias + row);
                    const float b[4] = {b4.x, b4.y, b4.z, b4.w};
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float z = acc[i][j][4 * q + r] * planes::kBack<P> + b[r];
                        v[r] = on[j] ? __expf(z - lse[j]) : 0.f;  // whatever a row without a label holds
                    }
                    if (labels)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r == t[j]) v[r] -= 1.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[4 * q + r] += v[r];
                    planes::split_pair<PG>(v[0], v[1], pk[i][j][q][0]);
                    planes::split_pair<PG>(v[2], v[3], pk[i][j][q][1]);
                }
            if (pbias) {
                // over the 32 lanes: halves of the values are exchanged, so that
                // each lane adds half as many in the next round
                const int e = sum32(sum);
                const int row = at.row0 + 32 * i + gemm::acc_row(e);
                if ((lane & 16) == 0 && row < K)
                    pbias[((int64_t)at.tile_n * T::WN + wave % T::WN) * K + row] = sum[0] * f;
            }
        }
        planes::store_both<T, PG>(pk, at, lds, g, ldg, (int64_t)n * ldg, n, Kp, gt, ldt, (int64_t)K * ldt, K, np);
    }
};

// Epilogue of a gradient's product: fp32 partial sums [split][rows][cols],
// begun, or added to: the accumulators then start as them (reading them at the
// end, with nothing left to multiply, took 55 of 330 us for 8192 x 1024 sums).
// A product in one part and one piece gives the gradient itself.
template <int P>
struct Part : gemm::Simple {
    float *out;
    int rows, cols;
    bool add;
    void *result;         // the gradient, or null
    const float *factor;  // s

    Part(float *out, int rows, int cols, bool add, void *result, const float *factor)
        : out(out), rows(rows), cols(cols), add(add), result(result), factor(factor) {}

    template <class T, class F>
    __device__ __forceinline__ void each(const gemm::Place &at, F &&f) const {
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = at.row0 + 32 * i + gemm::acc_row(e), col = at.col0 + 32 * j + (threadIdx.x & 31);
                    if (row < rows && col < cols) f((int64_t)row * cols + col, i, j, e);
                }
    }
    template <class T>
    __device__ __forceinline__ void init(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at) const {
        const float *o = out + (int64_t)at.split * rows * cols;
        if (add) each<T>(at, [&](int64_t to, int i, int j, int e) { acc[i][j][e] = o[to] * (1.f / planes::kBack<P>); });
    }
    template <class T>
    __device__ __forceinline__ void run(gemm::f32x16_t (&acc)[T::TM][T::TN], const gemm::Place &at, char *, char *) const {
        if (result) {
            const float s = *factor;
            each<T>(at, [&](int64_t to, int i, int j, int e) {
                const float v = acc[i][j][e] * planes::kBack<P> * s;
                if (P == 1)
                    reinterpret_cast<uint16_t *>(result)[to] = (uint16_t)pack_bf16(v, 0.f);
                else
                    reinterpret_cast<float *>(result)[to] = v;
            });
            return;
        }
        float *o = out + (int64_t)at.split * rows * cols;
        each<T>(at, [&](int64_t to, int i, int j, int e) { o[to] = acc[i][j][e] * planes::kBack<P>; });
    }
};

// The gradient from the partial sums of its product's splits and the factor s.
template <bool BF16>
__global__ __launch_bounds__(256) void k_join(const float *__restrict__ part, int splits, int64_t n,
                                              const float *factor, void *out) {
    const float f = splits > 0 ? *factor : 0.f;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        float s = 0.f;  // without any part, zeros
        int k = 0;
        for (; k + 8 <= splits; k += 8) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = part[(k + u) * n + i];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += x[u];
        }
        for (; k < splits; ++k) s += part[k * n + i];
        s *= f;
        if (BF16)
            reinterpret_cast<uint16_t *>(out)[i] = (uint16_t)pack_bf16(s, 0.f);
        else
            reinterpret_cast<float *>(out)[i] = s;
    }
}

struct FewTile {
    static constexpr int BM = 128, BN = 64, WM = 4, WN = 1, TM = 1, TN = 2, THREADS = 256;
};

// Tiles: classes x rows for the logits, rows x channels and classes x channels
// for the gradients.
template <int P>
struct Tiles;
template <>
struct Tiles<1> {
    using Large = gemm::Tile<256, 256, 4, 2, 64, 1>;
    using Middle = gemm::Tile<128, 128, 2, 2, 64, 1>;
    using Few = gemm::Tile<128, 64, 4, 1, 64, 1>;
    using Small = gemm::Tile<64, 64, 2, 2, 64, 1>;
    using Thin = Small;
};
template <>
struct Tiles<3> {
    using Large = gemm::Tile<256, 128, 4, 2, 32, 3>;
    using Middle = gemm::Tile<128, 128, 2, 2, 32, 3>;
    using Few = gemm::Tile<128, 64, 4, 1, 32, 3>;
    using Small = gemm::Tile<64, 64, 2, 2, 32, 3>;
    using Thin = gemm::Tile<64, 64, 2, 2, 64, 3>;
};

enum { LARGE, MIDDLE, FEW, STRAIGHT, SMALL, THIN };  // STRAIGHT: FewTile, of k_few

// The large tile reads the least; it is for products with enough of them to go
// round, and the one of 64 columns for few.
template <int P>
int tile_for(int64_t m, int64_t n, int cu) {
    using L = typename Tiles<P>::Large;
    if (n <= 64) return FEW;
    const int64_t large = (m + L::BM - 1) / L::BM * ((n + L::BN - 1) / L::BN);
    return large * 4 >= (int64_t)cu * 3 ? LARGE : MIDDLE;
}

template <int P>
int tile_m(int kind) {
    using X = Tiles<P>;
    const int of[] = {X::Large::BM, X::Middle::BM, X::Few::BM, FewTile::BM, X::Small::BM, X::Thin::BM};
    return of[kind];
}

template <int P>
int tile_n(int kind) {
    using X = Tiles<P>;
    const int of[] = {X::Large::BN, X::Middle::BN, X::Few::BN, FewTile::BN, X::Small::BN, X::Thin::BN};
    return of[kind];
}

template <int P>
int64_t tile_count(int kind, int64_t m, int64_t n) {
    return (m + tile_m<P>(kind) - 1) / tile_m<P>(kind) * ((n + tile_n<P>(kind) - 1) / tile_n<P>(kind));
}

// Columns' partial rows of the bias gradient that a product over n rows gives.
template <int P>
int64_t bias_rows(int kind, int64_t n) {
    using X = Tiles<P>;
    const int64_t wn = kind == LARGE ? X::Large::WN : kind == MIDDLE ? X::Middle::WN : kind == SMALL ? X::Small::WN : 1;
    return (n + tile_n<P>(kind) - 1) / tile_n<P>(kind) * wn;
}

// Splits of a contraction of k for m x n tiles that do not fill the chip, each of
// 256 values at least (100 x 256 over 50000 rows in fp32: 38 us in 112 parts and
// 7 to join them, 146 and 17 in 16).
template <int P>
int splits_for(int kind, int64_t m, int64_t n, int64_t k, int cu) {
    const int64_t t = tile_count<P>(kind, m, n);
    int64_t s = cu / t > 1 ? cu / t : 1;  // no more workgroups than CUs: one more takes as long again
    const int64_t most = k / 256 > 0 ? k / 256 : 1;
    s = s < most ? s : most;
    return (int)(s < 128 ? s : 128);
}

// For products whose contraction of k may be split.  Short contractions are
// bound by what they write, and many small workgroups on a CU write while others
// load (21384 x 472 over 43 rows in fp32: 24 us, 31 in large tiles; over 120
// rows 33 and 38, in bf16 17 and 23; 50000 x 256 over 100 classes 42 and 43, in
// bf16 20 and 25).  Few rows leave most of a tile of 128 empty (43 x 472 over
// 21384: 19 us, 46 in 128 x 128).  Else the large tile too where parts of it
// that fill the chip are long.
template <int P>
int split_tile_for(int64_t m, int64_t n, int64_t k, int cu) {
    if (k <= 128) return SMALL;
    if (m <= 64) return THIN;
    const int kind = tile_for<P>(m, n, cu);
    using L = typename Tiles<P>::Large;
    if (kind != MIDDLE || m < L::BM || n < L::BN) return kind;
    return k / splits_for<P>(LARGE, m, n, k, cu) >= 1024 ? LARGE : MIDDLE;
}

// For the logits, whose contraction is not split: the smallest tile where the
// middle one would leave half the CUs idle (1332 x 439 over 1536 channels in
// bf16: 10.6 us, and 14.4).
template <int P>
int logit_tile_for(int64_t m, int64_t n, int cu) {
    const int kind = tile_for<P>(m, n, cu);
    return kind == MIDDLE && tile_count<P>(MIDDLE, m, n) * 2 < cu ? SMALL : kind;
}

template <int P, class E>
hipError_t product(hipStream_t st, int kind, const gemm::Operand &A, const gemm::Operand &B, int64_t K, int64_t part,
                   const E &e) {
    using X = Tiles<P>;
    if constexpr (!std::is_same<E, Grad<1, 2>>::value)  // the plan has no large tile for it
        if (kind == LARGE) return gemm::launch<typename X::Large>(st, A, B, K, part, 1, false, e);
    if (kind == MIDDLE) return gemm::launch<typename X::Middle>(st, A, B, K, part, 1, false, e);
    if (kind == SMALL) return gemm::launch<typename X::Small>(st, A, B, K, part, 1, false, e);
    if (kind == THIN) return gemm::launch<typename X::Thin>(st, A, B, K, part, 1, false, e);
    return gemm::launch<typename X::Few>(st, A, B, K, part, 1, false, e);
}

// Workgroups of k_lse for n rows: 4 threads a row, or where that leaves CUs
// without work a wavefront.
bool lse_wide(const lattice_dense *D, int64_t n) { return n < (int64_t)64 * D->cu_count; }
int64_t lse_blocks(const lattice_dense *D, int64_t n) { return lse_wide(D, n) ? (n + 3) / 4 : (n + 63) / 64; }

// The first pass for at most 64 rows, straight from the caller's w: it is read
// once, by lanes that each take the 8 channels of a class that their operand of
// a product holds, and split there; laying it out first would read and write it
// twice more (18 rows against 61228 x 1209 in fp32: 250 us so, and 79, 3.7 TB/s
// of w, straight).  The rows' planes go through LDS in slices of 64 channels, of
// 32 rows only where there are no more.  Four wavefronts of 32 classes each: what
// a CU's wavefronts read of scattered rows of w adds up, so that fewer to a CU
// are faster where there are CUs left (5 rows against 6450 x 1132: 34 us, 51 with
// eight), and with two the rows' planes are read too often (97 of 79 us above).
template <bool BF16>
__global__ __launch_bounds__(256, BF16 ? 4 : 2) void k_few(const void *__restrict__ w, int64_t w_stride, int K, int C,
                                                                   gemm::Operand X, Stats<BF16 ? 1 : 3> epi) {
    constexpr int P = BF16 ? 1 : 3, SLICE = P * 64 * 64 * 2;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = gemm::wave_index();
    gemm::Place at;
    at.tile_m = blockIdx.x;
    at.tile_n = at.split = at.batch = 0;
    at.row0 = blockIdx.x * FewTile::BM + 32 * wave;
    at.col0 = 0;
    epi.template begin<FewTile>(at, lds + 2 * SLICE);
    const int k = at.row0 + (lane & 31);
    const char *row = reinterpret_cast<const char *>(w) + (int64_t)(k < K ? k : K - 1) * w_stride * (BF16 ? 2 : 4);
    // a wavefront's load brings 8 rows of a plane of x: 8 chunks of 16 bytes a row,
    // swizzled as in gemm.h
    gemm::rsrc_t from[P];
#pragma unroll
    for (int p = 0; p < P; ++p) from[p] = gemm::buffer(X.p + p * X.plane);
    constexpr int NW = FewTile::WM, U = 8 / NW;
    uint32_t off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int xr = 8 * (NW * u + wave) + lane / 8;
        off[u] = (uint32_t)(xr < X.rows ? xr : X.rows - 1) * (uint32_t)(X.ld * 2) + ((lane & 7) ^ ((xr >> 1) & 7)) * 16;
    }
    const bool both = X.rows > 32;  // halves of the tile's columns
    auto bring = [&](int buf, int c0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < U / 2 || both)
#pragma unroll
                for (int p = 0; p < P; ++p)
                    gemm::dma16(from[p], off[u], (uint32_t)c0 * 2, lds + buf * SLICE + p * 8192 + (NW * u + wave) * 1024);
    };
    Raw<BF16, 8> now[4], next[4];
    auto read = [&](int c0) {
        if (c0 + 64 <= C) {
#pragma unroll
            for (int s = 0; s < 4; ++s) load_raw<BF16, 8>(row, c0 + 16 * s + 8 * (lane >> 5), 1 << 30, next[s]);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) load_raw<BF16, 8>(row, c0 + 16 * s + 8 * (lane >> 5), C, next[s]);
        }
    };
    gemm::f32x16_t acc[1][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[0][j][e] = 0.f;
    bring(0, 0);
    read(0);
    int buf = 0;
    for (int c0 = 0; c0 < C; c0 += 64, buf ^= 1) {
        gemm::wait_and_barrier<0>();  // this slice is there, the other one is read no more
#pragma unroll
        for (int s = 0; s < 4; ++s) now[s] = next[s];
        if (c0 + 64 < C) {
            bring(buf ^ 1, c0 + 64);
            read(c0 + 64);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            gemm::bf16x8_t a[P], b[P][2];
            if constexpr (BF16) {
                a[0] = __builtin_bit_cast(gemm::bf16x8_t, gemm::u32x4_t{now[s].w[0], now[s].w[1], now[s].w[2], now[s].w[3]});
            } else {
                float v[8];
                unpack<BF16, 8>(now[s], v);
                uint32_t h[4][P];
#pragma unroll
                for (int i = 0; i < 4; ++i) planes::split_pair<P>(v[2 * i], v[2 * i + 1], h[i]);
#pragma unroll
                for (int p = 0; p < P; ++p)
                    a[p] = __builtin_bit_cast(gemm::bf16x8_t, gemm::u32x4_t{h[0][p], h[1][p], h[2][p], h[3][p]});
            }
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (j > 0 && !both) continue;
                    const int r = 32 * j + (lane & 31), chunk = 2 * s + (lane >> 5);
                    b[p][j] = *reinterpret_cast<const gemm::bf16x8_t *>(lds + buf * SLICE + p * 8192 +
                                                                        (r * 8 + (chunk ^ ((r >> 1) & 7))) * 16);
                }
#pragma unroll
            for (int t = P - 1; t >= 0; --t)  // the smaller products first
#pragma unroll
                for (int p = 0; p <= t; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (j == 0 || both) acc[0][j] = gemm::mfma(a[p], b[t - p][j], acc[0][j]);
        }
    }
    gemm::wait_and_barrier<0>();
    epi.template run<FewTile>(acc, at, lds, lds + 2 * SLICE);
}

template <int P>
hipError_t launch_few(hipStream_t st, const LossArgs &a, const gemm::Operand &X, const Stats<P> &e) {
    constexpr int LDS = 2 * P * 64 * 64 * 2 + Stats<P>::template extra<FewTile>();
    static_assert(Stats<P>::template lds<FewTile>() <= 2 * P * 64 * 64 * 2 && LDS <= 64 * 1024, "LDS");
    hipLaunchKernelGGL((k_few<P == 1>), dim3((a.K + FewTile::BM - 1) / FewTile::BM), dim3(FewTile::THREADS), LDS, st, a.w, a.w_stride, a.K, a.C, X, e);
    return hipGetLastError();
}

template <int P, class E>
hipError_t again(hipStream_t st, int kind, const gemm::Store &kept, const E &e) {
    using X = Tiles<P>;
    if (kind == LARGE) return gemm::launch_again<typename X::Large>(st, kept, e);
    if (kind == MIDDLE) return gemm::launch_again<typename X::Middle>(st, kept, e);
    if (kind == SMALL) return gemm::launch_again<typename X::Small>(st, kept, e);
    if (kind == FEW) return gemm::launch_again<typename X::Few>(st, kept, e);
    return gemm::launch_again<FewTile>(st, kept, e);
}

// Sizes of the pieces and where everything lies in the scratch.  PG: planes of G.
template <int P, int PG>
struct Plan {
    int64_t R;           // rows of a piece
    int64_t Kpad;        // classes in whole tiles
    int64_t KP;          // classes of a piece
    int fkind, gkind;    // tiles of the two passes over the logits
    int xkind, wkind;    // of the gradients' products
    int64_t xpart, wpart;      // lengths of their contractions' parts
    int64_t xsplits, wsplits;  // and how many there are at most
    bool own_x, own_w;   // operands that have to be laid out first
    bool keep;           // the logits of a piece of rows
    bool one_piece;      // of rows, and of classes
    int64_t count, bias, label, factor, lse, picked, stats, part, xp, xt, wp, wt, g, gt, pbias, bias_acc, px, pw, kept, bytes;
    int64_t parts;       // partial sums of the loss

    Plan(const lattice_dense *D, const LossArgs &a) {
        const int cu = D->cu_count;
        const int64_t C = a.C, K = a.K;
        const int64_t Cl = gemm::row_length(C);
        Kpad = (K + 255) / 256 * 256;
        R = a.N < kMaxPiece ? a.N : kMaxPiece;
        // tiles' statistics of a piece: at most 256 MiB
        const int64_t most = ((int64_t)1 << 25) / (Kpad / 128);
        if (R > most) R = most < 256 ? 256 : most / 256 * 256;
        if (R < 1) R = 1;
        keep = P == 3 && C >= 192 && a.any_grad();
        if (keep && R > 256 && R * Kpad > kKeep / 4) R = kKeep / 4 / Kpad > 256 ? kKeep / 4 / Kpad / 256 * 256 : 256;
        const int64_t Rp = gemm::padded(R), Rl = gemm::row_length(R);
        KP = kPieceBytes / (Rp * PG * 2 * 2) / 256 * 256;
        KP = KP < 256 ? 256 : KP;
        KP = KP < Kpad ? KP : Kpad;
        const int64_t kp = KP < K ? KP : K;
        one_piece = a.N <= R && K <= KP;
        auto as_is = [&](const void *q, int64_t stride) {
            return P == 1 && C % gemm::kPad == 0 && stride % 8 == 0 && stride < gemm::kMaxLd && ((uintptr_t)q & 15) == 0;
        };
        // few rows: w as it is, if nothing else wants its planes
        const bool few = a.N <= 64 && (P == 3 ? !a.any_grad() || keep : !a.any_grad() && !as_is(a.w, a.w_stride));
        fkind = few ? STRAIGHT : logit_tile_for<P>(K, R, cu);
        gkind = keep ? fkind : logit_tile_for<P>(kp, R, cu);
        // two planes beside the large tile's sums do not fit the registers
        if (PG != P && gkind == LARGE) gkind = MIDDLE;
        xkind = split_tile_for<P>(R, C, kp, cu);
        wkind = split_tile_for<P>(kp, C, R, cu);
        xpart = gemm::part_length(gemm::padded(kp), splits_for<P>(xkind, R, C, kp, cu));
        wpart = gemm::part_length(Rp, splits_for<P>(wkind, kp, C, R, cu));
        xsplits = (gemm::padded(kp) + xpart - 1) / xpart;
        wsplits = (Rp + wpart - 1) / wpart;
        own_x = few || !as_is(a.x, a.x_stride);
        own_w = !few && !as_is(a.w, a.w_stride);
        ScratchLayout s;
        count = s.take(kCounts * 4);
        bias = s.take(Kpad * 4);
        label = s.take(R * 4);
        factor = s.take(4);
        lse = s.take(R * 4);
        picked = s.take(R * 4);
        const int64_t bm = tile_m<P>(fkind);
        stats = s.take((K + bm - 1) / bm * R * 8);
        parts = 0;
        for (int64_t r = 0; r < a.N; r += R) parts += lse_blocks(D, a.N - r < R ? a.N - r : R);
        part = s.take(parts * 8);
        xp = own_x ? s.take(P * R * Cl * 2) : 0;
        wp = own_w ? s.take(P * K * Cl * 2) : 0;
        xt = a.grad_w ? s.take(P * C * Rl * 2) : 0;
        wt = a.grad_x ? s.take(P * C * gemm::row_length(K) * 2) : 0;
        g = a.grad_x ? s.take(PG * R * gemm::row_length(kp) * 2) : 0;
        gt = a.grad_w ? s.take(PG * kp * Rl * 2) : 0;
        if (a.grad_bias) {
            const int64_t rows = bias_rows<P>(gkind, R);
            pbias = s.take((rows * kp + rowsum::scratch_floats(rows, kp)) * 4);
            const int64_t pieces = (a.N + R - 1) / R;
            bias_acc = s.take((pieces < kHeld ? pieces : kHeld) * K * 4);
        }
        px = a.grad_x ? s.take(PG == P && one_piece && xsplits == 1 ? 0 : xsplits * R * C * 4) : 0;
        pw = a.grad_w ? s.take(PG == P && a.N <= R && wsplits == 1 ? 0 : wsplits * K * C * 4) : 0;
        kept = keep ? s.take(tile_count<P>(fkind, K, R) * tile_m<P>(fkind) * tile_n<P>(fkind) * 4) : 0;
        bytes = s.bytes;
    }
};

template <int P, int PG>
hipError_t run(lattice_dense *D, const LossArgs &a) {
    const Plan<P, PG> p(D, a);
    char *ws = reinterpret_cast<char *>(D->ws);
    hipStream_t st = D->stream;
    auto f = [&](int64_t at) { return reinterpret_cast<float *>(ws + at); };
    auto h = [&](int64_t at) { return reinterpret_cast<uint16_t *>(ws + at); };
    auto ints = [&](int64_t at) { return reinterpret_cast<int32_t *>(ws + at); };
    const int C = a.C, K = a.K;
    const int64_t Cp = gemm::padded(C);
    const int esz = a.bf16 ? 2 : 4;
    constexpr int BF = P == 1;

    const int first = (int)(a.N < p.R ? a.N : p.R);
    auto layout = [&](const void *from, int64_t stride, int64_t rows, bool labelled, uint16_t *to, uint16_t *to_t) {
        const planes::Source s = {from, stride, 0, (int)rows, C, nullptr, labelled ? a.target : nullptr, K, a.ignore};
        const int bx = (int)(Cp / 64);
        return Layout{s, to, to_t, gemm::row_length(C), gemm::row_length(rows), bx,
                      to || to_t ? bx * (int)(gemm::padded(rows) / 64) : 0};
    };
    const Layout lw = layout(a.w, a.w_stride, K, false, p.own_w ? h(p.wp) : nullptr, a.grad_x ? h(p.wt) : nullptr);
    const Layout lx = layout(a.x, a.x_stride, first, true, p.own_x ? h(p.xp) : nullptr, a.grad_w ? h(p.xt) : nullptr);
    hipLaunchKernelGGL((k_begin<P == 1, P>), dim3(kCounts + lw.blocks + lx.blocks), dim3(256), 0, st, a.target, a.N,
                       first, K, a.ignore, ints(p.count), D->status, ints(p.label), a.bias, (int)p.Kpad, f(p.bias), lw,
                       lx);
    TRY(hipGetLastError());
    gemm::Operand W = {reinterpret_cast<const uint16_t *>(a.w), a.w_stride, 0, 0, K};
    if (p.own_w) W = planes::operand(h(p.wp), K, C, P);
    // gradients that their product's epilogue writes as they are
    const bool x_at_once = PG == P && p.one_piece && p.xsplits == 1;
    const bool w_at_once = PG == P && a.N <= p.R && p.wsplits == 1;
    constexpr int MORE = PG - P;  // planes of G that are multiplied apart: the smaller ones, first
    int64_t parts = 0;
    int piece = 0, held = 0;  // pieces, and rows of bias_acc that wait to be added
    for (int64_t r0 = 0; r0 < a.N; r0 += p.R, ++piece) {
        if (a.grad_bias && held == kHeld) {
            // into the first of them: a workgroup reads all of its columns before it writes them
            TRY(rowsum::sum(st, f(p.bias_acc), held, K, nullptr, f(p.bias_acc)));
            held = 1;
        }
        const int n = (int)(a.N - r0 < p.R ? a.N - r0 : p.R);
        const int64_t np = gemm::padded(n);
        const char *x = reinterpret_cast<const char *>(a.x) + r0 * a.x_stride * esz;
        if (piece > 0) {
            hipLaunchKernelGGL(k_labels, dim3((n + 255) / 256), dim3(256), 0, st, a.target + r0, n, K, a.ignore,
                               ints(p.label));
            TRY(hipGetLastError());
        }
        gemm::Operand X = {reinterpret_cast<const uint16_t *>(x), a.x_stride, 0, 0, n};
        if (piece > 0 && (p.own_x || a.grad_w)) {
            const planes::Source s = {x, a.x_stride, 0, n, C, nullptr, a.target + r0, K, a.ignore};
            TRY(planes::launch<P>(st, a.bf16, s, 1, p.own_x ? h(p.xp) : nullptr, a.grad_w ? h(p.xt) : nullptr));
        }
        if (p.own_x) X = planes::operand(h(p.xp), n, C, P);
        const int bm = tile_m<P>(p.fkind), bn = tile_n<P>(p.fkind);
        const int tiles = (K + bm - 1) / bm, tiles_n = (n + bn - 1) / bn;
        const gemm::Store kept(p.keep ? f(p.kept) : nullptr, {(int)Cp, (int)Cp, tiles, tiles_n, false}, 1);
        const Stats<P> stats = {{}, f(p.bias), ints(p.label), n, reinterpret_cast<float2 *>(ws + p.stats), f(p.picked), kept};
        if (p.fkind == STRAIGHT)
            TRY(launch_few<P>(st, a, X, stats));
        else
            TRY((product<P>(st, p.fkind, W, X, Cp, Cp, stats)));
        const unsigned lse_grid = (unsigned)lse_blocks(D, n);
        float *row_loss = a.rows ? a.rows + r0 : nullptr;
        double *part = reinterpret_cast<double *>(ws + p.part) + parts;
        if (lse_wide(D, n))
            hipLaunchKernelGGL(k_lse<64>, dim3(lse_grid), dim3(256), 0, st, stats.stats, tiles, n, f(p.picked),
                               ints(p.label), f(p.lse), row_loss, part, ints(p.count), a.mean, f(p.factor));
        else
            hipLaunchKernelGGL(k_lse<4>, dim3(lse_grid), dim3(256), 0, st, stats.stats, tiles, n, f(p.picked),
                               ints(p.label), f(p.lse), row_loss, part, ints(p.count), a.mean, f(p.factor));
        TRY(hipGetLastError());
        parts += lse_grid;
        if (!a.any_grad()) continue;
        for (int64_t k0 = 0; k0 < K; k0 += p.KP) {
            const int kn = (int)(K - k0 < p.KP ? K - k0 : p.KP);
            const int64_t kp = gemm::padded(kn);
            gemm::Operand Wk = W;
            Wk.p += k0 * W.ld;
            Wk.rows = kn;
            const Grad<P, PG> grad = {{}, f(p.bias) + k0, {ints(p.label), f(p.lse), n}, (int)k0, kn, (int)kp, (int)np,
                                      gemm::row_length(kn), gemm::row_length(n),
                                      a.grad_x ? h(p.g) : nullptr, a.grad_w ? h(p.gt) : nullptr,
                                      a.grad_bias ? f(p.pbias) : nullptr, f(p.factor)};
            bool formed = false;
            if constexpr (P == 3) {
                if (p.keep) {
                    gemm::Store of = kept;  // the piece's tiles
                    of.out += k0 / bm * tiles_n * (int64_t)bm * bn;
                    of.s.tiles_m = (kn + bm - 1) / bm;
                    TRY((again<P>(st, p.gkind, of, grad)));
                    formed = true;
                }
            }
            if (!formed) TRY((product<P>(st, p.gkind, Wk, X, Cp, Cp, grad)));
            if (a.grad_bias) {
                const int64_t rows = bias_rows<P>(p.gkind, n);
                float *to = a.N <= p.R ? a.grad_bias + k0 : f(p.bias_acc) + (int64_t)held * K + k0;
                TRY(rowsum::sum(st, f(p.pbias), rows, kn, f(p.pbias) + rows * kn, to));
            }
            if (a.grad_x) {
                gemm::Operand Wt = planes::operand(h(p.wt), C, K, P);
                Wt.p += k0;
                for (int q = MORE; q >= 0; --q)
                    TRY((product<P>(st, p.xkind,
                                    planes::operand(h(p.g) + q * n * gemm::row_length(kn), n, kn, P), Wt, kp, p.xpart,
                                    Part<P>{f(p.px), n, C, k0 > 0 || q < MORE, x_at_once ? a.grad_x : nullptr,
                                            f(p.factor)})));
            }
            if (a.grad_w) {
                float *sums = f(p.pw) + k0 * C * p.wsplits;
                for (int q = MORE; q >= 0; --q)
                    TRY((product<P>(st, p.wkind,
                                    planes::operand(h(p.gt) + q * kn * gemm::row_length(n), kn, n, P),
                                    planes::operand(h(p.xt), C, n, P), np, p.wpart,
                                    Part<P>{sums, kn, C, r0 > 0 || q < MORE,
                                            w_at_once ? reinterpret_cast<char *>(a.grad_w) + k0 * C * esz : nullptr,
                                            f(p.factor)})));
                if (r0 + p.R >= a.N && !w_at_once) {
                    const int64_t v = (int64_t)kn * C;
                    // a later piece of rows is no longer than the first, and has no more parts
                    const int splits = (int)(piece > 0 ? p.wsplits : (np + p.wpart - 1) / p.wpart);
                    hipLaunchKernelGGL((k_join<BF>), dim3(grid_for(v, 256, D->cu_count)), dim3(256), 0, st, sums,
                                       splits, v, f(p.factor), reinterpret_cast<char *>(a.grad_w) + k0 * C * esz);
                    TRY(hipGetLastError());
                }
            }
        }
        ++held;
        if (a.grad_x && !x_at_once) {
            const int64_t v = (int64_t)n * C;
            hipLaunchKernelGGL((k_join<BF>), dim3(grid_for(v, 256, D->cu_count)), dim3(256), 0, st, f(p.px),
                               (int)p.xsplits, v, f(p.factor),
                               reinterpret_cast<char *>(a.grad_x) + r0 * C * esz);
            TRY(hipGetLastError());
        }
    }
    hipLaunchKernelGGL(k_total, dim3(1), dim3(256), 0, st, reinterpret_cast<const double *>(ws + p.part), parts,
                       ints(p.count), a.mean, a.loss);
    TRY(hipGetLastError());
    if (a.grad_bias && piece != 1) TRY(rowsum::sum(st, f(p.bias_acc), held, K, nullptr, a.grad_bias));
    if (a.N == 0 && a.grad_w) {
        const int64_t v = (int64_t)K * C;
        hipLaunchKernelGGL((k_join<BF>), dim3(grid_for(v, 256, D->cu_count)), dim3(256), 0, st, nullptr, 0, v, nullptr,
                           a.grad_w);
        TRY(hipGetLastError());
    }
    return hipSuccess;
}

}  // namespace

int64_t loss_scratch(const lattice_dense *D, const LossArgs &a) {
    if (loss_fused_covers(a)) return loss_fused_scratch(D, a);
    if (!a.bf16) return Plan<3, 3>(D, a).bytes;
    return a.split && a.any_grad() ? Plan<1, 2>(D, a).bytes : Plan<1, 1>(D, a).bytes;
}

hipError_t launch_loss(lattice_dense *D, const LossArgs &a) {
    if (loss_fused_covers(a)) return launch_loss_fused(D, a);
    if (!a.bf16) return run<3, 3>(D, a);
    return a.split && a.any_grad() ? run<1, 2>(D, a) : run<1, 1>(D, a);
}
