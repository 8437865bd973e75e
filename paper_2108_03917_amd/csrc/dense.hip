// Host side of the dense operators declared in include/lattice.h: argument
// checking, the handle with its scratch and device status, and dispatch to the
// kernels of norm.hip, loss.hip, update.hip, attention.hip, attention_bwd.hip,
// rotate.hip and clip.hip.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <new>

#include "dense.h"

namespace {

void set_err(lattice_dense *D, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(D->err, sizeof(D->err), fmt, ap);
    va_end(ap);
}

lattice_status hip_fail(lattice_dense *D, hipError_t e, const char *what) {
    set_err(D, "%s: %s", what, hipGetErrorString(e));
    return e == hipErrorOutOfMemory ? LATTICE_E_NOMEM : LATTICE_E_HIP;
}

// Whether calls on the handle's stream are being captured (the null stream is
// never).
bool capturing(const lattice_dense *D) {
    if (!D->stream) return false;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(D->stream, &status) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    return status != hipStreamCaptureStatusNone;
}

// hipMalloc, also while a stream of this thread is being captured in a mode that
// forbids it: an allocation is no part of the graph.
hipError_t allocate(void **p, int64_t bytes, bool captured) {
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    if (captured) TRY(hipThreadExchangeStreamCaptureMode(&mode));
    const hipError_t e = hipMalloc(p, bytes);
    if (captured) (void)hipThreadExchangeStreamCaptureMode(&mode);
    return e;
}

// Grow the scratch to at least `need` bytes (a device allocation, only when it
// is too small; freeing the old one waits for the work that uses it).  A graph
// goes on using the scratch that its calls were captured with: that one is
// kept until the handle is destroyed, and so is any that is replaced during a
// capture, which cannot wait.
lattice_status grow(lattice_dense *D, int64_t need, const char *what) {
    if (need <= 0) return LATTICE_OK;
    const bool now = capturing(D);
    if (need <= D->ws_bytes) {
        D->ws_captured |= now;
        return LATTICE_OK;
    }
    if (D->ws && (D->ws_captured || now)) {
        KeptScratch *k = new (std::nothrow) KeptScratch{D->ws, D->kept};
        if (!k) {
            set_err(D, "%s: out of host memory", what);
            return LATTICE_E_NOMEM;
        }
        D->kept = k;
    } else if (D->ws) {
        const hipError_t e = hipFree(D->ws);
        if (e != hipSuccess) return hip_fail(D, e, what);
    }
    D->ws = nullptr;
    D->ws_bytes = 0;
    D->ws_captured = now;
    if (allocate(&D->ws, need, now) != hipSuccess) {
        (void)hipGetLastError();
        D->ws = nullptr;
        set_err(D, "%s: cannot allocate %lld bytes of scratch", what, (long long)need);
        return LATTICE_E_NOMEM;
    }
    D->ws_bytes = need;
    return LATTICE_OK;
}

// Makes the handle's device the current one for a call, whichever the caller's is:
// allocations and launches go to the current device, the null stream's too.
struct OnDevice {
    int before = -1;
    hipError_t error;
    explicit OnDevice(const lattice_dense *D) {
        int now = 0;
        error = hipGetDevice(&now);
        if (error != hipSuccess || now == D->device) return;
        error = hipSetDevice(D->device);
        if (error == hipSuccess) before = now;
    }
    ~OnDevice() {
        if (before >= 0) (void)hipSetDevice(before);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
};

bool is_storage(lattice_dtype t) { return t == LATTICE_F32 || t == LATTICE_BF16; }

// Bytes of rows x C values at `stride` values a row (0 for no rows).
int64_t span(int64_t rows, int64_t C, int64_t stride, lattice_dtype t) {
    return rows > 0 ? ((rows - 1) * stride + C) * (t == LATTICE_BF16 ? 2 : 4) : 0;
}

bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int kMaxChannels = 1 << 20;
constexpr int64_t kMaxStride = (int64_t)1 << 31;

lattice_status check_rows(lattice_dense *D, const lattice *rows_of, int64_t rows, int C, const char *what) {
    if (rows < 0 || rows > kMaxRows || C < 1 || C > kMaxChannels) {
        set_err(D, "%s: rows = %lld outside [0, 2^31] or C = %d outside [1, 2^20]", what, (long long)rows, C);
        return LATTICE_E_ARG;
    }
    if (!rows_of) return LATTICE_OK;
    if (!rows_of->splatted) {
        set_err(D, "%s: the lattice of the rows has not been splatted", what);
        return LATTICE_E_STATE;
    }
    if (rows_of->device != D->device || rows_of->stream != D->stream) {
        set_err(D, "%s: the lattice of the rows is on another device or stream", what);
        return LATTICE_E_ARG;
    }
    return LATTICE_OK;
}

// Values from the first to behind the last of a [rows][heads][C] tensor with these
// strides (0 for none).
int64_t extent(int64_t rows, int64_t heads, int64_t C, int64_t row, int64_t head) {
    return rows > 0 && heads > 0 ? (rows - 1) * row + (heads - 1) * head + C : 0;
}

// Whether the heads' rows of a tensor that is written lie apart from each other.
bool apart(int64_t rows, int64_t heads, int64_t C, int64_t row, int64_t head) {
    const bool r = rows <= 1, h = heads <= 1;
    if (r && h) return true;
    if (r) return head >= C;
    if (h) return row >= C;
    return (head >= C && row >= (heads - 1) * head + C) || (row >= C && head >= (rows - 1) * row + C);
}

// Strides that go forward, to no more values than there are addresses (2^48 bytes).
bool strides_ok(int64_t rows, int64_t heads, int64_t row, int64_t head) {
    return row >= 0 && head >= 0 && (double)(rows - 1) * (double)row + (double)(heads - 1) * (double)head < 0x1p47;
}

// A tensor that is read, or written, by an operator on heads.
struct Heads {
    const char *name;
    const void *p;
    int64_t rows, heads, row, head;
    lattice_dtype type;
    bool written;
    int may_be;  // index of the tensor that this one may be itself, or -1
};

// Pointers, strides, and that no written one overlaps itself or another.
lattice_status check_heads(lattice_dense *D, const char *what, const Heads *t, int n, int C) {
    const auto bytes = [&](const Heads &x) {
        return extent(x.rows, x.heads, C, x.row, x.head) * (x.type == LATTICE_BF16 ? 2 : 4);
    };
    for (int i = 0; i < n; ++i) {
        if (t[i].rows <= 0 || t[i].heads <= 0) continue;
        if (!t[i].p || !strides_ok(t[i].rows, t[i].heads, t[i].row, t[i].head)) {
            set_err(D, "%s: %s is missing or has a bad stride", what, t[i].name);
            return LATTICE_E_ARG;
        }
        if (!t[i].written) continue;
        if (!apart(t[i].rows, t[i].heads, C, t[i].row, t[i].head)) {
            set_err(D, "%s: rows of %s overlap", what, t[i].name);
            return LATTICE_E_ARG;
        }
        for (int j = 0; j < n; ++j) {
            if (j == i || t[j].rows <= 0 || t[j].heads <= 0 || !overlap(t[i].p, bytes(t[i]), t[j].p, bytes(t[j]))) continue;
            if (t[i].may_be == j && t[i].p == t[j].p && t[i].row == t[j].row && t[i].head == t[j].head) continue;
            // heads of one buffer, next to each other, share rows but no values
            if (t[i].row == t[j].row && t[i].row > 0 && t[i].type == t[j].type && t[i].may_be != j) {
                const int64_t e = t[i].type == LATTICE_BF16 ? 2 : 4;
                const int64_t gap = static_cast<const char *>(t[j].p) - static_cast<const char *>(t[i].p);
                const int64_t wi = (t[i].heads - 1) * t[i].head + C, wj = (t[j].heads - 1) * t[j].head + C;
                if (gap % e == 0) {
                    const int64_t in_row = ((gap / e) % t[i].row + t[i].row) % t[i].row;
                    if (in_row >= wi && in_row + wj <= t[i].row) continue;
                }
            }
            set_err(D, "%s: %s overlaps %s", what, t[i].name, t[j].name);
            return LATTICE_E_ARG;
        }
    }
    return LATTICE_OK;
}

lattice_status check_attention(lattice_dense *D, const AttendArgs &a, lattice_dtype dtype, const char *what) {
    if (a.q_rows < 0 || a.kv_rows < 0 || a.q_rows > LATTICE_ATTENTION_MAX_ROWS || a.kv_rows > LATTICE_ATTENTION_MAX_ROWS ||
        a.heads < 1 || a.kv_heads < 1 || a.heads > LATTICE_ATTENTION_MAX_HEADS || a.heads % a.kv_heads != 0 || a.D < 1 ||
        a.D > LATTICE_ATTENTION_MAX_CHANNELS) {
        set_err(D, "%s: rows = %lld and %lld, heads = %d and %d or D = %d out of range", what, (long long)a.q_rows,
                (long long)a.kv_rows, a.heads, a.kv_heads, a.D);
        return LATTICE_E_ARG;
    }
    if (!is_storage(dtype) || !(a.scale > 0.f) || !(a.scale <= 1e30f) || a.sequences < 0 ||
        a.sequences > LATTICE_ATTENTION_MAX_SEQUENCES) {
        set_err(D, "%s: bad type, scale or number of sequences (%lld)", what, (long long)a.sequences);
        return LATTICE_E_ARG;
    }
    if (!a.q_starts && (a.kv_starts || a.sequences != 1)) {
        set_err(D, "%s: without q_starts there is one sequence and no kv_starts", what);
        return LATTICE_E_ARG;
    }
    return LATTICE_OK;
}

}  // namespace

extern "C" {

lattice_status lattice_dense_create(void *stream, lattice_dense **out) {
    if (!out) return LATTICE_E_ARG;
    *out = nullptr;
    lattice_dense *D = new (std::nothrow) lattice_dense();
    if (!D) return LATTICE_E_NOMEM;
    D->stream = reinterpret_cast<hipStream_t>(stream);
    if (hipGetDevice(&D->device) != hipSuccess) {
        (void)hipGetLastError();
        delete D;
        return LATTICE_E_HIP;
    }
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, D->device) == hipSuccess && cus > 0)
        D->cu_count = cus;
    const bool ok = hipMalloc(&D->status, sizeof(int32_t)) == hipSuccess &&
                    hipMemsetAsync(D->status, 0, sizeof(int32_t), D->stream) == hipSuccess &&
                    hipHostMalloc(&D->host_status, sizeof(int32_t), hipHostMallocDefault) == hipSuccess;
    if (!ok) {
        (void)hipGetLastError();
        (void)hipFree(D->status);
        delete D;
        return LATTICE_E_NOMEM;
    }
    *out = D;
    return LATTICE_OK;
}

void lattice_dense_destroy(lattice_dense *D) {
    if (!D) return;
    {
        const OnDevice on(D);
        (void)hipStreamSynchronize(D->stream);
        (void)hipFree(D->ws);
        while (D->kept) {
            KeptScratch *k = D->kept;
            D->kept = k->next;
            (void)hipFree(k->p);
            delete k;
        }
        (void)hipFree(D->status);
        (void)hipHostFree(D->host_status);
    }
    delete D;
}

const char *lattice_dense_last_error(const lattice_dense *D) { return D ? D->err : "null handle"; }

lattice_status lattice_dense_get_status(lattice_dense *D) {
    if (!D) return LATTICE_E_ARG;
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "get_status");
    hipError_t e = hipMemcpyAsync(D->host_status, D->status, sizeof(int32_t), hipMemcpyDeviceToHost, D->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(D->stream);
    if (e != hipSuccess) return hip_fail(D, e, "get_status");
    if (*D->host_status == 0) return LATTICE_OK;
    e = hipMemsetAsync(D->status, 0, sizeof(int32_t), D->stream);
    if (e != hipSuccess) return hip_fail(D, e, "get_status");
    if (*D->host_status & DENSE_ST_STARTS)
        set_err(D, "attention: starts that go back or lie outside the rows, or a length outside its sequence (clamped)");
    else
        set_err(D, "linear_cross_entropy: a label is neither a class nor ignore_index (its row counted as one without)");
    return LATTICE_E_RANGE;
}

lattice_status lattice_dense_set_gradient_bits(lattice_dense *D, int bits) {
    if (!D) return LATTICE_E_ARG;
    if (bits != 8 && bits != 16) {
        set_err(D, "set_gradient_bits: bits = %d is neither 8 nor 16", bits);
        return LATTICE_E_ARG;
    }
    D->split_gradients = bits == 16;
    return LATTICE_OK;
}

lattice_status lattice_layer_norm(lattice_dense *D, const lattice *rows_of, const void *x, lattice_dtype x_dtype,
                                  int64_t x_stride, int64_t rows, int C, const float *gamma, const float *beta,
                                  float eps, void *y, lattice_dtype y_dtype, int64_t y_stride, float *mean,
                                  float *rstd) {
    if (!D) return LATTICE_E_ARG;
    const lattice_status s = check_rows(D, rows_of, rows, C, "layer_norm");
    if (s) return s;
    if (!is_storage(x_dtype) || !is_storage(y_dtype) || x_stride < C || y_stride < C || x_stride > kMaxStride ||
        y_stride > kMaxStride || !(eps >= 0.f) || !isfinite(eps) || (rows > 0 && (!x || !y))) {
        set_err(D, "layer_norm: bad pointer, type, stride or eps (C = %d, strides %lld and %lld)", C,
                (long long)x_stride, (long long)y_stride);
        return LATTICE_E_ARG;
    }
    const bool in_place = x == y && x_dtype == y_dtype && x_stride == y_stride;
    if (!in_place && overlap(x, span(rows, C, x_stride, x_dtype), y, span(rows, C, y_stride, y_dtype))) {
        set_err(D, "layer_norm: y overlaps x (it may be x itself)");
        return LATTICE_E_ARG;
    }
    if (rows == 0) return LATTICE_OK;
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "layer_norm");
    NormArgs a = {rows_of ? rows_of->counters : nullptr, rows, C, eps, x, x_stride, x_dtype == LATTICE_BF16, gamma,
                  beta, y, y_stride, y_dtype == LATTICE_BF16, mean, rstd};
    const hipError_t e = launch_layer_norm(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "layer_norm");
}

lattice_status lattice_layer_norm_backward(lattice_dense *D, const lattice *rows_of, const void *grad_y,
                                           lattice_dtype g_dtype, int64_t g_stride, const void *x,
                                           lattice_dtype x_dtype, int64_t x_stride, int64_t rows, int C,
                                           const float *mean, const float *rstd, const float *gamma, void *grad_x,
                                           int64_t grad_x_stride, float *grad_gamma, float *grad_beta) {
    if (!D) return LATTICE_E_ARG;
    lattice_status s = check_rows(D, rows_of, rows, C, "layer_norm_backward");
    if (s) return s;
    if (!is_storage(x_dtype) || !is_storage(g_dtype) || x_stride < C || g_stride < C || x_stride > kMaxStride ||
        g_stride > kMaxStride || (grad_x && (grad_x_stride < C || grad_x_stride > kMaxStride)) ||
        (rows > 0 && (!grad_y || !x || !mean || !rstd || (!grad_x && !grad_gamma && !grad_beta)))) {
        set_err(D, "layer_norm_backward: bad pointer, type or stride (C = %d)", C);
        return LATTICE_E_ARG;
    }
    if (rows == 0 && !grad_gamma && !grad_beta) return LATTICE_OK;  // a grad_x without rows may have no address
    const int64_t nx = span(rows, C, x_stride, x_dtype), ng = span(rows, C, g_stride, g_dtype);
    const int64_t no = grad_x ? span(rows, C, grad_x_stride, x_dtype) : 0;
    const bool on_x = grad_x == x && grad_x_stride == x_stride;
    const bool on_g = grad_x == grad_y && grad_x_stride == g_stride && g_dtype == x_dtype;
    // long rows are read again after grad_x has been written
    const bool again = (grad_gamma || grad_beta) && C > kMaxChannels / 128;
    if ((overlap(grad_x, no, x, nx) && (!on_x || again)) || (overlap(grad_x, no, grad_y, ng) && (!on_g || again))) {
        set_err(D, "layer_norm_backward: grad_x overlaps x or grad_y");
        return LATTICE_E_ARG;
    }
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "layer_norm_backward");
    NormBackwardArgs a = {rows_of ? rows_of->counters : nullptr, rows, C, grad_y, g_stride, g_dtype == LATTICE_BF16, x,
                          x_stride, x_dtype == LATTICE_BF16, mean, rstd, gamma, grad_x, grad_x_stride, grad_gamma,
                          grad_beta};
    if ((s = grow(D, layer_norm_backward_scratch(D, a), "layer_norm_backward"))) return s;
    const hipError_t e = launch_layer_norm_backward(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "layer_norm_backward");
}

lattice_status lattice_linear_cross_entropy(lattice_dense *D, lattice_dtype dtype, const void *x, int64_t x_stride,
                                            int64_t N, int C, const void *w, int64_t w_stride, int K,
                                            const float *bias, const int64_t *target, int64_t ignore_index, int mean,
                                            float *loss, float *row_loss, void *grad_x, void *grad_w,
                                            float *grad_bias) {
    if (!D) return LATTICE_E_ARG;
    if (N < 0 || N > LATTICE_LOSS_MAX_ROWS || C < 1 || C > LATTICE_LOSS_MAX_CHANNELS || K < 1 ||
        K > LATTICE_LOSS_MAX_CLASSES) {
        set_err(D, "linear_cross_entropy: N = %lld, C = %d or K = %d out of range", (long long)N, C, K);
        return LATTICE_E_ARG;
    }
    if (!is_storage(dtype) || x_stride < C || w_stride < C || x_stride > kMaxStride || w_stride > kMaxStride || !w ||
        !loss || (N > 0 && (!x || !target))) {
        set_err(D, "linear_cross_entropy: bad pointer, type or stride (C = %d, strides %lld and %lld)", C,
                (long long)x_stride, (long long)w_stride);
        return LATTICE_E_ARG;
    }
    const int64_t e = dtype == LATTICE_BF16 ? 2 : 4;
    const int64_t nx = span(N, C, x_stride, dtype), nw = span(K, C, w_stride, dtype);
    if (overlap(grad_x, N * C * e, x, nx) || overlap(grad_x, N * C * e, w, nw) ||
        overlap(grad_w, (int64_t)K * C * e, x, nx) || overlap(grad_w, (int64_t)K * C * e, w, nw)) {
        set_err(D, "linear_cross_entropy: a gradient overlaps x or w");
        return LATTICE_E_ARG;
    }
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "linear_cross_entropy");
    LossArgs a = {dtype == LATTICE_BF16, N, C, x, x_stride, w, K, w_stride, bias, target, ignore_index, mean != 0, loss,
                  row_loss, grad_x, grad_w, grad_bias, D->split_gradients};
    const lattice_status s = grow(D, loss_scratch(D, a), "linear_cross_entropy");
    if (s) return s;
    const hipError_t err = launch_loss(D, a);
    return err == hipSuccess ? LATTICE_OK : hip_fail(D, err, "linear_cross_entropy");
}

lattice_status lattice_orthogonalize(lattice_dense *D, const void *g, lattice_dtype g_dtype, int64_t batch, int m,
                                     int n, int64_t batch_stride, int64_t row_stride, int steps,
                                     const float *coefficients, float eps, void *out, lattice_dtype out_dtype) {
    if (!D) return LATTICE_E_ARG;
    if (batch < 0 || batch > LATTICE_UPDATE_MAX_BATCH || m < 1 || n < 1 || m > LATTICE_UPDATE_MAX_SIDE ||
        n > LATTICE_UPDATE_MAX_SIDE || steps < 0 || steps > 64) {
        set_err(D, "orthogonalize: batch = %lld, m = %d, n = %d or steps = %d out of range", (long long)batch, m, n,
                steps);
        return LATTICE_E_ARG;
    }
    if (!is_storage(g_dtype) || !is_storage(out_dtype) || !coefficients || !(eps >= 0.f) || !isfinite(eps) ||
        row_stride < n || row_stride > kMaxStride || batch_stride < 0 || (batch > 0 && (!g || !out))) {
        set_err(D, "orthogonalize: bad pointer, type, stride, coefficients or eps (m = %d, n = %d)", m, n);
        return LATTICE_E_ARG;
    }
    for (int i = 0; i < 3; ++i)
        if (!isfinite(coefficients[i])) {
            set_err(D, "orthogonalize: a coefficient is not finite");
            return LATTICE_E_ARG;
        }
    const int64_t ng = batch > 0 ? (batch - 1) * batch_stride * (g_dtype == LATTICE_BF16 ? 2 : 4) +
                                       span(m, n, row_stride, g_dtype)
                                 : 0;
    if (overlap(g, ng, out, batch * m * n * (out_dtype == LATTICE_BF16 ? 2 : 4))) {
        set_err(D, "orthogonalize: out overlaps g");
        return LATTICE_E_ARG;
    }
    if (batch == 0) return LATTICE_OK;
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "orthogonalize");
    UpdateArgs a = {g, g_dtype == LATTICE_BF16, batch, m, n, batch_stride, row_stride, steps,
                    {coefficients[0], coefficients[1], coefficients[2]}, eps, out, out_dtype == LATTICE_BF16};
    const lattice_status s = grow(D, update_scratch(D, a), "orthogonalize");
    if (s) return s;
    const hipError_t e = launch_update(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "orthogonalize");
}

lattice_status lattice_attention(lattice_dense *D, lattice_dtype dtype, int64_t q_rows, int64_t kv_rows, int heads,
                                 int kv_heads, int C, const void *q, int64_t q_row, int64_t q_head, const void *k,
                                 int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                                 const int32_t *q_starts, const int32_t *kv_starts, const int32_t *kv_lengths,
                                 int64_t sequences, int causal, float scale, int zero_rest, void *out, int64_t out_row,
                                 int64_t out_head, float *lse) {
    if (!D) return LATTICE_E_ARG;
    AttendArgs a = {};
    a.bf16 = dtype == LATTICE_BF16;
    a.q_rows = q_rows;
    a.kv_rows = kv_rows;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.D = C;
    a.q = q, a.q_row = q_row, a.q_head = q_head;
    a.k = k, a.k_row = k_row, a.k_head = k_head;
    a.v = v, a.v_row = v_row, a.v_head = v_head;
    a.q_starts = q_starts;
    a.kv_starts = kv_starts;
    a.kv_lengths = kv_lengths;
    a.sequences = sequences;
    a.causal = causal != 0;
    a.scale = scale;
    a.zero_rest = zero_rest != 0;
    a.out = out, a.o_row = out_row, a.o_head = out_head;
    a.lse = lse;
    lattice_status s = check_attention(D, a, dtype, "attention");
    if (s) return s;
    const Heads t[] = {{"q", q, q_rows, heads, q_row, q_head, dtype, false, -1},
                       {"k", k, q_rows > 0 ? kv_rows : 0, kv_heads, k_row, k_head, dtype, false, -1},
                       {"v", v, q_rows > 0 ? kv_rows : 0, kv_heads, v_row, v_head, dtype, false, -1},
                       {"out", out, q_rows, heads, out_row, out_head, dtype, true, -1}};
    if ((s = check_heads(D, "attention", t, 4, C))) return s;
    if (q_rows == 0) return LATTICE_OK;
    if (!attention_fits(D, a)) {
        set_err(D, "attention: more tiles than a launch takes");
        return LATTICE_E_ARG;
    }
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "attention");
    if ((s = grow(D, attention_scratch(D, a), "attention"))) return s;
    const hipError_t e = launch_attention(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "attention");
}

lattice_status lattice_attention_backward(lattice_dense *D, lattice_dtype dtype, int64_t q_rows, int64_t kv_rows,
                                          int heads, int kv_heads, int C, const void *grad_out, int64_t grad_row,
                                          int64_t grad_head, const void *q, int64_t q_row, int64_t q_head,
                                          const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                          int64_t v_head, const void *out, int64_t out_row, int64_t out_head,
                                          const float *lse, const int32_t *q_starts, const int32_t *kv_starts,
                                          const int32_t *kv_lengths, int64_t sequences, int causal, float scale,
                                          int zero_rest, void *grad_q, void *grad_k, void *grad_v) {
    if (!D) return LATTICE_E_ARG;
    AttendArgs a = {};
    a.bf16 = dtype == LATTICE_BF16;
    a.q_rows = q_rows;
    a.kv_rows = kv_rows;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.D = C;
    a.grad = grad_out, a.g_row = grad_row, a.g_head = grad_head;
    a.q = q, a.q_row = q_row, a.q_head = q_head;
    a.k = k, a.k_row = k_row, a.k_head = k_head;
    a.v = v, a.v_row = v_row, a.v_head = v_head;
    a.out = const_cast<void *>(out), a.o_row = out_row, a.o_head = out_head;
    a.lse = const_cast<float *>(lse);
    a.q_starts = q_starts;
    a.kv_starts = kv_starts;
    a.kv_lengths = kv_lengths;
    a.sequences = sequences;
    a.causal = causal != 0;
    a.scale = scale;
    a.zero_rest = zero_rest != 0;
    a.grad_q = grad_q;
    a.grad_k = grad_k;
    a.grad_v = grad_v;
    lattice_status s = check_attention(D, a, dtype, "attention_backward");
    if (s) return s;
    const int64_t qw = (int64_t)heads * C, kw = (int64_t)kv_heads * C;
    const Heads t[] = {{"q", q, q_rows, heads, q_row, q_head, dtype, false, -1},
                       {"k", k, kv_rows, kv_heads, k_row, k_head, dtype, false, -1},
                       {"v", v, kv_rows, kv_heads, v_row, v_head, dtype, false, -1},
                       {"out", out, q_rows, heads, out_row, out_head, dtype, false, -1},
                       {"grad_out", grad_out, q_rows, heads, grad_row, grad_head, dtype, false, -1},
                       {"grad_q", grad_q, q_rows, heads, qw, C, dtype, true, -1},
                       {"grad_k", grad_k, kv_rows, kv_heads, kw, C, dtype, true, -1},
                       {"grad_v", grad_v, kv_rows, kv_heads, kw, C, dtype, true, -1}};
    if ((s = check_heads(D, "attention_backward", t, 8, C))) return s;
    if (q_rows > 0 && !lse) {
        set_err(D, "attention_backward: lse is missing");
        return LATTICE_E_ARG;
    }
    if (!attention_backward_fits(D, a)) {
        set_err(D, "attention_backward: more tiles than a launch takes");
        return LATTICE_E_ARG;
    }
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "attention_backward");
    if ((s = grow(D, attention_backward_scratch(D, a), "attention_backward"))) return s;
    const hipError_t e = launch_attention_backward(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "attention_backward");
}

static lattice_status check_rotate(lattice_dense *D, const RotateArgs &a, lattice_dtype dtype, const char *what) {
    if (a.rows < 0 || a.rows > LATTICE_ATTENTION_MAX_ROWS || a.heads < 1 || a.kv_heads < 0 ||
        a.heads > LATTICE_ATTENTION_MAX_HEADS || a.kv_heads > LATTICE_ATTENTION_MAX_HEADS || a.D < 1 ||
        a.D > LATTICE_ROTATE_MAX_CHANNELS || a.axes < 1 || a.axes > LATTICE_ROTATE_MAX_AXES) {
        set_err(D, "%s: rows = %lld, heads = %d and %d, C = %d or axes = %d out of range", what, (long long)a.rows, a.heads,
                a.kv_heads, a.D, a.axes);
        return LATTICE_E_ARG;
    }
    int64_t pairs = 0;
    bool ok = a.sections != nullptr;
    for (int i = 0; ok && i < a.axes; ++i) {
        ok = a.sections[i] >= 0 && a.sections[i] <= a.D;
        pairs += a.sections[i];
    }
    if (!ok || 2 * pairs > a.D) {
        set_err(D, "%s: the sections are missing or hold more than %d pairs", what, a.D / 2);
        return LATTICE_E_ARG;
    }
    if (!is_storage(dtype) || !(a.eps >= 0.f) || !isfinite(a.eps) || (pairs > 0 && !a.freq) || (a.rows > 0 && !a.pos) ||
        a.pos_stride < 0 || a.pos_stride > kMaxStride) {
        set_err(D, "%s: bad type, eps, frequencies or positions", what);
        return LATTICE_E_ARG;
    }
    if (!a.norm && (a.gain_q || a.gain_k || a.grad_gain_q || a.grad_gain_k)) {
        set_err(D, "%s: gains without the norm", what);
        return LATTICE_E_ARG;
    }
    return LATTICE_OK;
}

lattice_status lattice_rotate_heads(lattice_dense *D, lattice_dtype dtype, int64_t rows, int heads, int kv_heads, int C,
                                    const void *q, int64_t q_row, int64_t q_head, const void *k, int64_t k_row,
                                    int64_t k_head, const void *positions, int integers, int64_t position_stride,
                                    int axes, const int *sections, const float *freq, int norm, const float *gain_q,
                                    const float *gain_k, float eps, int interleaved, void *out_q, int64_t out_q_row,
                                    int64_t out_q_head, void *out_k, int64_t out_k_row, int64_t out_k_head) {
    if (!D) return LATTICE_E_ARG;
    RotateArgs a = {};
    a.bf16 = dtype == LATTICE_BF16;
    a.rows = rows;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.D = C;
    a.q = q, a.q_row = q_row, a.q_head = q_head;
    a.k = k, a.k_row = k_row, a.k_head = k_head;
    a.pos = positions;
    a.integers = integers != 0;
    a.pos_stride = position_stride;
    a.axes = axes;
    a.sections = sections;
    a.freq = freq;
    a.norm = norm != 0;
    a.gain_q = gain_q;
    a.gain_k = gain_k;
    a.eps = eps;
    a.interleaved = interleaved != 0;
    a.out_q = out_q, a.oq_row = out_q_row, a.oq_head = out_q_head;
    a.out_k = out_k, a.ok_row = out_k_row, a.ok_head = out_k_head;
    lattice_status s = check_rotate(D, a, dtype, "rotate_heads");
    if (s) return s;
    const Heads t[] = {{"q", q, rows, heads, q_row, q_head, dtype, false, -1},
                       {"k", k, rows, kv_heads, k_row, k_head, dtype, false, -1},
                       {"out_q", out_q, rows, heads, out_q_row, out_q_head, dtype, true, 0},
                       {"out_k", out_k, rows, kv_heads, out_k_row, out_k_head, dtype, true, 1}};
    if ((s = check_heads(D, "rotate_heads", t, 4, C))) return s;
    if (rows == 0) return LATTICE_OK;
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "rotate_heads");
    const hipError_t e = launch_rotate(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "rotate_heads");
}

lattice_status lattice_rotate_heads_backward(lattice_dense *D, lattice_dtype dtype, int64_t rows, int heads,
                                             int kv_heads, int C, const void *grad_out_q, int64_t grad_out_q_row,
                                             int64_t grad_out_q_head, const void *grad_out_k, int64_t grad_out_k_row,
                                             int64_t grad_out_k_head, const void *q, int64_t q_row, int64_t q_head,
                                             const void *k, int64_t k_row, int64_t k_head, const void *positions,
                                             int integers, int64_t position_stride, int axes, const int *sections,
                                             const float *freq, int norm, const float *gain_q, const float *gain_k,
                                             float eps, int interleaved, void *grad_q, int64_t grad_q_row,
                                             int64_t grad_q_head, void *grad_k, int64_t grad_k_row, int64_t grad_k_head,
                                             float *grad_gain_q, float *grad_gain_k) {
    if (!D) return LATTICE_E_ARG;
    RotateArgs a = {};
    a.bf16 = dtype == LATTICE_BF16;
    a.rows = rows;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.D = C;
    a.grad_q = grad_out_q, a.gq_row = grad_out_q_row, a.gq_head = grad_out_q_head;
    a.grad_k = grad_out_k, a.gk_row = grad_out_k_row, a.gk_head = grad_out_k_head;
    a.q = q, a.q_row = q_row, a.q_head = q_head;
    a.k = k, a.k_row = k_row, a.k_head = k_head;
    a.pos = positions;
    a.integers = integers != 0;
    a.pos_stride = position_stride;
    a.axes = axes;
    a.sections = sections;
    a.freq = freq;
    a.norm = norm != 0;
    a.gain_q = gain_q;
    a.gain_k = gain_k;
    a.eps = eps;
    a.interleaved = interleaved != 0;
    a.out_q = grad_q, a.oq_row = grad_q_row, a.oq_head = grad_q_head;
    a.out_k = grad_k, a.ok_row = grad_k_row, a.ok_head = grad_k_head;
    a.grad_gain_q = grad_gain_q;
    a.grad_gain_k = grad_gain_k;
    lattice_status s = check_rotate(D, a, dtype, "rotate_heads_backward");
    if (s) return s;
    if (grad_gain_k && kv_heads == 0) {
        set_err(D, "rotate_heads_backward: grad_gain_k without keys");
        return LATTICE_E_ARG;
    }
    const Heads t[] = {{"q", q, rows, heads, q_row, q_head, dtype, false, -1},
                       {"k", k, rows, kv_heads, k_row, k_head, dtype, false, -1},
                       {"grad_out_q", grad_out_q, rows, heads, grad_out_q_row, grad_out_q_head, dtype, false, -1},
                       {"grad_out_k", grad_out_k, rows, kv_heads, grad_out_k_row, grad_out_k_head, dtype, false, -1},
                       {"grad_q", grad_q, rows, heads, grad_q_row, grad_q_head, dtype, true, 2},
                       {"grad_k", grad_k, rows, kv_heads, grad_k_row, grad_k_head, dtype, true, 3}};
    if ((s = check_heads(D, "rotate_heads_backward", t, 6, C))) return s;
    if (rows == 0 && !grad_gain_q && !grad_gain_k) return LATTICE_OK;
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "rotate_heads_backward");
    if ((s = grow(D, rotate_backward_scratch(D, a), "rotate_heads_backward"))) return s;
    const hipError_t e = launch_rotate_backward(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "rotate_heads_backward");
}

lattice_status lattice_clip_gradients(lattice_dense *D, int count, const void *const *in, const lattice_dtype *in_dtype,
                                      void *const *out, const lattice_dtype *out_dtype, const int64_t *values,
                                      float max_norm, float eps, float *norm) {
    if (!D) return LATTICE_E_ARG;
    if (count < 0 || count > LATTICE_CLIP_MAX_TENSORS || (count > 0 && (!in || !in_dtype || !out || !out_dtype || !values)) ||
        !(max_norm >= 0.f) || !(eps >= 0.f) || !isfinite(eps) || !norm) {
        set_err(D, "clip_gradients: bad number of tensors (%d), pointer, max_norm or eps", count);
        return LATTICE_E_ARG;
    }
    for (int i = 0; i < count; ++i)
        if (values[i] < 0 || values[i] > ((int64_t)1 << 40) || !is_storage(in_dtype[i]) || !is_storage(out_dtype[i]) ||
            (values[i] > 0 && (!in[i] || !out[i]))) {
            set_err(D, "clip_gradients: tensor %d has a bad pointer, type or number of values", i);
            return LATTICE_E_ARG;
        }
    // An output may be its own input; otherwise none may touch another output or input.
    struct Range {
        uintptr_t lo, hi;
        int tensor;
    };
    Range *ranges = new (std::nothrow) Range[(size_t)count + 1];
    if (!ranges) {
        set_err(D, "clip_gradients: out of host memory");
        return LATTICE_E_NOMEM;
    }
    const auto bytes = [](int64_t n, lattice_dtype t) { return (uintptr_t)n * (t == LATTICE_BF16 ? 2 : 4); };
    int n = 0, bad = -1;
    for (int i = 0; i < count; ++i) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(out[i]);
        if (values[i] > 0) ranges[n++] = {lo, lo + bytes(values[i], out_dtype[i]), i};
    }
    std::sort(ranges, ranges + n, [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (int i = 1; i < n && bad < 0; ++i)
        if (ranges[i].lo < ranges[i - 1].hi) bad = ranges[i].tensor;
    for (int i = 0; i < count && bad < 0; ++i) {
        if (values[i] <= 0) continue;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(in[i]), hi = lo + bytes(values[i], in_dtype[i]);
        const Range *r = std::upper_bound(ranges, ranges + n, lo, [](uintptr_t x, const Range &a) { return x < a.hi; });
        for (; r < ranges + n && r->lo < hi && bad < 0; ++r)
            if (r->tensor != i || r->lo != lo || in_dtype[i] != out_dtype[i]) bad = i;
    }
    delete[] ranges;
    if (bad >= 0) {
        set_err(D, "clip_gradients: an output overlaps another one or an input that is not its own (tensor %d)", bad);
        return LATTICE_E_ARG;
    }
    const OnDevice on(D);
    if (on.error != hipSuccess) return hip_fail(D, on.error, "clip_gradients");
    ClipArgs a = {count, in, out, values, in_dtype, out_dtype, max_norm, eps, norm};
    const lattice_status s = grow(D, clip_scratch(D, a), "clip_gradients");
    if (s) return s;
    const hipError_t e = launch_clip(D, a);
    return e == hipSuccess ? LATTICE_OK : hip_fail(D, e, "clip_gradients");
}

}  // extern "C"
