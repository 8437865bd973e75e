// Host side of the dense operators declared in include/lattice.h: argument
// checking, the handle with its scratch and device status, and dispatch to the
// kernels of norm.hip, loss.hip and update.hip.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

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

}  // extern "C"
