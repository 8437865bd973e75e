// The dense operators' host side without a GPU: this program is linked with
// the library and defines the HIP calls that it makes, so that what a call
// allocates, frees and launches, with which arguments and on which device, can
// be looked at.  No kernel runs, and no address that hipMalloc gives is read or
// written: they only stand for device memory.
//
//   host_driver CHECK      prints "ok", or what is wrong and exits with 1
#include <cxxabi.h>
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>
#include <utility>
#include <vector>

#include "lattice.h"

namespace {

[[noreturn]] void fail(const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vprintf(fmt, ap);
    va_end(ap);
    std::printf("\n");
    std::exit(1);
}

struct Launch {
    std::string name;
    dim3 grid;
    int device;
    void **args;
};

int device = 0;                           // current
hipError_t last = hipSuccess;
std::map<uintptr_t, size_t> blocks;       // live, by address
uintptr_t next_address = (uintptr_t)1 << 44;
int64_t launches = 0;
int want_device = -1;                     // on which all work has to be, or any
hipStream_t want_stream = nullptr;        // likewise
void (*on_launch)(const Launch &) = nullptr;
dim3 pushed_grid, pushed_block;
size_t pushed_lds;
hipStream_t pushed_stream;
bool capturing = false;
hipStreamCaptureMode capture_mode = hipStreamCaptureModeGlobal;   // of this thread

void here(const char *what) {
    if (want_device >= 0 && device != want_device) fail("%s on device %d, not %d", what, device, want_device);
}

void on(const char *what, hipStream_t s) {
    if (want_stream && s != want_stream) fail("%s on another stream than the handle's", what);
}

std::map<const void *, std::string> &names() {
    static std::map<const void *, std::string> all;   // filled before main
    return all;
}

// The live block that holds [p, p + bytes), or 0.
uintptr_t block_of(const void *p, int64_t bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    auto it = blocks.upper_bound(a);
    if (it == blocks.begin()) return 0;
    --it;
    return bytes >= 0 && a + (uintptr_t)bytes <= it->first + it->second ? it->first : 0;
}

}  // namespace

extern "C" {

void **__hipRegisterFatBinary(const void *) {
    static void *module;
    return &module;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *,
                           int *) {
    names()[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    pushed_grid = grid;
    pushed_block = block;
    pushed_lds = lds;
    pushed_stream = stream;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
    *grid = pushed_grid;
    *block = pushed_block;
    *lds = pushed_lds;
    *stream = pushed_stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t stream) {
    if (!grid.x || !grid.y || !grid.z || !block.x || !block.y || !block.z || block.x * block.y * block.z > 1024 ||
        lds > 160 * 1024)
        return last = hipErrorInvalidConfiguration;
    here("a launch");
    on("a launch", stream);
    ++launches;
    if (on_launch) on_launch({names()[fn], grid, device, args});
    return hipSuccess;
}
hipError_t hipGetLastError(void) {
    const hipError_t e = last;
    last = hipSuccess;
    return e;
}
const char *hipGetErrorString(hipError_t e) { return e == hipSuccess ? "no error" : "an error"; }
hipError_t hipGetDevice(int *d) {
    *d = device;
    return hipSuccess;
}
hipError_t hipSetDevice(int d) {
    device = d;
    return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) {
    *v = 256;
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) {
    *p = reinterpret_cast<void *>(next_address);
    blocks[next_address] = n;
    next_address += (n + 8191) / 4096 * 4096;   // a gap after each
    here("an allocation");
    if (capturing && capture_mode != hipStreamCaptureModeRelaxed) fail("hipMalloc breaks off a capture");
    return hipSuccess;
}
hipError_t hipFree(void *p) {
    here("hipFree");
    if (capturing) fail("hipFree waits for the device during a capture");
    if (p && !blocks.erase(reinterpret_cast<uintptr_t>(p))) fail("hipFree of %p, which is no block", p);
    return hipSuccess;
}
hipError_t hipHostMalloc(void **p, size_t n, unsigned) {
    *p = std::calloc(1, n);
    return hipSuccess;
}
hipError_t hipHostFree(void *p) {
    std::free(p);
    return hipSuccess;
}
hipError_t hipMemset(void *, int, size_t) {
    here("hipMemset");
    on("hipMemset", nullptr);
    return hipSuccess;
}
hipError_t hipMemsetAsync(void *, int, size_t, hipStream_t stream) {
    here("hipMemsetAsync");
    on("hipMemsetAsync", stream);
    return hipSuccess;
}
hipError_t hipMemcpyAsync(void *to, const void *, size_t n, hipMemcpyKind, hipStream_t stream) {
    here("a copy");
    on("a copy", stream);
    std::memset(to, 0, n);
    return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) {
    here("hipStreamSynchronize");
    return hipSuccess;
}
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode *mode) {
    std::swap(*mode, capture_mode);
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) {
    *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}

}  // extern "C"

namespace {

template <class T>
T *buffer(int64_t values) {
    void *p = nullptr;
    (void)hipMalloc(&p, values > 0 ? (size_t)values * sizeof(T) : 1);
    return static_cast<T *>(p);
}

lattice_dense *handle(void *stream = nullptr) {
    lattice_dense *D = nullptr;
    if (lattice_dense_create(stream, &D) != LATTICE_OK) fail("lattice_dense_create failed");
    return D;
}

void expect(const char *what, lattice_dense *D, lattice_status got, lattice_status want) {
    if (got != want) fail("%s: status %d, not %d (%s)", what, (int)got, (int)want, lattice_dense_last_error(D));
}

// -- rowsum ------------------------------------------------------------------

struct RowsumJobs {   // the kernel's first argument
    struct {
        const float *part;
        float *out;
        int64_t rows, n;
    } j[4];
    int64_t first[5];
};

// Every sum over partial rows reads and writes inside blocks that are there.
void look_at_rowsum(const Launch &l) {
    if (l.name.find("k_rowsum") == std::string::npos) return;
    const RowsumJobs &jobs = *static_cast<const RowsumJobs *>(l.args[0]);
    const int count = *static_cast<const int *>(l.args[1]);
    for (int i = 0; i < count; ++i) {
        const auto &j = jobs.j[i];
        if (j.rows > 0 && !block_of(j.part, j.rows * j.n * 4))
            fail("a sum reads %lld rows of %lld from %p, outside every block", (long long)j.rows, (long long)j.n,
                 (const void *)j.part);
        if (!block_of(j.out, (int64_t)l.grid.y * j.n * 4)) fail("a sum writes to %p, outside every block", (void *)j.out);
    }
}

// The bias gradient of more pieces of rows than one sum adds up: kept logits
// (fp32, 192 channels) of the most classes come in pieces of 256 rows.
void many_pieces() {
    on_launch = look_at_rowsum;
    const int64_t N = (int64_t)256 * 8193 - 100;
    const int C = 192, K = LATTICE_LOSS_MAX_CLASSES;
    const float *x = buffer<float>(N * C), *w = buffer<float>((int64_t)K * C), *bias = buffer<float>(K);
    const int64_t *target = buffer<int64_t>(N);
    float *loss = buffer<float>(1), *grad_bias = buffer<float>(K);
    lattice_dense *D = handle();
    expect("linear_cross_entropy", D,
           lattice_linear_cross_entropy(D, LATTICE_F32, x, C, N, C, w, C, K, bias, target, -100, 1, loss, nullptr, nullptr,
                                        nullptr, grad_bias),
           LATTICE_OK);
    lattice_dense_destroy(D);
}

// -- products ----------------------------------------------------------------

// The arguments of k_gemm<Tile<BM, BN, WM, WN, BK, P, STAGES>, ..>.
struct Operand {
    const uint16_t *p;
    int64_t ld, plane, batch;
    int rows;
};
struct Shape {
    int K, k_split, tiles_m, tiles_n;
    bool lower;
};

std::string demangled(const std::string &name) {
    int status = 0;
    char *d = abi::__cxa_demangle(name.c_str(), nullptr, nullptr, &status);
    std::string s = d ? d : name;
    std::free(d);
    return s;
}

// What a product's direct loads read of an operand: 16-byte pieces of all its
// rows and planes, for every matrix of a batch, up to the contraction's end.
void look_at_products(const Launch &l) {
    look_at_rowsum(l);
    if (l.name.find("6k_gemmI") == std::string::npos) return;
    static std::map<std::string, int> planes_of;
    auto it = planes_of.find(l.name);
    if (it == planes_of.end()) {
        const std::string s = demangled(l.name);
        int t[7];
        const size_t at = s.find("Tile<");
        if (at == std::string::npos || std::sscanf(s.c_str() + at, "Tile<%d, %d, %d, %d, %d, %d, %d", t, t + 1, t + 2, t + 3,
                                                   t + 4, t + 5, t + 6) != 7)
            fail("a product without a tile: %s", s.c_str());
        it = planes_of.emplace(l.name, t[5]).first;
    }
    const Shape &s = *static_cast<const Shape *>(l.args[2]);
    if (s.K < 64 || s.K % 64 || s.k_split < 64 || s.k_split % 64 || (int64_t)(l.grid.y - 1) * s.k_split >= s.K)
        fail("a contraction of %d in %u parts of %d", s.K, l.grid.y, s.k_split);
    for (int i = 0; i < 2; ++i) {
        const Operand &o = *static_cast<const Operand *>(l.args[i]);
        if (o.rows < 1 || o.ld < s.K || o.ld >= (int64_t)1 << 22 || o.ld % 8 || (reinterpret_cast<uintptr_t>(o.p) & 15))
            fail("operand %d: %d rows of %lld at %p over %d", i, o.rows, (long long)o.ld, (const void *)o.p, s.K);
        const int64_t values = (int64_t)(l.grid.z - 1) * o.batch + (it->second - 1) * o.plane + (o.rows - 1) * o.ld + s.K;
        if (!block_of(o.p, values * 2))
            fail("operand %d: %lld values from %p leave their block", i, (long long)values, (const void *)o.p);
    }
}

// Losses and updates of many sizes, most of them odd, up to pieces of rows and
// classes and chunks of a batch.
void products_stay_inside() {
    on_launch = look_at_products;
    std::mt19937 rng(5);
    auto size = [&](double lo, double hi) {
        return (int64_t)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng));
    };
    const float ns[3] = {3.4445f, -4.7750f, 2.0315f};
    for (int i = 0; i < 3000; ++i) {
        const std::map<uintptr_t, size_t> none;
        blocks = none;
        lattice_dense *D = handle();
        const lattice_dtype t = rng() % 2 ? LATTICE_F32 : LATTICE_BF16;
        const int64_t e = t == LATTICE_F32 ? 4 : 2;
        lattice_status got;
        if (rng() % 3) {
            const int64_t N = size(1, rng() % 4 ? 9000 : 1e6);
            const int C = (int)(rng() % 3 ? size(1, 3000) : 64 * (1 + rng() % 32)), K = (int)size(1, rng() % 4 ? 70000 : 1 << 20);
            const int64_t xs = C + (rng() % 2 ? 0 : (rng() % 2 ? 8 : rng() % 9)), ws = C + (rng() % 2 ? 0 : 8);
            const int want = rng() % 8;
            lattice_dense_set_gradient_bits(D, rng() % 2 ? 8 : 16);
            got = lattice_linear_cross_entropy(
                D, t, buffer<char>(((N - 1) * xs + C) * e), xs, N, C, buffer<char>(((K - 1) * ws + C) * e), ws, K,
                rng() % 2 ? buffer<float>(K) : nullptr, buffer<int64_t>(N), -100, 1, buffer<float>(1), buffer<float>(N),
                want & 1 ? buffer<char>(N * C * e) : nullptr, want & 2 ? buffer<char>((int64_t)K * C * e) : nullptr,
                want & 4 ? buffer<float>(K) : nullptr);
        } else {
            const int64_t batch = size(1, 300), m = size(1, 3000), n = size(1, 9000);
            const lattice_dtype o = rng() % 2 ? LATTICE_F32 : LATTICE_BF16;
            got = lattice_orthogonalize(D, buffer<char>(batch * m * n * e), t, batch, (int)m, (int)n, m * n, n, 2, ns, 1e-7f,
                                        buffer<char>(batch * m * n * 4), o);
        }
        expect("a call", D, got, LATTICE_OK);
        lattice_dense_destroy(D);
    }
    if (launches < 20000) fail("only %lld launches", (long long)launches);
}

// -- scratch -----------------------------------------------------------------

// The scratch that a call was captured with outlives every larger call.
void captured_scratch() {
    int stream_of_its_own = 0;
    const float *g = buffer<float>(64 * 4096);
    float *out = buffer<float>(64 * 4096);
    const float ns[3] = {3.4445f, -4.7750f, 2.0315f};
    const size_t callers = blocks.size();
    lattice_dense *D = handle(&stream_of_its_own);
    const size_t without = blocks.size();
    auto update = [&](int n, lattice_status want) {
        expect("orthogonalize", D,
               lattice_orthogonalize(D, g, LATTICE_F32, 1, 64, n, 0, n, 5, ns, 1e-7f, out, LATTICE_F32), want);
    };
    update(128, LATTICE_OK);
    if (blocks.size() != without + 1) fail("no scratch after a call");
    update(256, LATTICE_OK);
    if (blocks.size() != without + 1) fail("scratch that no graph uses was not freed");
    const uintptr_t scratch = blocks.rbegin()->first;
    capturing = true;
    update(256, LATTICE_OK);
    update(512, LATTICE_OK);   // allocates
    const uintptr_t second = blocks.rbegin()->first;
    capturing = false;
    if (capture_mode != hipStreamCaptureModeGlobal) fail("the thread's capture mode was changed");
    for (int n : {1024, 2048, 4096}) update(n, LATTICE_OK);
    if (!blocks.count(scratch) || !blocks.count(second)) fail("the scratch of a captured call was freed by a larger one");
    if (blocks.size() != without + 3) fail("%zu blocks of scratch, not 3", blocks.size() - without);
    lattice_dense_destroy(D);
    if (blocks.size() != callers) fail("%zu blocks left by the handle", blocks.size() - callers);
}

// -- device ------------------------------------------------------------------

// A handle's work is on its device, whichever is current at the call.
void another_current_device() {
    device = 1;
    lattice_dense *D = handle();
    const int64_t rows = 3000;
    const int C = 64, K = 20;
    float *x = buffer<float>(rows * C), *y = buffer<float>(rows * C), *v = buffer<float>(4 * rows), *w = buffer<float>(K * C);
    int64_t *target = buffer<int64_t>(rows);
    const float ns[3] = {1.5f, -0.5f, 0.f};
    auto after = [&](const char *what, lattice_status got) {
        expect(what, D, got, LATTICE_OK);
        if (device != 0) fail("%s left device %d current", what, device);
    };
    want_device = 1;
    device = 0;
    after("layer_norm", lattice_layer_norm(D, nullptr, x, LATTICE_F32, C, rows, C, nullptr, nullptr, 0.f, y, LATTICE_F32, C,
                                           v, v + rows));
    after("layer_norm_backward",
          lattice_layer_norm_backward(D, nullptr, y, LATTICE_F32, C, x, LATTICE_F32, C, rows, C, v, v + rows, nullptr,
                                      nullptr, C, v + 2 * rows, v + 3 * rows));
    after("linear_cross_entropy",
          lattice_linear_cross_entropy(D, LATTICE_F32, x, C, rows, C, w, C, K, nullptr, target, -100, 1, v, nullptr, y,
                                       nullptr, nullptr));
    after("orthogonalize", lattice_orthogonalize(D, x, LATTICE_F32, 1, C, (int)rows, 0, rows, 5, ns, 0.f, y, LATTICE_F32));
    after("get_status", lattice_dense_get_status(D));
    lattice_dense_destroy(D);
    if (device != 0) fail("destroy left device %d current", device);
}

// -- stream ------------------------------------------------------------------

// Everything a handle does from its making on is in the order of its stream,
// which need not wait for the null stream.
void the_handles_stream() {
    int stream_of_its_own = 0;
    const int64_t rows = 70000;
    const int C = 200, K = 300;
    float *x = buffer<float>(rows * C), *y = buffer<float>(rows * C), *v = buffer<float>(4 * rows), *w = buffer<float>(K * C);
    int64_t *target = buffer<int64_t>(rows);
    const float ns[3] = {1.5f, -0.5f, 0.f};
    want_stream = reinterpret_cast<hipStream_t>(&stream_of_its_own);
    lattice_dense *D = handle(want_stream);
    for (const lattice_dtype t : {LATTICE_F32, LATTICE_BF16}) {
        expect("layer_norm", D, lattice_layer_norm(D, nullptr, x, t, C, rows, C, nullptr, nullptr, 0.f, y, t, C, v, v + rows),
               LATTICE_OK);
        expect("layer_norm_backward", D,
               lattice_layer_norm_backward(D, nullptr, y, t, C, x, t, C, rows, C, v, v + rows, nullptr, nullptr, C,
                                           v + 2 * rows, v + 3 * rows),
               LATTICE_OK);
        for (const int k : {20, K})
            expect("linear_cross_entropy", D,
                   lattice_linear_cross_entropy(D, t, x, C, rows, C, w, C, k, nullptr, target, -100, 1, v, v + 1, y, nullptr,
                                                v + 2 * rows),
                   LATTICE_OK);
        for (const int n : {100, 400})
            expect("orthogonalize", D, lattice_orthogonalize(D, x, t, 2, n, n, n * n, n, 5, ns, 0.f, y, t), LATTICE_OK);
    }
    expect("get_status", D, lattice_dense_get_status(D), LATTICE_OK);
    lattice_dense_destroy(D);
}

// -- empty inputs ------------------------------------------------------------

// No rows: every width and output is taken, and no launch is malformed.
void no_rows() {
    const int most = 1 << 20;
    lattice_dense *D = handle();
    float *grad = buffer<float>(2 * most);
    for (const int C : {32, 9000, 17000, most})
        for (const lattice_dtype t : {LATTICE_F32, LATTICE_BF16})
            for (int wanted = 0; wanted < 4; ++wanted)
                expect("layer_norm_backward", D,
                       lattice_layer_norm_backward(D, nullptr, nullptr, t, C, nullptr, t, C, 0, C, nullptr, nullptr, nullptr,
                                                   nullptr, C, wanted & 1 ? grad : nullptr, wanted & 2 ? grad + C : nullptr),
                       LATTICE_OK);
    lattice_dense_destroy(D);
}

}  // namespace

int main(int argc, char **argv) {
    const std::map<std::string, void (*)()> checks = {{"many_pieces", many_pieces},
                                                         {"captured_scratch", captured_scratch},
                                                         {"another_current_device", another_current_device},
                                                         {"the_handles_stream", the_handles_stream},
                                                         {"no_rows", no_rows},
                                                         {"products_stay_inside", products_stay_inside}};
    const auto it = checks.find(argc > 1 ? argv[1] : "");
    if (it == checks.end()) fail("which check?");
    it->second();
    std::printf("ok\n");
    return 0;
}
