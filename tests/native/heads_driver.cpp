// The host side of attention, of the rotation of heads and of clipping without a GPU:
// more checks for the stand-in of the HIP runtime in host_driver.cpp.
//
//   heads_driver CHECK      prints "ok", or what is wrong and exits with 1
#define main host_driver_main
#include "host_driver.cpp"
#undef main

namespace {

struct Attention {
    lattice_dtype dtype = LATTICE_F32;
    int64_t q_rows = 100, kv_rows = 90, sequences = 3;
    int heads = 4, kv_heads = 2, C = 32;
    float scale = 0.5f;
    int causal = 1, rest = 1;
    char *q = nullptr, *k = nullptr, *v = nullptr, *out = nullptr, *grad = nullptr, *gq = nullptr, *gk = nullptr, *gv = nullptr;
    float *lse = nullptr;
    int32_t *starts = nullptr, *kv_starts = nullptr, *lengths = nullptr;

    int64_t q_row() const { return (int64_t)heads * C; }
    int64_t k_row() const { return (int64_t)kv_heads * C; }
    // Buffers of the sizes that the fields say.
    void take() {
        const int64_t e = dtype == LATTICE_BF16 ? 2 : 4, nq = q_rows * q_row() * e, nk = kv_rows * k_row() * e;
        for (char **p : {&q, &out, &grad, &gq}) *p = buffer<char>(nq);
        for (char **p : {&k, &v, &gk, &gv}) *p = buffer<char>(nk);
        lse = buffer<float>(heads * q_rows);
        starts = buffer<int32_t>(sequences + 1);
        kv_starts = buffer<int32_t>(sequences + 1);
        lengths = buffer<int32_t>(sequences);
    }
    lattice_status forward(lattice_dense *D) const {
        return lattice_attention(D, dtype, q_rows, kv_rows, heads, kv_heads, C, q, q_row(), C, k, k_row(), C, v, k_row(), C,
                                 starts, kv_starts, lengths, sequences, causal, scale, rest, out, q_row(), C, lse);
    }
    lattice_status backward(lattice_dense *D) const {
        return lattice_attention_backward(D, dtype, q_rows, kv_rows, heads, kv_heads, C, grad, q_row(), C, q, q_row(), C, k,
                                          k_row(), C, v, k_row(), C, out, q_row(), C, lse, starts, kv_starts, lengths,
                                          sequences, causal, scale, rest, gq, gk, gv);
    }
};

struct Rotation {
    lattice_dtype dtype = LATTICE_BF16;
    int64_t rows = 50;
    int heads = 4, kv_heads = 2, C = 32, axes = 3, sections[8] = {5, 5, 6, 0, 0, 0, 0, 0}, norm = 1;
    float eps = 1e-6f;
    char *q = nullptr, *k = nullptr, *oq = nullptr, *ok = nullptr, *gq = nullptr, *gk = nullptr;
    float *pos = nullptr, *freq = nullptr, *gain = nullptr, *gg = nullptr;

    int64_t q_row() const { return (int64_t)heads * C; }
    int64_t k_row() const { return (int64_t)kv_heads * C; }
    void take() {
        const int64_t e = dtype == LATTICE_BF16 ? 2 : 4;
        for (char **p : {&q, &oq, &gq}) *p = buffer<char>(rows * q_row() * e);
        for (char **p : {&k, &ok, &gk}) *p = buffer<char>(rows * k_row() * e);
        pos = buffer<float>(rows * axes);
        freq = buffer<float>(C);
        gain = buffer<float>(C);
        gg = buffer<float>(2 * C);
    }
    lattice_status forward(lattice_dense *D) const {
        return lattice_rotate_heads(D, dtype, rows, heads, kv_heads, C, q, q_row(), C, k, k_row(), C, pos, 0, axes, axes,
                                    sections, freq, norm, gain, gain, eps, 0, oq, q_row(), C, ok, k_row(), C);
    }
    lattice_status backward(lattice_dense *D) const {
        return lattice_rotate_heads_backward(D, dtype, rows, heads, kv_heads, C, gq, q_row(), C, gk, k_row(), C, q, q_row(),
                                             C, k, k_row(), C, pos, 0, axes, axes, sections, freq, norm, gain, gain, eps, 0,
                                             oq, q_row(), C, ok, k_row(), C, gg, gg + C);
    }
};

template <class F>
void refused(const char *what, lattice_dense *D, F call) {
    const int64_t before = launches;
    const size_t held = blocks.size();
    expect(what, D, call(), LATTICE_E_ARG);
    if (launches != before || blocks.size() != held) fail("%s: refused, but something was enqueued or allocated", what);
}

void refusals() {
    lattice_dense *D = handle();
    const Attention good = [] { Attention a; a.take(); return a; }();
    expect("attention", D, good.forward(D), LATTICE_OK);
    expect("attention_backward", D, good.backward(D), LATTICE_OK);
    auto attention = [&](const char *what, auto change) {
        Attention a = good;
        change(a);
        refused(what, D, [&] { return a.forward(D); });
        refused(what, D, [&] { return a.backward(D); });
    };
    attention("heads not a multiple", [](Attention &a) { a.kv_heads = 3; });
    attention("no key heads", [](Attention &a) { a.kv_heads = 0; });
    attention("no heads", [](Attention &a) { a.heads = 0; });
    attention("no channels", [](Attention &a) { a.C = 0; });
    attention("many channels", [](Attention &a) { a.C = 129; });
    attention("negative rows", [](Attention &a) { a.q_rows = -1; });
    attention("many rows", [](Attention &a) { a.kv_rows = LATTICE_ATTENTION_MAX_ROWS + 1; });
    attention("negative sequences", [](Attention &a) { a.sequences = -1; });
    attention("many sequences", [](Attention &a) { a.sequences = LATTICE_ATTENTION_MAX_SEQUENCES + 1; });
    attention("no starts for sequences", [](Attention &a) { a.starts = a.kv_starts = nullptr; });
    attention("kv_starts alone", [](Attention &a) { a.starts = nullptr; a.sequences = 1; });
    attention("scale 0", [](Attention &a) { a.scale = 0.f; });
    attention("scale NaN", [](Attention &a) { a.scale = NAN; });
    attention("scale infinite", [](Attention &a) { a.scale = INFINITY; });
    attention("a type there is not", [](Attention &a) { a.dtype = (lattice_dtype)7; });
    attention("no q", [](Attention &a) { a.q = nullptr; });
    attention("no k", [](Attention &a) { a.k = nullptr; });
    attention("no v", [](Attention &a) { a.v = nullptr; });
    attention("no out", [](Attention &a) { a.out = nullptr; });
    refused("out is q", D, [&] { Attention a = good; a.out = a.q; return a.forward(D); });
    refused("out overlaps v", D, [&] { Attention a = good; a.out = a.v + 64; return a.forward(D); });
    refused("no lse", D, [&] { Attention a = good; a.lse = nullptr; return a.backward(D); });
    refused("grad_q is grad_out", D, [&] { Attention a = good; a.gq = a.grad; return a.backward(D); });
    refused("grad_k is grad_v", D, [&] { Attention a = good; a.gk = a.gv; return a.backward(D); });
    refused("no grad_v", D, [&] { Attention a = good; a.gv = nullptr; return a.backward(D); });
    refused("rows of out overlap", D, [&] {
        return lattice_attention(D, LATTICE_F32, 100, 90, 4, 2, 32, good.q, 128, 32, good.k, 64, 32, good.v, 64, 32, nullptr,
                                 nullptr, nullptr, 1, 0, 1.f, 1, good.out, 100, 32, nullptr);
    });
    refused("a negative stride", D, [&] {
        return lattice_attention(D, LATTICE_F32, 100, 90, 4, 2, 32, good.q, -128, 32, good.k, 64, 32, good.v, 64, 32, nullptr,
                                 nullptr, nullptr, 1, 0, 1.f, 1, good.out, 128, 32, nullptr);
    });

    refused("strides past all addresses", D, [&] {
        return lattice_attention(D, LATTICE_F32, LATTICE_ATTENTION_MAX_ROWS, 90, 4, 2, 32, good.q, (int64_t)1 << 34, 32, good.k,
                                 64, 32, good.v, 64, 32, nullptr, nullptr, nullptr, 1, 0, 1.f, 1, good.out, (int64_t)1 << 34, 32,
                                 nullptr);
    });

    const Rotation fine = [] { Rotation r; r.take(); return r; }();
    expect("rotate_heads", D, fine.forward(D), LATTICE_OK);
    expect("rotate_heads_backward", D, fine.backward(D), LATTICE_OK);
    auto rotation = [&](const char *what, auto change) {
        Rotation r = fine;
        change(r);
        refused(what, D, [&] { return r.forward(D); });
        refused(what, D, [&] { return r.backward(D); });
    };
    rotation("many pairs", [](Rotation &r) { r.sections[2] = 7; });
    rotation("a negative section", [](Rotation &r) { r.sections[0] = -1; });
    rotation("a section past an int's sum", [](Rotation &r) { r.sections[0] = r.sections[1] = 0x7fffffff; });
    rotation("no axes", [](Rotation &r) { r.axes = 0; });
    rotation("many axes", [](Rotation &r) { r.axes = 9; });
    rotation("many channels", [](Rotation &r) { r.C = 257; });
    rotation("no heads", [](Rotation &r) { r.heads = 0; });
    rotation("negative rows", [](Rotation &r) { r.rows = -1; });
    rotation("eps NaN", [](Rotation &r) { r.eps = NAN; });
    rotation("gains without the norm", [](Rotation &r) { r.norm = 0; });
    rotation("no positions", [](Rotation &r) { r.pos = nullptr; });
    rotation("no frequencies", [](Rotation &r) { r.freq = nullptr; });
    rotation("no q", [](Rotation &r) { r.q = nullptr; });
    rotation("no out", [](Rotation &r) { r.oq = nullptr; });
    rotation("out_q is k", [](Rotation &r) { r.oq = r.k; });
    rotation("out_k overlaps q", [](Rotation &r) { r.ok = r.q + 2; });
    Rotation in_place = fine;
    in_place.oq = in_place.q;
    in_place.ok = in_place.k;
    expect("rotate_heads in place", D, in_place.forward(D), LATTICE_OK);
    in_place.oq = in_place.gq;
    in_place.ok = in_place.gk;
    expect("rotate_heads_backward in place", D, in_place.backward(D), LATTICE_OK);

    float *x = buffer<float>(100), *y = buffer<float>(100), *norm = buffer<float>(1);
    const auto clip = [&](std::vector<float *> in, std::vector<float *> out, std::vector<int64_t> n, float most = 1.f,
                          float eps = 0.f, float *to = nullptr, lattice_dtype out_type = LATTICE_F32) {
        const std::vector<lattice_dtype> t(in.size(), LATTICE_F32), u(in.size(), out_type);
        return lattice_clip_gradients(D, (int)in.size(), reinterpret_cast<const void *const *>(in.data()), t.data(),
                                      reinterpret_cast<void *const *>(out.data()), u.data(), n.data(), most, eps,
                                      to ? to : norm);
    };
    expect("clip_gradients", D, clip({x, y}, {x, y}, {100, 100}), LATTICE_OK);
    expect("clip_gradients of the same input twice", D, clip({x, x}, {y, y + 50}, {50, 50}), LATTICE_OK);
    expect("clip_gradients of nothing", D, clip({}, {}, {}), LATTICE_OK);
    expect("clip_gradients of no values", D, clip({nullptr}, {nullptr}, {0}), LATTICE_OK);
    refused("the same tensor twice", D, [&] { return clip({x, x}, {x, x}, {100, 100}); });
    refused("a part of another", D, [&] { return clip({x, x + 20}, {x, x + 20}, {50, 10}); });
    refused("each other's outputs", D, [&] { return clip({x, y}, {y, x}, {100, 100}); });
    refused("shifted", D, [&] { return clip({x}, {x + 1}, {99}); });
    refused("in place of another type", D, [&] { return clip({x}, {x}, {50}, 1.f, 0.f, nullptr, LATTICE_BF16); });
    refused("no input", D, [&] { return clip({nullptr}, {y}, {50}); });
    refused("no output", D, [&] { return clip({x}, {nullptr}, {50}); });
    refused("negative values", D, [&] { return clip({x}, {y}, {-1}); });
    refused("negative max_norm", D, [&] { return clip({x}, {y}, {50}, -1.f); });
    refused("max_norm NaN", D, [&] { return clip({x}, {y}, {50}, NAN); });
    refused("negative eps", D, [&] { return clip({x}, {y}, {50}, 1.f, -1.f); });
    refused("no norm", D, [&] {
        return lattice_clip_gradients(D, 0, nullptr, nullptr, nullptr, nullptr, nullptr, 1.f, 0.f, nullptr);
    });
    lattice_dense_destroy(D);
}

// Calls without rows, keys or sequences: no error, whatever has no address.
void nothing_there() {
    lattice_dense *D = handle();
    for (int64_t q : {0, 5})
        for (int64_t kv : {0, 7})
            for (int64_t n : {0, 2}) {
                Attention a;
                a.q_rows = q;
                a.kv_rows = kv;
                a.sequences = n;
                a.take();
                if (q == 0) a.q = a.out = a.grad = a.gq = nullptr, a.lse = nullptr;
                if (kv == 0) a.k = a.v = a.gk = a.gv = nullptr;
                expect("attention", D, a.forward(D), LATTICE_OK);
                expect("attention_backward", D, a.backward(D), LATTICE_OK);
            }
    Rotation r;
    r.rows = 0;
    r.take();
    r.q = r.k = r.oq = r.ok = r.gq = r.gk = nullptr;
    r.pos = nullptr;
    expect("rotate_heads", D, r.forward(D), LATTICE_OK);
    expect("rotate_heads_backward", D, r.backward(D), LATTICE_OK);
    lattice_dense_destroy(D);
}

// 3000 calls of random sizes, another device current: all launches, waits and allocations are
// the handle's, and no launch has an empty grid or one that is too large.
void random_sizes() {
    std::mt19937_64 rng(7);
    const auto log_size = [&](double lo, double hi) {
        return (int64_t)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi + 1))(rng));
    };
    device = 1;
    lattice_dense *D = handle(reinterpret_cast<void *>(0x1234));
    want_device = 1;
    want_stream = reinterpret_cast<hipStream_t>(0x1234);
    device = 0;
    on_launch = [](const Launch &l) {
        if ((uint64_t)l.grid.x * l.grid.y * l.grid.z > (uint64_t)1 << 31) fail("%s: a grid of %u x %u x %u", l.name.c_str(),
                                                                               l.grid.x, l.grid.y, l.grid.z);
    };
    for (int i = 0; i < 3000; ++i) {
        Attention a;
        a.dtype = rng() % 2 ? LATTICE_BF16 : LATTICE_F32;
        a.q_rows = log_size(1, 3e5);
        a.kv_rows = log_size(1, 3e5);
        a.sequences = log_size(1, 2e5);
        a.kv_heads = (int)log_size(1, 64);
        a.heads = a.kv_heads * (int)log_size(1, 200);
        a.C = 1 + (int)(rng() % 128);
        a.causal = rng() % 2;
        device = 1;
        a.take();
        device = 0;
        expect("attention", D, a.forward(D), LATTICE_OK);
        expect("attention_backward", D, a.backward(D), LATTICE_OK);
        Rotation r;
        r.dtype = a.dtype;
        r.rows = a.q_rows;
        r.heads = a.heads;
        r.kv_heads = a.kv_heads;
        r.C = 1 + (int)(rng() % 256);
        const int pairs = (int)(rng() % (r.C / 2 + 1));
        r.sections[0] = pairs / 2;
        r.sections[1] = pairs - pairs / 2;
        r.sections[2] = 0;
        device = 1;
        r.take();
        device = 0;
        expect("rotate_heads", D, r.forward(D), LATTICE_OK);
        expect("rotate_heads_backward", D, r.backward(D), LATTICE_OK);
        if (device != 0) fail("a call left device %d current", device);
    }
    lattice_dense_destroy(D);
}

// More tiles than the threads along a side of a launch have bits for (32, 512 or fewer of a
// workgroup): several launches, which have all tiles between them.
void many_tiles() {
    lattice_dense *D = handle();
    static int64_t workgroups = 0;
    on_launch = [](const Launch &l) {
        if (l.grid.x >= 1u << 23 || l.grid.y > 65535 || l.grid.z > 65535)
            fail("%s: a grid of %u x %u x %u", l.name.c_str(), l.grid.x, l.grid.y, l.grid.z);
        workgroups += (int64_t)l.grid.x * l.grid.y;
    };
    for (const lattice_dtype dtype : {LATTICE_BF16, LATTICE_F32})
        for (const int64_t kv_rows : {(int64_t)700000, (int64_t)2800000})
            for (const int heads : {1, 32}) {
                Attention a;
                a.dtype = dtype;
                a.sequences = heads == 1 ? LATTICE_ATTENTION_MAX_SEQUENCES : 600000;
                a.q_rows = 700000;
                a.kv_rows = kv_rows;
                a.heads = a.kv_heads = heads;
                a.C = 8;
                a.take();
                workgroups = 0;
                expect("attention", D, a.forward(D), LATTICE_OK);
                if (workgroups < heads * a.sequences) fail("attention: %lld workgroups", (long long)workgroups);
                workgroups = 0;
                expect("attention_backward", D, a.backward(D), LATTICE_OK);
                if (workgroups < 2 * heads * a.sequences) fail("attention_backward: %lld workgroups", (long long)workgroups);
            }
    lattice_dense_destroy(D);
}

}  // namespace

int main(int argc, char **argv) {
    const std::map<std::string, void (*)()> checks = {
        {"refusals", refusals}, {"nothing_there", nothing_there}, {"random_sizes", random_sizes},
        {"many_tiles", many_tiles}};
    const auto it = checks.find(argc > 1 ? argv[1] : "");
    if (it == checks.end()) fail("which check?");
    it->second();
    std::printf("ok\n");
    return 0;
}
