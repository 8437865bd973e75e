// The launches of the dense operators' largest calls, without a GPU: a launch of 2^32 or
// more threads along a side is refused by the runtime.  The stand-in of the HIP runtime
// is host_driver.cpp's.
//
//   launch_driver CHECK      prints "ok", or what is wrong and exits with 1
#define main host_driver_main
#include "host_driver.cpp"
#undef main

namespace {

void bounded(const Launch &l) {
    const uint64_t most = (uint64_t)1 << 32;
    if ((uint64_t)l.grid.x * pushed_block.x >= most || (uint64_t)l.grid.y * pushed_block.y >= most ||
        (uint64_t)l.grid.z * pushed_block.z >= most)
        fail("%s: %u x %u x %u workgroups of %u x %u x %u threads", l.name.c_str(), l.grid.x, l.grid.y, l.grid.z,
             pushed_block.x, pushed_block.y, pushed_block.z);
}

// Rows up to the most there may be, of every group of lanes that a head is given.
void rotations() {
    lattice_dense *D = handle();
    for (const lattice_dtype t : {LATTICE_BF16, LATTICE_F32})
        for (const int C : {1, 3, 8, 20, 32, 48, 64, 100, 128, 130, 200, 256})
            for (int bits = 22; bits <= 30; ++bits)
                for (const int heads : {1, 3, 16}) {
                    const int64_t rows = ((int64_t)1 << bits) - (bits % 2 ? 1 : 0), w = (int64_t)heads * C;
                    const int sections[1] = {C / 2};
                    char *q = buffer<char>(rows * w * 4), *k = buffer<char>(rows * w * 4);
                    char *gq = buffer<char>(rows * w * 4), *gk = buffer<char>(rows * w * 4);
                    float *pos = buffer<float>(rows), *freq = buffer<float>(C), *gg = buffer<float>(2 * C);
                    expect("rotate_heads", D,
                           lattice_rotate_heads(D, t, rows, heads, heads, C, q, w, C, k, w, C, pos, 0, 1, 1, sections, freq, 1,
                                                nullptr, nullptr, 1e-6f, 0, q, w, C, k, w, C),
                           LATTICE_OK);
                    expect("rotate_heads_backward", D,
                           lattice_rotate_heads_backward(D, t, rows, heads, heads, C, gq, w, C, gk, w, C, q, w, C, k, w, C, pos,
                                                         0, 1, 1, sections, freq, 1, nullptr, nullptr, 1e-6f, 0, gq, w, C, gk,
                                                         w, C, gg, gg + C),
                           LATTICE_OK);
                }
    lattice_dense_destroy(D);
}

void attention() {
    lattice_dense *D = handle();
    for (const lattice_dtype t : {LATTICE_BF16, LATTICE_F32})
        for (const int C : {1, 64, 128})
            for (int bits = 20; bits <= 30; bits += 5)
                for (const int heads : {1, 3, 64}) {
                    const int64_t rows = (int64_t)1 << bits, w = (int64_t)heads * C;
                    char *x[8];
                    for (char *&p : x) p = buffer<char>(rows * w * 4);
                    float *lse = buffer<float>(heads * rows);
                    expect("attention", D,
                           lattice_attention(D, t, rows, rows, heads, heads, C, x[0], w, C, x[1], w, C, x[2], w, C, nullptr,
                                             nullptr, nullptr, 1, 1, 1.f, 1, x[3], w, C, lse),
                           LATTICE_OK);
                    expect("attention_backward", D,
                           lattice_attention_backward(D, t, rows, rows, heads, heads, C, x[4], w, C, x[0], w, C, x[1], w, C, x[2],
                                                      w, C, x[3], w, C, lse, nullptr, nullptr, nullptr, 1, 1, 1.f, 1, x[5], x[6],
                                                      x[7]),
                           LATTICE_OK);
                }
    lattice_dense_destroy(D);
}

void clipping() {
    lattice_dense *D = handle();
    float *norm = buffer<float>(1);
    for (const int count : {1, 64, 1000, LATTICE_CLIP_MAX_TENSORS})
        for (const int64_t n : {(int64_t)1, (int64_t)1 << 20, (int64_t)1 << 40}) {
            std::vector<const void *> in;
            std::vector<void *> out;
            const std::vector<lattice_dtype> types(count, LATTICE_F32);
            const std::vector<int64_t> values(count, n);
            // (as far apart as they must be; nothing is allocated for them)
            for (int i = 0; i < count; ++i) {
                out.push_back(reinterpret_cast<void *>(((uintptr_t)1 << 44) + (uintptr_t)i * (uintptr_t)n * 4));
                in.push_back(out.back());
            }
            expect("clip_gradients", D,
                   lattice_clip_gradients(D, count, in.data(), types.data(), out.data(), types.data(), values.data(), 1.f, 0.f,
                                          norm),
                   LATTICE_OK);
        }
    lattice_dense_destroy(D);
}

void normalisation() {
    lattice_dense *D = handle();
    for (const int C : {1, 7, 64, 1000, 1 << 20})
        for (int bits = 20; bits <= 31; ++bits) {
            const int64_t rows = (int64_t)1 << bits;
            char *x = buffer<char>(rows * C * 4), *g = buffer<char>(rows * C * 4);
            float *mean = buffer<float>(rows), *rstd = buffer<float>(rows), *sums = buffer<float>(2 * C);
            char *gx = buffer<char>(rows * C * 4);
            expect("layer_norm", D,
                   lattice_layer_norm(D, nullptr, x, LATTICE_F32, C, rows, C, nullptr, nullptr, 1e-5f, g, LATTICE_F32, C, mean,
                                      rstd),
                   LATTICE_OK);
            expect("layer_norm_backward", D,
                   lattice_layer_norm_backward(D, nullptr, g, LATTICE_F32, C, x, LATTICE_F32, C, rows, C, mean, rstd, nullptr,
                                               gx, C, sums, sums + C),
                   LATTICE_OK);
        }
    lattice_dense_destroy(D);
}

}  // namespace

int main(int argc, char **argv) {
    const std::map<std::string, void (*)()> checks = {
        {"rotations", rotations}, {"attention", attention}, {"clipping", clipping}, {"normalisation", normalisation}};
    const auto it = checks.find(argc > 1 ? argv[1] : "");
    if (it == checks.end()) fail("which check?");
    on_launch = bounded;
    it->second();
    std::printf("ok\n");
    return 0;
}
