// Softmax attention, backward.  With g = dL/do, delta_i = g_i . o_i and
// p_ij = exp(s_ij - lse_i) made again from the scores,
//   t_ij = p_ij (g_i . v_j - delta_i)          (dL/ds_ij)
//   dq_i = scale sum_j t_ij k_j,  dk_j = scale sum_i t_ij q_i,  dv_j = sum_i p_ij g_i.
//
// Two launches, each with sums of its own in registers, so that no float is added
// by atomics and two calls give the same bits, at the price of making p and g . v
// twice (seven products in place of five):
//   by queries   tiles of columns as in the forward pass, the keys go by; makes
//                delta on the way and dq.
//   by keys      each wavefront has 32 keys of a key head; the rows of all its
//                query heads go by; makes dk and dv, so that heads which share
//                keys are added here.
// p and t are rounded to bf16 for the products with bf16 tensors (by up to 2^-8 of
// each term), all sums are fp32.
//
// 12 sequences of 1 to 3400 rows of 16 (4) heads of 128, causal, bf16, take 283 us by
// queries (0.77 PFLOP/s) and 464 by keys (0.63), and 16 for the parts of keys.  Neither keeps one
// unit busy all the time: the matrix cores work for 0.36 of it by queries and 0.31 by keys (counters),
// and by keys a wavefront reads 48 KB of LDS for 32 products: eight wavefronts' reads, at 128 bytes
// a cycle, take half as long again as their products (2048 cycles), so LDS is the nearer bound.
//
// Vector registers that do not fit: k_by_keys<PLANES, 64> keeps 15 in memory, k_by_keys<F32, 128> without
// direct loads 31; no other instance has any.
#include <algorithm>

#include "attention.h"

namespace {

using namespace attend;

struct Params {
    Packing pack;
    View q, k, v, g;
    View o, g_stored;         // as they are stored
    void *dq, *dk, *dv;       // without gaps
    const float *lse;         // [heads][rows]
    float *delta;             // the same
    int heads, kv_heads, D, group;
    int parts, tile_heads;    // by queries, as in the forward pass
    int units, R, slots;
    int64_t block0;           // of the launch's workgroups, among all of them
    Cut cut;                  // of blocks of keys, or of rows
    float c, scale;
    bool zero_rest;
    float *part;              // of the parts, without gaps, one after another
    int32_t *status;
};

// This lane's part of a bf16 row to its place in a tile.
template <int DP>
__device__ __forceinline__ void load_fragments_to(const View &x, int64_t row, int head, int D, char *tile) {
    using L = RowsOf<BF16, DP>;
    const int lane = threadIdx.x & 63;
    Fragments<BF16, DP> f;
    load_fragments<BF16, DP>(x, row, head, D, f);
#pragma unroll
    for (int t = 0; t < L::STEPS; ++t)
        *reinterpret_cast<u32x4_t *>(tile + L::at(lane & 31, 2 * t + (lane >> 5))) = f.v[0][t];
}

// acc = (32 rows of one bf16 tile) (32 rows of another)^T.
template <int DP>
__device__ __forceinline__ void rows_times_rows(const char *a, const char *b, f32x16_t &acc) {
    using L = RowsOf<BF16, DP>;
    const int lane = threadIdx.x & 63, row = lane & 31, h = lane >> 5;
#pragma unroll
    for (int t = 0; t < L::STEPS; ++t) {
        const int at = L::at(row, 2 * t + h);
        mma<true>(*reinterpret_cast<const u32x4_t *>(a + at), *reinterpret_cast<const u32x4_t *>(b + at), acc);
    }
}

// Add the second group's sums to the first's, by way of LDS (4 wavefronts x 32 x DP).
template <int DP>
__device__ __forceinline__ void add_groups(char *lds, int wave, int group, f32x16_t (&x)[DP / 32]) {
    float4 *room = reinterpret_cast<float4 *>(lds + wave * 32 * DP * 4) + (threadIdx.x & 63);
    __syncthreads();
    if (group == 1)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                room[(4 * d + g) * 64] = make_float4(x[d][4 * g], x[d][4 * g + 1], x[d][4 * g + 2], x[d][4 * g + 3]);
    __syncthreads();
    if (group == 0)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 t = room[(4 * d + g) * 64];
                x[d][4 * g] += t.x, x[d][4 * g + 1] += t.y, x[d][4 * g + 2] += t.z, x[d][4 * g + 3] += t.w;
            }
}

// This lane's share of the product of two rows as they are stored.
template <bool BF16>
__device__ __forceinline__ float dot(const View &x, const View &y, int64_t row, int head, int D) {
    constexpr int VEC = BF16 ? 8 : 4, E = BF16 ? 2 : 4;
    const char *a = reinterpret_cast<const char *>(x.p) + (row * x.row + head * x.head) * E;
    const char *b = reinterpret_cast<const char *>(y.p) + (row * y.row + head * y.head) * E;
    float s = 0.f;
    for (int c0 = VEC * ((threadIdx.x & 63) >> 5); c0 < D; c0 += 2 * VEC) {
        float u[VEC], v[VEC];
        load_row<BF16, VEC>(a, c0, D, u);
        load_row<BF16, VEC>(b, c0, D, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s = fmaf(u[i], v[i], s);
    }
    return s;
}

// Store a column's channels times f: row `at` of D values, at its type or, of a
// split, in fp32.
template <bool BF16, int DP>
__device__ __forceinline__ void store_column(void *out, float *part, int64_t at, int D, const f32x16_t (&x)[DP / 32],
                                             float f) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c0 = 32 * d + 8 * g + 4 * h;
            if (c0 >= D) continue;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = x[d][4 * g + i] * f;
            if (part)
                store4<false>(part + at * D, c0, D, v);
            else
                store4<BF16>(reinterpret_cast<char *>(out) + at * D * (BF16 ? 2 : 4), c0, D, v);
        }
}

// By queries: 4 wavefronts of 32 columns, blocks of keys of
constexpr int kKeyBlock = 32;
constexpr int kShort = 128;  // keys of a tile whose delta is made from the scores
template <Type T, int DP, bool DMA>
__global__ __launch_bounds__(256, T != F32 || DP < 128 ? 2 : 1) void k_by_queries(Params a) {
    using L = RowsOf<T, DP>;
    constexpr int KT = kKeyBlock, HALF = tile_bytes<T, DP>(KT), STAGE = 2 * HALF;
    constexpr bool OUT16 = T == BF16;
    const int D = T == PLANES ? DP : a.D;  // as the operands are laid out
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int unit, slot, first;
    const int split = blockIdx.y;
    if (!unit_of(a.block0 + blockIdx.x, a.units, a.slots, true, unit, slot)) return;
    const int kv_head = unit / a.parts, part = unit % a.parts, head0 = kv_head * a.group + part * a.tile_heads;
    const int left = a.group - part * a.tile_heads, heads = left < a.tile_heads ? left : a.tile_heads;
    const Sequence s = locate(a.pack, a.R, slot, false, first, a.status);
    if (first >= s.q_len || heads <= 0) return;
    const int rows = s.q_len - first < a.R ? s.q_len - first : a.R;
    if (!s.real) {
        if (a.zero_rest && split == 0)
            for (int r = 0; r < rows; ++r)
                for (int h = 0; h < heads; ++h)
                    zero_row<OUT16>(reinterpret_cast<char *>(a.dq) +
                                       ((s.q0 + first + r) * a.heads + head0 + h) * a.D * (OUT16 ? 2 : 4),
                                   a.D, threadIdx.x, 256);
        return;
    }
    const int least = keys_seen(s, a.pack.causal, first), most = keys_seen(s, a.pack.causal, first + rows - 1);
    const int n = (most + KT - 1) / KT, parts = parts_of(a.cut, n);
    if (split >= parts) return;
    float *mine_part = parts > 1 ? a.part + (int64_t)split * a.pack.q_rows * a.heads * a.D : nullptr;
    const int lane = threadIdx.x & 63, wave = gemm::wave_index();
    const int column = wave * 32 + (lane & 31);
    int r = column / heads;
    const int head = head0 + column - r * heads;
    const bool mine = r < rows;
    r = mine ? r : rows - 1;
    const int64_t row = s.q0 + first + r;
    const int seen = keys_seen(s, a.pack.causal, first + r);
    int last = (wave * 32 + 31) / heads;
    last = last < rows ? last : rows - 1;
    const int wave_most = uniform(keys_seen(s, a.pack.causal, first + last));

    Fragments<T, DP> q, g;
    float delta = pair_sum(dot<OUT16>(a.g_stored, a.o, row, head, a.D));
    load_fragments<T, DP>(a.g, row, head, D, g);
    load_fragments<T, DP>(a.q, row, head, D, q);
    const float lse = a.lse[head * a.pack.q_rows + row];
    const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;

    f32x16_t dq[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) clear(dq[d]);
    const int t0 = (int)((int64_t)n * split / parts), t1 = (int)((int64_t)n * (split + 1) / parts);
    Loader<T, DP, KT, 4, DMA> lk(a.k, s.k0, kv_head, D, wave), lv(a.v, s.k0, kv_head, D, wave);
    // blocks [from, to); ONLY_DELTA: no more than this lane's share of sum p (g . v) is made
    float sum = 0.f;
    auto blocks = [&](int from, int to, auto only_delta) {
        constexpr bool ONLY_DELTA = decltype(only_delta)::value;
        if (from < to) {
            lk.fetch(lds, from * KT, s.keys);
            lv.fetch(lds + HALF, from * KT, s.keys);
            lk.commit(lds);
            lv.commit(lds + HALF);
        }
        auto block = [&](int i, const char *__restrict now, char *__restrict next) {
            gemm::wait_and_barrier<0>();
            const bool more = i + 1 < to;
            if (more) {
                lk.fetch(next, (i + 1) * KT, s.keys);
                lv.fetch(next + HALF, (i + 1) * KT, s.keys);
            }
            if (i * KT < wave_most) {
                f32x16_t x, y;
                gemm::sched_barrier();
                clear(x);
                clear(y);
                rows_times<T, DP, KT>(now, 0, q, x);
                rows_times<T, DP, KT>(now + HALF, 0, g, y);
                if (T != F32) read_ahead<2 * kProducts<T> * L::STEPS, 2 * kPlanes<T> * L::STEPS, 6>();
                gemm::sched_barrier();
                if ((i + 1) * KT > least) {
                    seldom();
                    mask(x, i * KT, seen);
                }
                if constexpr (ONLY_DELTA) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum = fmaf(exp2_(fmaf(x[e], a.c, -lse2)), y[e], sum);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = exp2_(fmaf(x[e], a.c, -lse2)) * (y[e] - delta);
                    Right<T> t;
                    t.set(x);
                    columns_times<T, DP, KT>(now, 0, t, dq);
                }
            }
            if (more) {
                lk.commit(next);
                lv.commit(next + HALF);
            }
        };
        for (int i = from; i < to; i += 2) {
            block(i, lds, lds + STAGE);
            if (i + 1 < to) block(i + 1, lds + STAGE, lds);
        }
    };
    // Of few keys the outputs are as large as the values, and what rounding them to bf16 took
    // from delta shows in dq and dk (2.6e-3 of them for sequences of 1 to 558 rows, 2.3e-3 so;
    // rounding the results alone makes 1.7e-3).  Of many keys it does not.
    if (T == BF16 && most <= kShort) {
        blocks(0, n, std::true_type{});
        delta = pair_sum(sum);
        gemm::wait_and_barrier<0>();  // the blocks have been read
    }
    if (mine && lane < 32 && split == 0) a.delta[head * a.pack.q_rows + row] = delta;
    blocks(t0, t1, std::false_type{});
    if (mine) store_column<OUT16, DP>(a.dq, mine_part, row * a.heads + head, a.D, dq, a.scale);
}

// By keys: 128 keys, 32 for each of 4 wavefronts, or of 4 of each of QW groups of
// them that take the blocks of rows in turns and are added at the end.
//
// With K and V as right operands in registers and both results there, 128 channels take
// 300 registers, one wavefront a SIMD, and nothing runs beside its exponentials and
// waits (283 TFLOP/s); K and V are read from LDS instead (KV_LDS), which leaves room for
// two (0.63 PFLOP/s).
template <Type T, int DP>
struct ByKeys {
    static constexpr bool KV_LDS = T == BF16 && DP == 128;
    static constexpr int QW = T != F32 ? 2 : 1;
    static constexpr int WAVES = 4 * QW, THREADS = 64 * WAVES;
    static constexpr int HALF = tile_bytes<T, DP>(32), STAGE = 2 * HALF;   // of a group
    static constexpr int KV_BYTES = KV_LDS ? 8 * HALF : 0;
    static constexpr int LDS = 2 * QW * STAGE + KV_BYTES;
    // a group's result in LDS: 4 wavefronts of 32 x DP
    static_assert(QW == 1 || 4 * 32 * DP * 4 <= 2 * QW * STAGE, "LDS");
};

// Where the rows begin that see a tile of keys from `first` on.
constexpr int kRowBlock = 32;
__device__ __forceinline__ int first_row(const Params &a, const Sequence &s, int first) {
    const int r = a.pack.causal ? first + s.q_len - s.keys : 0;
    return (r < 0 ? 0 : r) / kRowBlock * kRowBlock;
}
__device__ __forceinline__ int row_blocks(const Params &a, const Sequence &s, int first) {
    const int r = first_row(a, s, first);
    return r < s.q_len ? (s.q_len - r + kRowBlock - 1) / kRowBlock : 0;
}

template <Type T, int DP, bool DMA>
__global__ __launch_bounds__((ByKeys<T, DP>::THREADS), T != F32 ? 2 : 1) void k_by_keys(Params a) {
    using L = RowsOf<T, DP>;
    using B = ByKeys<T, DP>;
    constexpr bool OUT16 = T == BF16;
    const int D = T == PLANES ? DP : a.D;  // as the operands are laid out
    constexpr int QT = kRowBlock, QW = B::QW;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ __attribute__((aligned(16))) float stats[2][QW][2][QT];  // lse (of 2) and delta of the blocks' rows
    const int split = blockIdx.y;
    int kv_head, slot, first;
    if (!unit_of(a.block0 + blockIdx.x, a.kv_heads, a.slots, false, kv_head, slot)) return;
    const Sequence s = locate(a.pack, a.R, slot, true, first, a.status);
    if (first >= s.kv_len) return;
    const int lane = threadIdx.x & 63, wave = gemm::wave_index() & 3, group = gemm::wave_index() >> 2, h = lane >> 5;
    const int64_t size = a.pack.kv_rows * a.kv_heads * a.D;
    const int key = first + wave * 32 + (lane & 31);
    // rows that no key of the tile counts in
    if (!s.real || first >= s.keys) {
        const int end = s.kv_len - first < a.R ? s.kv_len : first + a.R;
        if (a.zero_rest && split == 0)
            for (int j = first; j < end; ++j) {
                const int64_t at = ((s.k0 + j) * a.kv_heads + kv_head) * a.D * (OUT16 ? 2 : 4);
                zero_row<OUT16>(reinterpret_cast<char *>(a.dk) + at, a.D, threadIdx.x, B::THREADS);
                zero_row<OUT16>(reinterpret_cast<char *>(a.dv) + at, a.D, threadIdx.x, B::THREADS);
            }
        return;
    }
    // blocks of rows: those of each query head, one head after another
    const int r0 = first_row(a, s, first), per = row_blocks(a, s, first);
    const int64_t blocks = (int64_t)per * a.group;
    const int parts = parts_of(a.cut, blocks);
    if (split >= parts) return;
    const int64_t begin = blocks * split / parts, end = blocks * (split + 1) / parts;

    const bool counts = key < s.keys;
    const int64_t row = s.k0 + (counts ? key : s.keys - 1);
    Fragments<T, DP> k, v;
    char *k_tile = lds + 2 * QW * B::STAGE + 2 * wave * B::HALF, *v_tile = k_tile + B::HALF;
    if constexpr (B::KV_LDS) {
        if (group == 0)
            load_fragments_to<DP>(a.k, row, kv_head, D, k_tile);
        else
            load_fragments_to<DP>(a.v, row, kv_head, D, v_tile);
    } else {
        load_fragments<T, DP>(a.k, row, kv_head, D, k);
        load_fragments<T, DP>(a.v, row, kv_head, D, v);
    }
    f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
        clear(dk[d]);
        clear(dv[d]);
    }
    // this lane's key is seen from row `from` on, all keys of the tile from `all_see` on
    const int shift = a.pack.causal ? s.q_len - s.keys : 0;
    const int from = !counts ? 0x7fffffff : a.pack.causal ? key + shift : 0;
    const int all_see = first + a.R <= s.keys ? (a.pack.causal ? first + a.R - 1 + shift : 0) : 0x7fffffff;

    int64_t i = begin + group;
    int head = per > 0 ? (int)(i / per) : 0, at = per > 0 ? (int)(i % per) : 0;
    float stat = 0.f;  // lanes 0 .. 31 of a group's first wavefront: lse, the others delta
    bool inside = false;
    Loader<T, DP, QT, 4, DMA> lq(a.q, s.q0, kv_head * a.group, D, wave), lg(a.g, s.q0, kv_head * a.group, D, wave);
    const int64_t q_step = a.q.head * L::E, g_step = a.g.head * L::E;
    const char *q_base = lq.base, *g_base = lg.base;
    char *own = lds + group * 2 * B::STAGE;
    auto fetch = [&](char *to, int head, int at) {
        lq.base = q_base + head * q_step;
        lg.base = g_base + head * g_step;
        const int r = r0 + at * QT;
        lq.fetch(to, r, s.q_len);
        lg.fetch(to + B::HALF, r, s.q_len);
        if (wave == 0) {
            const int rr = r + (lane & 31);
            const int64_t where = (kv_head * a.group + head) * a.pack.q_rows + s.q0 + (rr < s.q_len ? rr : s.q_len - 1);
            stat = (h == 0 ? a.lse : a.delta)[where];
            inside = rr < s.q_len;
        }
    };
    auto commit = [&](char *to, int stage) {
        lq.commit(to);
        lg.commit(to + B::HALF);
        // (made here and not where it is loaded: that would wait for the blocks' loads)
        if (wave == 0)
            stats[stage][group][h][lane & 31] =
                h == 0 ? (inside && stat != -INFINITY ? stat * kLog2e : INFINITY) : (inside ? stat : 0.f);
    };
    if (i < end) {
        fetch(own, head, at);
        commit(own, 0);
    }
    // (all that is read in LDS is told to be apart from where the next block goes: the reads
    // would wait for its loads)
    auto block = [&](const char *__restrict now, char *__restrict next, const char *__restrict k_own,
                     const char *__restrict v_own, const float *__restrict stats_now, auto stage) {
        gemm::wait_and_barrier<0>();
        const bool here = i < end, more = i + QW < end;
        const int r = r0 + at * QT;
        i += QW;
        at += QW;
        while (at >= per) {
            at -= per;
            ++head;
        }
        if (more) fetch(next, head, at);
        if (here) {
            f32x16_t x, y;
            gemm::sched_barrier();
            clear(x);
            clear(y);
            if constexpr (B::KV_LDS) {
                rows_times_rows<DP>(now, k_own, x);
                rows_times_rows<DP>(now + B::HALF, v_own, y);
            } else {
                rows_times<T, DP, QT>(now, 0, k, x);
                rows_times<T, DP, QT>(now + B::HALF, 0, v, y);
            }
            if (T != F32) read_ahead<2 * kProducts<T> * L::STEPS, (B::KV_LDS ? 4 : 2 * kPlanes<T>) * L::STEPS, 8>();
            gemm::sched_barrier();
            if (r < all_see) {
                seldom();
                const int hidden = from - r - 4 * h;  // rows before it do not see this lane's key
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) < hidden) x[e] = -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float4 l = *reinterpret_cast<const float4 *>(stats_now + 8 * b + 4 * h);
                const float4 d = *reinterpret_cast<const float4 *>(stats_now + QT + 8 * b + 4 * h);
                const float ls[4] = {l.x, l.y, l.z, l.w}, ds[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    const int e = 4 * b + k4;
                    x[e] = exp2_(fmaf(x[e], a.c, -ls[k4]));
                    y[e] = x[e] * (y[e] - ds[k4]);
                }
            }
            Right<T> p;
            p.set(x);
            columns_times<T, DP, QT>(now + B::HALF, 0, p, dv);
            p.set(y);
            columns_times<T, DP, QT>(now, 0, p, dk);
        }
        if (more) commit(next, 1 - stage.value);
    };
    for (int64_t turn = begin; turn < end; turn += 2 * QW) {
        block(own, own + B::STAGE, k_tile, v_tile, stats[0][group][0], std::integral_constant<int, 0>{});
        if (turn + QW < end)
            block(own + B::STAGE, own, k_tile, v_tile, stats[1][group][0], std::integral_constant<int, 1>{});
    }
    if constexpr (QW == 2) {
        add_groups<DP>(lds, wave, group, dk);
        add_groups<DP>(lds, wave, group, dv);
        if (group > 0) return;
    }
    const int64_t at_row = (s.k0 + key) * a.kv_heads + kv_head;
    if (counts) {
        float *pk = parts > 1 ? a.part + split * 2 * size : nullptr, *pv = pk ? pk + size : nullptr;
        store_column<OUT16, DP>(a.dk, pk, at_row, a.D, dk, a.scale);
        store_column<OUT16, DP>(a.dv, pv, at_row, a.D, dv, 1.f);
    } else if (a.zero_rest && split == 0 && key < s.kv_len && key < first + a.R) {
        zero_row<OUT16>(reinterpret_cast<char *>(a.dk) + at_row * a.D * (OUT16 ? 2 : 4), a.D, h, 2);
        zero_row<OUT16>(reinterpret_cast<char *>(a.dv) + at_row * a.D * (OUT16 ? 2 : 4), a.D, h, 2);
    }
}

// Sums of the parts' values in their order, of kJoinRows rows of a tile: those of a
// sequence, or of its keys that count.
template <bool BF16>
__global__ __launch_bounds__(256) void k_join(Params a, bool by_keys) {
    int first;
    const Sequence s = locate(a.pack, a.R, blockIdx.x, by_keys, first, a.status);
    const int all = by_keys ? s.keys : s.q_len;
    if (!s.real || first >= all) return;
    int rows = all - first < a.R ? all - first : a.R;
    const int splits = parts_of(a.cut, by_keys ? (int64_t)row_blocks(a, s, first) * a.group
                                               : (keys_seen(s, a.pack.causal, first + rows - 1) + kKeyBlock - 1) / kKeyBlock);
    const int skip = (int)blockIdx.y * kJoinRows;
    if (splits == 1 || skip >= rows) return;
    first += skip;
    rows = rows - skip < kJoinRows ? rows - skip : kJoinRows;
    const int64_t width = (int64_t)(by_keys ? a.kv_heads : a.heads) * a.D;
    const int64_t size = (by_keys ? a.pack.kv_rows : a.pack.q_rows) * width;
    const int64_t from = ((by_keys ? s.k0 : s.q0) + first) * width;
    const int64_t step = (by_keys ? 2 : 1) * size, all_values = rows * width;
    // four values a thread, of both tensors by keys; the last ones of a row of odd width alone
    const int vec = width % 4 == 0 ? 4 : 1;
    for (int t = 0; t < (by_keys ? 2 : 1); ++t) {
        void *out = !by_keys ? a.dq : t == 0 ? a.dk : a.dv;
        const float *part = a.part + t * size + from;
        for (int64_t i = ((int64_t)blockIdx.z * 256 + threadIdx.x) * vec; i < all_values; i += (int64_t)256 * vec * gridDim.z) {
            float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int n = 0; n < splits; ++n) {
                float p[4];
                load_row<false, 4>(part + n * step + i, 0, vec, p);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] += p[k];
            }
            store4<BF16>(reinterpret_cast<char *>(out) + (from + i) * (BF16 ? 2 : 4), 0, vec, x);
        }
    }
}

// The two launches of a call, with their joins.
struct Plan {
    Params by_queries, by_keys;
    bool dma_queries, dma_keys, planes;
    int64_t grid_queries, grid_keys, part;  // floats that the larger of the joins needs
};

Plan plan_of(const lattice_dense *D, const AttendArgs &a) {
    Plan r = {};
    Params &p = r.by_queries;
    p.pack = packing_of(a);
    p.q = {a.q, a.q_row, a.q_head};
    p.k = {a.k, a.k_row, a.k_head};
    p.v = {a.v, a.v_row, a.v_head};
    p.o = {a.out, a.o_row, a.o_head};
    p.g = p.g_stored = {a.grad, a.g_row, a.g_head};
    p.dq = a.grad_q;
    p.dk = a.grad_k;
    p.dv = a.grad_v;
    p.lse = a.lse;
    p.heads = a.heads;
    p.kv_heads = a.kv_heads;
    p.D = a.D;
    p.group = a.heads / a.kv_heads;
    p.c = a.scale * kLog2e;
    p.scale = a.scale;
    p.zero_rest = a.zero_rest;
    p.status = D->status;
    r.by_keys = p;
    const int E = a.bf16 ? 2 : 4;
    r.dma_queries = straight(p.k, a.D, E) && straight(p.v, a.D, E);
    r.dma_keys = straight(p.q, a.D, E) && straight(p.g, a.D, E);
    const int64_t sequences = a.sequences > 0 ? a.sequences : 1;
    const int64_t rows = (a.q_rows + sequences - 1) / sequences, keys = (a.kv_rows + sequences - 1) / sequences;
    r.planes = !a.bf16 && planes_pay(a, keys, 1e7);
    {
        const Columns c(p.group, 128);
        p.parts = c.parts;
        p.tile_heads = c.heads;
        p.R = c.R;
        p.units = a.kv_heads * p.parts;
        const int64_t slots = slots_of(a.q_starts, sequences, a.q_rows, p.R), tiles = (a.q_rows + p.R - 1) / p.R;
        p.slots = (int)slots;
        const int64_t grid = unit_grid(p.units, slots), width = a.q_rows * a.heads * a.D;
        p.cut = cut_of(p.units * std::max(tiles, sequences), (keys + kKeyBlock - 1) / kKeyBlock,
                       (a.kv_rows + kKeyBlock - 1) / kKeyBlock, grid, 2 * D->cu_count, 8, kMostParts / (width * 4 + 1));
        if (p.cut.splits > 1) r.part = p.cut.splits * width;
        r.grid_queries = grid;
    }
    Params &b = r.by_keys;
    b.R = 128;
    const int32_t *starts = !a.q_starts ? nullptr : a.kv_starts ? a.kv_starts : a.q_starts;
    const int64_t slots = slots_of(starts, sequences, a.kv_rows, b.R), tiles = (a.kv_rows + b.R - 1) / b.R;
    b.slots = (int)slots;
    // a tile's blocks are the rows of all its query heads
    const int64_t grid = unit_grid(a.kv_heads, slots), width = 2 * a.kv_rows * a.kv_heads * a.D;
    b.cut = cut_of(a.kv_heads * std::max(tiles, sequences), (rows + kRowBlock - 1) / kRowBlock * p.group,
                   (a.q_rows + kRowBlock - 1) / kRowBlock * p.group, grid, D->cu_count, 8, kMostParts / (width * 4 + 1));
    if (b.cut.splits > 1) r.part = std::max(r.part, b.cut.splits * width);
    r.grid_keys = grid;
    return r;
}

template <Type T, int DP, bool DMA>
hipError_t by_queries(lattice_dense *D, const Plan &r) {
    constexpr int LDS = 2 * 2 * tile_bytes<T, DP>(kKeyBlock);
    static_assert(LDS <= 64 * 1024, "LDS");
    return in_launches(r.by_queries, r.grid_queries, [&](dim3 grid, const Params &p) {
        hipLaunchKernelGGL((k_by_queries<T, DP, DMA>), grid, dim3(256), LDS, D->stream, p);
    });
}

template <Type T, int DP, bool DMA>
hipError_t by_keys(lattice_dense *D, const Plan &r) {
    using B = ByKeys<T, DP>;
    constexpr int LDS = B::LDS;
    static std::atomic<uint64_t> done{0};
    if (LDS + 2048 > 64 * 1024) TRY(gemm::allow_lds(reinterpret_cast<const void *>(&k_by_keys<T, DP, DMA>), LDS, done));
    return in_launches(r.by_keys, r.grid_keys, [&](dim3 grid, const Params &p) {
        hipLaunchKernelGGL((k_by_keys<T, DP, DMA>), grid, dim3(B::THREADS), LDS, D->stream, p);
    });
}

template <bool BF16>
hipError_t join(lattice_dense *D, const Params &p, bool keys) {
    if (p.cut.splits == 1) return hipSuccess;
    hipLaunchKernelGGL((k_join<BF16>), join_grid(p.slots, p.R, ((int64_t)kJoinRows * (keys ? p.kv_heads : p.heads) * p.D + 1023) / 1024),
                       dim3(256), 0, D->stream, p, keys);
    return hipGetLastError();
}

template <Type T, int DP>
hipError_t launch_dim(lattice_dense *D, const Plan &r) {
    if (r.by_queries.pack.q_rows > 0) {
        if constexpr (T == PLANES)
            TRY((by_queries<T, DP, true>(D, r)));
        else
            TRY(r.dma_queries ? (by_queries<T, DP, true>(D, r)) : (by_queries<T, DP, false>(D, r)));
        TRY(join<T == BF16>(D, r.by_queries, false));
    }
    if (r.by_queries.pack.kv_rows > 0) {
        if constexpr (T == PLANES)
            TRY((by_keys<T, DP, true>(D, r)));
        else
            TRY(r.dma_keys ? (by_keys<T, DP, true>(D, r)) : (by_keys<T, DP, false>(D, r)));
        TRY(join<T == BF16>(D, r.by_keys, true));
    }
    return hipSuccess;
}

template <Type T>
hipError_t launch_type(lattice_dense *D, const Plan &r) {
    const int dp = padded_dim(r.by_queries.D);
    if (dp == 32) return launch_dim<T, 32>(D, r);
    if constexpr (T != PLANES)
        if (dp == 128) return launch_dim<T, 128>(D, r);
    return launch_dim<T, 64>(D, r);
}

}  // namespace

int64_t attention_backward_scratch(const lattice_dense *D, const AttendArgs &a) {
    const Plan r = plan_of(D, a);
    ScratchLayout s;
    s.take(a.q_rows * a.heads * 4);
    s.take(r.part * 4);
    if (r.planes) {
        const int dp = padded_dim(a.D);
        s.take(2 * plane_bytes(a.q_rows, a.heads, dp));
        s.take(2 * plane_bytes(a.kv_rows, a.kv_heads, dp));
    }
    return s.bytes;
}

bool attention_backward_fits(const lattice_dense *D, const AttendArgs &a) {
    const Plan r = plan_of(D, a);
    return r.grid_queries < ((int64_t)1 << 31) && r.grid_keys < ((int64_t)1 << 31);
}

hipError_t launch_attention_backward(lattice_dense *D, const AttendArgs &a) {
    Plan r = plan_of(D, a);
    ScratchLayout s;
    char *ws = static_cast<char *>(D->ws);
    r.by_queries.delta = r.by_keys.delta = reinterpret_cast<float *>(ws + s.take(a.q_rows * a.heads * 4));
    r.by_queries.part = r.by_keys.part = reinterpret_cast<float *>(ws + s.take(r.part * 4));
    if (a.bf16) return launch_type<BF16>(D, r);
    if (!r.planes) return launch_type<F32>(D, r);
    Params &p = r.by_queries;
    const int dp = padded_dim(a.D);
    const int64_t q = plane_bytes(a.q_rows, a.heads, dp), kv = plane_bytes(a.kv_rows, a.kv_heads, dp);
    char *at_q = ws + s.take(2 * q), *at_kv = ws + s.take(2 * kv);
    PlaneJobs jobs = {};
    add_planes(jobs, 0, p.q, a.q_rows, a.heads, dp, at_q);
    add_planes(jobs, 1, p.g, a.q_rows, a.heads, dp, at_q + q);
    add_planes(jobs, 2, p.k, a.kv_rows, a.kv_heads, dp, at_kv);
    add_planes(jobs, 3, p.v, a.kv_rows, a.kv_heads, dp, at_kv + kv);
    TRY(launch_planes(D, jobs, 4, a.D, dp));
    Params &b = r.by_keys;
    b.q = p.q, b.g = p.g, b.k = p.k, b.v = p.v;
    return launch_type<PLANES>(D, r);
}
