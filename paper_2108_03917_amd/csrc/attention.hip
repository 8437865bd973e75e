// Softmax attention, forward:  o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i),
// s_ij = scale q_i . k_j.
//
// A tile is a number of columns, each one row of one query head; the heads that
// share a key head lie next to each other, so that a tile's keys and values are
// read once for all of them.  The keys of its sequence go by in blocks, and a
// column's maximum, sum and output are kept in registers (the output rescaled only when
// the maximum has grown by more than 2^8, which the last division makes good).
//
// Many rows: four wavefronts have 32 or 64 columns each, and share blocks of keys in
// LDS that are loaded one ahead.  Few rows (single tokens against a cache): one
// tile of 32 columns, whose keys the wavefronts of a workgroup take in turns,
// each with blocks of its own, so that they never wait for each other; their
// results are joined in LDS.
// Tiles with more blocks of keys than others, or too few of them for the CUs, are cut
// into parts, whose results a second launch joins in a fixed order.
//
// Many rows are bound by the matrix cores, then by the exponentials and conversions
// beside them: 16384 rows of 16 (4) heads of 128, causal, bf16, take 1.01 to 1.23 ms from
// card to card (1.09 to 0.9 PFLOP/s; a large product reaches 1.6).  32 columns a wavefront
// there, since 64 leave one wavefront a SIMD.  Few rows are bound by the bytes of the keys and values:
// 48 tokens against caches of 8192 x 8 heads of 128, bf16, 190 us and 8 for the parts
// (5.0 TB/s; a large copy 5.6).  A token against 77 keys takes 6.0 us.
//
// Vector registers that do not fit: k_attend<BF16, 64, 2> keeps 8 in memory (21 without direct loads),
// k_attend<PLANES, 64, 1> 2; no other instance has any.
#include "attention.h"

namespace {

using namespace attend;

struct Params {
    Packing pack;
    View q, k, v, o;
    float *lse;         // [heads][rows], or null
    int heads, units;   // units: (key head, part of its query heads)
    int D;
    int group;          // query heads of a key head
    int parts, tile_heads;  // parts that a group is cut into, query heads of one
    int R, slots;           // rows of a tile
    int64_t block0;         // of the launch's workgroups, among all of them
    Cut cut;                // of blocks of keys
    float c;            // scale, for powers of 2
    bool zero_rest;
    float *part_o;      // of the parts: [splits][rows][heads][D]
    float2 *part_stats; // [splits][heads][rows]: maximum and sum (an lse would round what sets the parts' weights)
    int32_t *status;
};

// One workgroup's tile.
struct Tile {
    Sequence s;
    int first, rows;      // its rows of the sequence
    int head0, heads;     // its query heads
    int kv_head, split, parts;
    int t0, t1;           // blocks of keys of this split
    int least, most;      // keys that its first and its last row see
};

// The workgroup's tile; false where there is nothing to compute (then rows of no
// sequence, or without keys, have been seen to).
template <Type T, int KT>
__device__ __forceinline__ bool tile_of(const Params &a, Tile &t) {
    int unit, slot;
    t.split = blockIdx.y;
    if (!unit_of(a.block0 + blockIdx.x, a.units, a.slots, true, unit, slot)) return false;
    const int part = unit % a.parts;
    t.kv_head = unit / a.parts;
    t.head0 = t.kv_head * a.group + part * a.tile_heads;
    const int left = a.group - part * a.tile_heads;
    t.heads = left < a.tile_heads ? left : a.tile_heads;
    t.s = locate(a.pack, a.R, slot, false, t.first, a.status);
    if (t.first >= t.s.q_len || t.heads <= 0) return false;
    t.rows = t.s.q_len - t.first < a.R ? t.s.q_len - t.first : a.R;
    if (!t.s.real) {
        if (t.split == 0 && a.zero_rest)
            for (int r = 0; r < t.rows; ++r)
                for (int h = 0; h < t.heads; ++h) {
                    const int64_t row = t.s.q0 + t.first + r;
                    const int head = t.head0 + h;
                    zero_row<T == BF16>(const_cast<char *>(reinterpret_cast<const char *>(a.o.p)) +
                                       (row * a.o.row + head * a.o.head) * (T == BF16 ? 2 : 4),
                                   a.D, threadIdx.x, blockDim.x);
                    if (a.lse && threadIdx.x == 0) a.lse[head * a.pack.q_rows + row] = -INFINITY;
                }
        return false;
    }
    t.least = keys_seen(t.s, a.pack.causal, t.first);
    t.most = keys_seen(t.s, a.pack.causal, t.first + t.rows - 1);
    const int n = (t.most + KT - 1) / KT;
    t.parts = parts_of(a.cut, n);
    t.t0 = (int)((int64_t)n * t.split / t.parts);
    t.t1 = (int)((int64_t)n * (t.split + 1) / t.parts);
    return t.split < t.parts;
}

// A column's state: its maximum (of the scores as they are), the sum of
// this lane's share of the exponentials, and the output's channels.  A maximum passes by what
// is no number, a sum does not: a column has seen no key (or ones that score -inf alone) where its
// maximum is -inf and its sum is 0, and where the latter is none, the result is none.
template <int DP>
struct Column {
    float top = -INFINITY, sum = 0.f;
    f32x16_t o[DP / 32];
};

// Scores (for powers of 2) that c times themselves rounds by 1/2 at most.
constexpr float kLargeScore = 0x1p24f;

// Take in a block of KB x 32 scores of a column.
template <Type T, int DP, int KB>
__device__ __forceinline__ void softmax(f32x16_t (&s)[KB], Column<DP> &col, float c, Right<T> (&p)[KB]) {
    float m = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, s[b][e]);
    m = fmaxf(pair_max(m), col.top);
    // grown too far: (m - top) c > 8; a first maximum always (top is -inf)
    if (__any((m - col.top) * c > 8.f)) {
        const float f = m == -INFINITY ? 1.f : exp2_((col.top - m) * c);
        col.top = m;
        col.sum *= f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) col.o[d][e] *= f;
    }
    float mc = col.top == -INFINITY ? 0.f : col.top * c;
    // c times a large score is off by more than an exponential bears: the difference first
    const bool large = fabsf(mc) > kLargeScore;
    if (__any(large)) {
        seldom();
        const float base = large ? col.top : 0.f;
        mc = large ? 0.f : mc;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[b][e] -= base;
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[b][e] = exp2_(fmaf(s[b][e], c, -mc));
            col.sum += s[b][e];
        }
        p[b].set(s[b]);
    }
}

// Write a column: 4 channels at a time, by f.
template <Type T, int DP>
__device__ __forceinline__ void finish(const Params &a, const Tile &t, int64_t row, int head, Column<DP> &col) {
    const float sum = pair_sum(col.sum);
    const bool none = col.top == -INFINITY && sum == 0.f;
    const float f = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : fmaf(col.top, a.c, 0.f) + log2f(sum);
    const int h = (threadIdx.x & 63) >> 5;
    const bool part = t.parts > 1;
    if (h == 0) {
        if (part)
            a.part_stats[((int64_t)t.split * a.heads + head) * a.pack.q_rows + row] = make_float2(col.top, sum);
        else if (a.lse)
            a.lse[head * a.pack.q_rows + row] = lse2 * kLn2;
    }
    char *o = const_cast<char *>(reinterpret_cast<const char *>(a.o.p)) + (row * a.o.row + head * a.o.head) * (T == BF16 ? 2 : 4);
    float *po = a.part_o + (((int64_t)t.split * a.pack.q_rows + row) * a.heads + head) * a.D;
    if (part && none) return;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c0 = 32 * d + 8 * g + 4 * h;
            if (c0 >= a.D) continue;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = none ? 0.f : col.o[d][4 * g + i] * f;
            if (part)
                store4<false>(po, c0, a.D, v);
            else
                store4<T == BF16>(o, c0, a.D, v);
        }
}

// Many rows: 4 wavefronts x NQ blocks of 32 columns.  Keys of a block:
template <Type T>
constexpr int keys_of_block() { return T == F32 ? 32 : 64; }

template <Type T, int DP, int NQ, bool DMA>
__global__ __launch_bounds__(256, T != F32 || NQ * DP <= 64 ? 2 : 1) void k_attend(Params a) {
    using L = RowsOf<T, DP>;
    constexpr int KT = keys_of_block<T>(), KB = KT / 32;
    constexpr int HALF = tile_bytes<T, DP>(KT), STAGE = 2 * HALF;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Tile t;
    if (!tile_of<T, KT>(a, t)) return;
    const int lane = threadIdx.x & 63, wave = gemm::wave_index();

    int seen[NQ];
    int64_t row[NQ];
    int head[NQ];
    bool mine[NQ];
    Fragments<T, DP> q[NQ];
    const int D = T == PLANES ? DP : a.D;  // as the operands are laid out
    Column<DP> col[NQ];
    int wave_most = 0;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int c = (wave * NQ + n) * 32 + (lane & 31);
        int r = c / t.heads;
        const int h = c - r * t.heads;
        mine[n] = r < t.rows;
        r = mine[n] ? r : t.rows - 1;
        row[n] = t.s.q0 + t.first + r;
        head[n] = t.head0 + h;
        seen[n] = keys_seen(t.s, a.pack.causal, t.first + r);
        int last = ((wave * NQ + n) * 32 + 31) / t.heads;
        last = last < t.rows ? last : t.rows - 1;
        wave_most = uniform(keys_seen(t.s, a.pack.causal, t.first + last));
        load_fragments<T, DP>(a.q, row[n], head[n], D, q[n]);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) clear(col[n].o[d]);
    }

    Loader<T, DP, KT, 4, DMA> lk(a.k, t.s.k0, t.kv_head, D, wave), lv(a.v, t.s.k0, t.kv_head, D, wave);
    if (t.t0 < t.t1) {
        lk.fetch(lds, t.t0 * KT, t.s.keys);
        lv.fetch(lds + HALF, t.t0 * KT, t.s.keys);
        lk.commit(lds);
        lv.commit(lds + HALF);
    }
    // the stage is a constant, so that addresses in LDS are
    // (and the two stages' addresses are told to be apart: reads of one need not wait for
    // what is on its way to the other)
    auto block = [&](int i, const char *__restrict now, char *__restrict next) {
        gemm::wait_and_barrier<0>();
        const bool more = i + 1 < t.t1;
        if (more) {
            lk.fetch(next, (i + 1) * KT, t.s.keys);
            lv.fetch(next + HALF, (i + 1) * KT, t.s.keys);
        }
        if (i * KT < wave_most) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                f32x16_t s[KB];
                gemm::sched_barrier();
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    clear(s[b]);
                    rows_times<T, DP, KT>(now, 32 * b, q[n], s[b]);
                }
                if (T != F32) read_ahead<kProducts<T> * KB * L::STEPS, kPlanes<T> * KB * L::STEPS, 6>();
                gemm::sched_barrier();
                if ((i + 1) * KT > t.least) {
                    seldom();
#pragma unroll
                    for (int b = 0; b < KB; ++b) mask(s[b], i * KT + 32 * b, seen[n]);
                }
                Right<T> p[KB];
                softmax<T, DP, KB>(s, col[n], a.c, p);
#pragma unroll
                for (int b = 0; b < KB; ++b) columns_times<T, DP, KT>(now + HALF, 32 * b, p[b], col[n].o);
            }
        }
        if (more) {
            lk.commit(next);
            lv.commit(next + HALF);
        }
    };
    for (int i = t.t0; i < t.t1; i += 2) {
        block(i, lds, lds + STAGE);
        if (i + 1 < t.t1) block(i + 1, lds + STAGE, lds);
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n)  // a column's two lanes go the same way
        if (mine[n]) finish<T, DP>(a, t, row[n], head[n], col[n]);
}

// Few rows: one tile of 32 columns, WAVES wavefronts with their own keys.
template <Type T, int DP>
constexpr int few_waves() { return RowsOf<T, DP>::BYTES <= 256 ? 4 : 2; }

template <Type T, int DP, bool DMA>
__global__ __launch_bounds__((64 * few_waves<T, DP>())) void k_attend_few(Params a) {
    using L = RowsOf<T, DP>;
    constexpr int KT = 32, WAVES = few_waves<T, DP>();
    constexpr int HALF = KT * L::BYTES, STAGE = 2 * HALF;
    constexpr int LOADS = 2 * KT * L::CHUNKS / 64;
    constexpr int PITCH = DP + 4;  // floats of a column's output in LDS
    static_assert(32 * PITCH * 4 <= 2 * STAGE && LOADS < 64, "LDS");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float tops[WAVES][32], sums[WAVES][32];
    Tile t;
    if (!tile_of<T, KT>(a, t)) return;
    const int lane = threadIdx.x & 63, wave = gemm::wave_index();
    char *own = lds + wave * 2 * STAGE;

    const int c = lane & 31;
    int r = c / t.heads;
    const int h = c - r * t.heads;
    r = r < t.rows ? r : t.rows - 1;
    const int seen = keys_seen(t.s, a.pack.causal, t.first + r);
    Fragments<T, DP> q;
    Column<DP> col;
    load_fragments<T, DP>(a.q, t.s.q0 + t.first + r, t.head0 + h, a.D, q);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) clear(col.o[d]);

    Loader<T, DP, KT, 1, DMA> lk(a.k, t.s.k0, t.kv_head, a.D, 0), lv(a.v, t.s.k0, t.kv_head, a.D, 0);
    int i = t.t0 + wave;
    if (i < t.t1) {
        lk.fetch(own, i * KT, t.s.keys);
        lv.fetch(own + HALF, i * KT, t.s.keys);
        lk.commit(own);
        lv.commit(own + HALF);
    }
    auto block = [&](const char *__restrict now, char *__restrict next) {
        const bool more = i + WAVES < t.t1;
        // what lay in `next` has been read
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) {
            lk.fetch(next, (i + WAVES) * KT, t.s.keys);
            lv.fetch(next + HALF, (i + WAVES) * KT, t.s.keys);
        }
        if (DMA) {
            if (more)
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        f32x16_t s[1];
        gemm::sched_barrier();
        clear(s[0]);
        rows_times<T, DP, KT>(now, 0, q, s[0]);
        if (T != F32) read_ahead<L::STEPS, L::STEPS, 8>();
        gemm::sched_barrier();
        if ((i + 1) * KT > t.least) {
            seldom();
            mask(s[0], i * KT, seen);
        }
        Right<T> p[1];
        softmax<T, DP, 1>(s, col, a.c, p);
        columns_times<T, DP, KT>(now + HALF, 0, p[0], col.o);
        if (more) {
            lk.commit(next);
            lv.commit(next + HALF);
        }
        i += WAVES;
    };
    for (int stage = 0; i < t.t1; stage ^= 1) block(own + stage * STAGE, own + (stage ^ 1) * STAGE);
    // join: every wavefront's columns to LDS (its own part, whose blocks are done with)
    const float sum = pair_sum(col.sum);
    const int half = lane >> 5;
    float *out = reinterpret_cast<float *>(own) + c * PITCH;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4 *>(out + 32 * d + 8 * g + 4 * half) =
                make_float4(col.o[d][4 * g], col.o[d][4 * g + 1], col.o[d][4 * g + 2], col.o[d][4 * g + 3]);
    if (half == 0) {
        tops[wave][c] = col.top;
        sums[wave][c] = sum;
    }
    __syncthreads();
    const int columns = t.rows * t.heads;
    for (int id = threadIdx.x; id < columns * (DP / 4); id += 64 * WAVES) {
        const int cc = id / (DP / 4), c0 = id % (DP / 4) * 4;
        float m = tops[0][cc];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, tops[w][cc]);
        float all = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (tops[w][cc] == -INFINITY && sums[w][cc] == 0.f) continue;
            const float f = exp2_((tops[w][cc] - m) * a.c);
            all += f * sums[w][cc];
            const float *x = reinterpret_cast<const float *>(lds + w * 2 * STAGE) + cc * PITCH + c0;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += f * x[k];
        }
        const bool none = m == -INFINITY && all == 0.f;
        const float inv = none ? 0.f : 1.f / all;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = none ? 0.f : v[k] * inv;
        const int rr = cc / t.heads, hh = t.head0 + cc - rr * t.heads;
        const int64_t row = t.s.q0 + t.first + rr;
        if (c0 == 0) {
            const float lse2 = none ? -INFINITY : m * a.c + log2f(all);
            if (t.parts > 1)
                a.part_stats[((int64_t)t.split * a.heads + hh) * a.pack.q_rows + row] = make_float2(m, all);
            else if (a.lse)
                a.lse[hh * a.pack.q_rows + row] = lse2 * kLn2;
        }
        if (c0 >= a.D) continue;
        if (t.parts > 1) {
            if (!none) store4<false>(a.part_o + (((int64_t)t.split * a.pack.q_rows + row) * a.heads + hh) * a.D, c0, a.D, v);
        } else {
            store4<T == BF16>(const_cast<char *>(reinterpret_cast<const char *>(a.o.p)) + (row * a.o.row + hh * a.o.head) * L::E,
                         c0, a.D, v);
        }
    }
}

// A part's sum as it is under the parts' common maximum.
__device__ __forceinline__ float weight(float2 stat, float m, float c) {
    return stat.x == -INFINITY && stat.y == 0.f ? 0.f : exp2_((stat.x - m) * c) * stat.y;
}

// The parts' results of kJoinRows rows of a tile (blocks of KT keys), weighted so.
template <bool BF16>
__global__ __launch_bounds__(256) void k_join(Params a, int KT) {
    int first;
    const Sequence s = locate(a.pack, a.R, blockIdx.x, false, first, a.status);
    if (!s.real || first >= s.q_len) return;
    int rows = s.q_len - first < a.R ? s.q_len - first : a.R;
    const int splits = parts_of(a.cut, (keys_seen(s, a.pack.causal, first + rows - 1) + KT - 1) / KT);
    const int skip = (int)blockIdx.y * kJoinRows;
    if (splits == 1 || skip >= rows) return;
    first += skip;
    rows = rows - skip < kJoinRows ? rows - skip : kJoinRows;
    const int64_t next = a.pack.q_rows * a.heads;
    const int lanes = (a.D + 3) / 4, pairs = rows * a.heads;  // of a head's row; rows' heads
    __shared__ float2 stats[kJoinPairs][kMostSplits];
    for (int base = (int)blockIdx.z * kJoinPairs; base < pairs; base += kJoinPairs * gridDim.z) {
        const int here = pairs - base < kJoinPairs ? pairs - base : kJoinPairs;
        __syncthreads();
        for (int id = threadIdx.x; id < here * splits; id += 256) {
            const int n = id / here, i = base + id - n * here;
            stats[id - n * here][n] = a.part_stats[n * next + (i % a.heads) * a.pack.q_rows + s.q0 + first + i / a.heads];
        }
        __syncthreads();
        for (int id = threadIdx.x; id < here * lanes; id += 256) {
            const int pair = id / lanes, i = base + pair, c0 = (id - pair * lanes) * 4;
            const int64_t row = s.q0 + first + i / a.heads;
            const int head = i % a.heads;
            const float2 *stat = stats[pair];
            float m = -INFINITY, sum = 0.f;
            for (int n = 0; n < splits; ++n) m = fmaxf(m, stat[n].x);
            for (int n = 0; n < splits; ++n) sum += weight(stat[n], m, a.c);
            const bool nothing = m == -INFINITY && sum == 0.f;
            if (a.lse && c0 == 0) a.lse[head * a.pack.q_rows + row] = nothing ? -INFINITY : (m * a.c + log2f(sum)) * kLn2;
            const float inv = nothing ? 0.f : 1.f / sum;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            const float *p = a.part_o + (row * a.heads + head) * a.D;
#pragma unroll 4
            for (int n = 0; n < splits; ++n) {
                // a part without keys has written nothing
                const bool none = stat[n].x == -INFINITY && stat[n].y == 0.f;
                const float f = weight(stat[n], m, a.c) * inv;
                float x[4];
                load_row<false, 4>(p + n * next * a.D, c0, a.D, x);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += none ? 0.f : f * x[k];
            }
            store4<BF16>(const_cast<char *>(reinterpret_cast<const char *>(a.o.p)) +
                             (row * a.o.row + head * a.o.head) * (BF16 ? 2 : 4),
                         c0, a.D, v);
        }
    }
}

// What a call does.
struct Plan {
    Params p;
    bool few, dma, planes;
    int nq, KT;  // blocks of 32 columns of a wavefront, keys of a block
    int64_t grid, part_o, part_stats;  // grid.x; values of scratch
};

Plan plan_of(const lattice_dense *D, const AttendArgs &a) {
    Plan r = {};
    Params &p = r.p;
    p.pack = packing_of(a);
    p.q = {a.q, a.q_row, a.q_head};
    p.k = {a.k, a.k_row, a.k_head};
    p.v = {a.v, a.v_row, a.v_head};
    p.o = {a.out, a.o_row, a.o_head};
    p.lse = a.lse;
    p.heads = a.heads;
    p.D = a.D;
    p.group = a.heads / a.kv_heads;
    p.c = a.scale * kLog2e;
    p.zero_rest = a.zero_rest;
    p.status = D->status;
    const int E = a.bf16 ? 2 : 4;
    r.dma = straight(p.k, a.D, E) && straight(p.v, a.D, E);
    const int64_t sequences = a.sequences > 0 ? a.sequences : 1;
    const int64_t rows = (a.q_rows + sequences - 1) / sequences, keys = (a.kv_rows + sequences - 1) / sequences;
    // One tile's columns hold a sequence's rows and heads, and its keys are many: a token of 16
    // sequences of 2000 keys 28 us (many rows' tiles 35), of 64 of 4096 keys, 64 columns, 113
    // (120); 200 sequences of 20 rows and keys 16 (12).
    r.few = rows * p.group <= 32 && keys >= 4 * rows;
    r.planes = !a.bf16 && !r.few && planes_pay(a, keys, 1e8);
    // 64 columns a wavefront halve the reads of LDS, but also the workgroups (8 heads of 64 in bf16:
    // 16384 rows 623 us, 648 with 32; 4096 rows 99 and 75); registers of three planes hold 32
    // channels so
    r.nq = !r.few && a.D <= (r.planes ? 32 : 64) && a.q_rows * a.heads >= (int64_t)256 * 2 * D->cu_count ? 2 : 1;
    const Columns c(p.group, r.few ? 32 : 128 * r.nq);
    p.parts = c.parts;
    p.tile_heads = c.heads;
    p.R = c.R;
    p.units = a.kv_heads * p.parts;
    const int64_t slots = slots_of(a.q_starts, sequences, a.q_rows, p.R);
    p.slots = (int)slots;
    r.grid = unit_grid(p.units, slots);
    r.KT = r.few ? 32 : a.bf16 || r.planes ? keys_of_block<BF16>() : keys_of_block<F32>();
    const int64_t tiles = (a.q_rows + p.R - 1) / p.R, width = (int64_t)a.q_rows * a.heads * a.D;
    p.cut = cut_of(p.units * (tiles > sequences ? tiles : sequences), (keys + r.KT - 1) / r.KT, (a.kv_rows + r.KT - 1) / r.KT,
                   r.grid, r.few ? D->cu_count : 2 * D->cu_count, r.few ? 8 : 4, kMostParts / (width * 4 + 1));
    if (p.cut.splits > 1) {
        r.part_o = p.cut.splits * width;
        r.part_stats = (int64_t)p.cut.splits * a.q_rows * a.heads;
    }
    return r;
}

template <Type T, int DP, int NQ, bool DMA>
hipError_t launch_many(lattice_dense *D, const Plan &r) {
    constexpr int LDS = 2 * 2 * tile_bytes<T, DP>(keys_of_block<T>());
    static std::atomic<uint64_t> done{0};
    if (LDS > 64 * 1024) TRY(gemm::allow_lds(reinterpret_cast<const void *>(&k_attend<T, DP, NQ, DMA>), LDS, done));
    return in_launches(r.p, r.grid, [&](dim3 grid, const Params &p) {
        hipLaunchKernelGGL((k_attend<T, DP, NQ, DMA>), grid, dim3(256), LDS, D->stream, p);
    });
}

template <Type T, int DP, bool DMA>
hipError_t launch_as(lattice_dense *D, const Plan &r) {
    if constexpr (T != PLANES)
        if (r.few) {
            constexpr int W = few_waves<T, DP>(), LDS = W * 2 * 2 * 32 * RowsOf<T, DP>::BYTES;
            static std::atomic<uint64_t> done{0};
            if (LDS + 1024 > 64 * 1024) TRY(gemm::allow_lds(reinterpret_cast<const void *>(&k_attend_few<T, DP, DMA>), LDS, done));
            return in_launches(r.p, r.grid, [&](dim3 grid, const Params &p) {
                hipLaunchKernelGGL((k_attend_few<T, DP, DMA>), grid, dim3(64 * W), LDS, D->stream, p);
            });
        }
    if constexpr (DP <= 64 && (T != PLANES || DP == 32))
        if (r.nq == 2) return launch_many<T, DP, 2, DMA>(D, r);
    return launch_many<T, DP, 1, DMA>(D, r);
}

template <Type T, int DP>
hipError_t launch_dim(lattice_dense *D, const Plan &r) {
    if constexpr (T != PLANES)
        if (!r.dma) return launch_as<T, DP, false>(D, r);
    return launch_as<T, DP, true>(D, r);
}

template <Type T>
hipError_t launch_type(lattice_dense *D, const Plan &r) {
    const int dp = padded_dim(r.p.D);
    if (dp == 32) {
        TRY((launch_dim<T, 32>(D, r)));
    } else if (dp == 64) {
        TRY((launch_dim<T, 64>(D, r)));
    } else if constexpr (T != PLANES) {
        TRY((launch_dim<T, 128>(D, r)));
    }
    if (r.p.cut.splits == 1) return hipSuccess;
    hipLaunchKernelGGL((k_join<T == BF16>), join_grid(r.p.slots, r.p.R, (kJoinRows * r.p.heads + kJoinPairs - 1) / kJoinPairs),
                       dim3(256), 0, D->stream, r.p, r.KT);
    return hipGetLastError();
}

}  // namespace

int64_t attention_scratch(const lattice_dense *D, const AttendArgs &a) {
    const Plan r = plan_of(D, a);
    ScratchLayout s;
    s.take(r.part_o * 4);
    s.take(r.part_stats * 8);
    if (r.planes) {
        const int dp = padded_dim(a.D);
        s.take(plane_bytes(a.q_rows, a.heads, dp));
        s.take(2 * plane_bytes(a.kv_rows, a.kv_heads, dp));
    }
    return s.bytes;
}

bool attention_fits(const lattice_dense *D, const AttendArgs &a) {
    return plan_of(D, a).grid < ((int64_t)1 << 31);
}

hipError_t launch_attention(lattice_dense *D, const AttendArgs &a) {
    Plan r = plan_of(D, a);
    ScratchLayout s;
    char *ws = static_cast<char *>(D->ws);
    r.p.part_o = reinterpret_cast<float *>(ws + s.take(r.part_o * 4));
    r.p.part_stats = reinterpret_cast<float2 *>(ws + s.take(r.part_stats * 8));
    if (a.bf16) return launch_type<BF16>(D, r);
    if (!r.planes) return launch_type<F32>(D, r);
    const int dp = padded_dim(a.D);
    const int64_t kv = plane_bytes(a.kv_rows, a.kv_heads, dp);
    PlaneJobs jobs = {};
    add_planes(jobs, 0, r.p.q, a.q_rows, a.heads, dp, ws + s.take(plane_bytes(a.q_rows, a.heads, dp)));
    char *at = ws + s.take(2 * kv);
    add_planes(jobs, 1, r.p.k, a.kv_rows, a.kv_heads, dp, at);
    add_planes(jobs, 2, r.p.v, a.kv_rows, a.kv_heads, dp, at + kv);
    TRY(launch_planes(D, jobs, 3, a.D, dp));
    return launch_type<PLANES>(D, r);
}
