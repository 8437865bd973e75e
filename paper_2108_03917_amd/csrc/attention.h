// Softmax attention over packed sequences: what the forward pass (attention.hip)
// and the backward pass (attention_bwd.hip) share.
//
//   s_ij = scale q_i . k_j  for the keys j that row i may see,
//   p_ij = exp(s_ij - lse_i),  lse_i = log sum_j exp s_ij,  o_i = sum_j p_ij v_j.
//
// Products run on the matrix cores in 32 x 32 blocks, v_mfma_f32_32x32x16_bf16
// for bf16 and v_mfma_f32_32x32x2_f32 for fp32 storage, or, where there are many of
// fp32 heads of up to 64 channels, the bf16 ones on three planes of bf16 whose sum
// is the value (24 bits): of the nine products the six largest, 2.7 times the rate
// of the fp32 cores.  An accumulator holds a block transposed to what the next product wants as its right operand: lane l
// has column l % 32 and rows 8 (e / 4) + 4 (l / 32) + e % 4 of it.  Scores are
// made as k q^T, so that a query's scores lie in the registers of two lanes
// (maxima and sums need one exchange between them) and the probabilities are,
// without a move, the right operand of v^T p^T: the order of the contraction's
// index is free as long as the left operand has the same one.  The left one, 4
// keys next to each other for each channel, comes out of LDS by the transposing
// read (ds_read_b64_tr_b16) for bf16 and lane by lane for fp32.
#pragma once

#include <algorithm>

#include "dense.h"
#include "gemm.h"

namespace attend {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
using gemm::bf16x8_t;
using gemm::f32x16_t;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kJoinRows = 4;     // of a workgroup that joins parts
constexpr int kJoinPairs = 16;   // of rows and heads that it takes at a time
constexpr int kMostSplits = 64;

// How a kernel takes its operands: fp32 words, bf16, or fp32 as three planes of bf16.
enum Type { F32, BF16, PLANES };
template <Type T>
constexpr int kPlanes = T == PLANES ? 3 : 1;
template <Type T>
constexpr int kProducts = T == PLANES ? 6 : 1;   // of planes

// A tensor [rows][heads][D]: values between rows and between heads, bytes between
// planes.
struct View {
    const void *p;
    int64_t row, head, plane;
};

// Where the rows of packed sequences lie, and the tiles that a launch cuts the
// rows of one side into.
struct Packing {
    int64_t q_rows, kv_rows;
    const int32_t *q_starts, *kv_starts, *kv_lengths;  // device, or null
    int sequences;
    bool causal;
};

// One sequence as the kernels see it.
struct Sequence {
    int64_t q0, k0;  // its first rows
    int q_len, keys, kv_len;  // kv_len: rows of keys, of which `keys` count
    bool real;       // otherwise rows of no sequence
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// The same for an address (otherwise each direct load becomes a loop over the lanes'
// descriptors).
__device__ __forceinline__ const char *uniform(const char *p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return reinterpret_cast<const char *>((uint64_t)hi << 32 | lo);
}

// Rows are cut into tiles of R that lie in one sequence each.  Sequence i of a
// list of starts s_0 = 0 <= s_1 <= .. gets the slots from s_i / R + i on: at
// least as many as it has tiles, and no sum over the sequences before it is
// needed to find them.  The list is the caller's with the rows before its first
// and behind its last start as sequences of their own; `find` returns the place
// in it of the slot's sequence, searching 64 places at a time.
__device__ __forceinline__ int clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ int start_of(const int32_t *starts, int sequences, int rows, int i) {
    if (i <= 0) return 0;
    if (i >= sequences + 2) return rows;
    return clamp(starts[i - 1], 0, rows);
}
__device__ __forceinline__ bool begins_by(int start, int i, int R, int slot) {
    return (int64_t)((uint32_t)start / (uint32_t)R) + i <= slot;
}
__device__ __forceinline__ int find(const int32_t *starts, int sequences, int rows, int R, int slot) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = sequences + 2;
    while (len > 1) {
        const int step = (len + 63) >> 6, i = lane * step;
        const bool here = i < len && begins_by(start_of(starts, sequences, rows, lo + i), lo + i, R, slot);
        int n = __popcll(__ballot(here));
        n = n < 1 ? 1 : n;
        const int skip = (n - 1) * step;
        lo += skip;
        len = len - skip < step ? len - skip : step;
    }
    return uniform(lo);
}

// The sequence of a slot, and the slot's first row in it (>= its length: none).
// `by_keys`: the slots are tiles of the keys' rows.  Starts that go back or lie
// outside the rows are clamped, and noted in *status.
//
// Up to 61 sequences are loaded in one go, a start a lane, and what belongs to the
// slot's is taken from the lanes, in place of a search, its ends and the other
// side's starts one after another (a token against 77 keys: 6.7 to 6.3 us).
__device__ __forceinline__ Sequence locate(const Packing &p, int R, int slot, bool by_keys, int &first, int32_t *status) {
    Sequence s;
    const int32_t *ks = p.kv_starts ? p.kv_starts : p.q_starts;
    const int q_rows = (int)p.q_rows, kv_rows = (int)p.kv_rows, lane = threadIdx.x & 63;
    s.real = true;
    if (!p.q_starts) {
        s.q0 = s.k0 = 0;
        s.q_len = q_rows;
        s.keys = s.kv_len = kv_rows;
        if (p.kv_lengths) s.keys = uniform(p.kv_lengths[0]);
        first = slot * R;
    } else {
        const int32_t *starts = by_keys ? ks : p.q_starts;
        const int rows = by_keys ? kv_rows : q_rows;
        int i, from, to, q_a, q_b, k_a, k_b, keys = 0;
        if (p.sequences <= 61) {
            const bool real = lane <= p.sequences;
            const int q = real ? p.q_starts[lane] : 0, k = real ? ks[lane] : 0;
            const int n = p.kv_lengths && lane < p.sequences ? p.kv_lengths[lane] : 0;
            // place i of the list is the start before it
            const int here = __shfl_up(by_keys ? k : q, 1);
            const int start = lane == 0 ? 0 : lane >= p.sequences + 2 ? rows : clamp(here, 0, rows);
            const uint64_t before = __ballot(lane < p.sequences + 2 && begins_by(start, lane, R, slot));
            i = __popcll(before) - 1;
            i = i < 0 ? 0 : i;
            from = __builtin_amdgcn_readlane(start, i);
            to = __builtin_amdgcn_readlane(start, i + 1);
            const int b = i > 0 ? i - 1 : 0;
            q_a = __builtin_amdgcn_readlane(q, b), q_b = __builtin_amdgcn_readlane(q, b + 1);
            k_a = __builtin_amdgcn_readlane(k, b), k_b = __builtin_amdgcn_readlane(k, b + 1);
            keys = __builtin_amdgcn_readlane(n, b);
        } else {
            i = find(starts, p.sequences, rows, R, slot);
            from = start_of(starts, p.sequences, rows, i);
            to = start_of(starts, p.sequences, rows, i + 1);
            const int b = i > 0 && i <= p.sequences ? i - 1 : 0;
            q_a = p.q_starts[b], q_b = p.q_starts[b + 1], k_a = ks[b], k_b = ks[b + 1];
            if (p.kv_lengths) keys = p.kv_lengths[b];
        }
        to = to < from ? from : to;
        // (starts that go back may put the slot before its sequence: none then)
        first = (uniform(slot - i) - (int)((uint32_t)uniform(from) / (uint32_t)R)) * R;
        first = first < 0 ? 0x7fffffff : first;
        s.real = i > 0 && i <= p.sequences;
        if (!s.real) {
            s.q0 = s.k0 = uniform(from);
            s.q_len = s.kv_len = uniform(to - from);
            s.keys = 0;
            return s;
        }
        const int q0 = clamp(q_a, 0, q_rows), k0 = clamp(k_a, 0, kv_rows);
        s.q_len = uniform(clamp(q_b, q0, q_rows) - q0);
        s.kv_len = uniform(clamp(k_b, k0, kv_rows) - k0);
        s.q0 = uniform(q0);
        s.k0 = uniform(k0);
        if (q_a != q0 || q_b != q0 + s.q_len || k_a != k0 || k_b != k0 + s.kv_len)
            if (threadIdx.x == 0) atomicOr(status, DENSE_ST_STARTS);
        s.keys = p.kv_lengths ? uniform(keys) : s.kv_len;
    }
    const int n = clamp(s.keys, 0, s.kv_len);
    if (s.keys != n && threadIdx.x == 0) atomicOr(status, DENSE_ST_STARTS);
    s.keys = n;
    return s;
}

// The keys that row r of a sequence sees: [0, keys_seen).
__device__ __forceinline__ int keys_seen(const Sequence &s, bool causal, int r) {
    if (!causal) return s.keys;
    const int n = r + 1 + s.keys - s.q_len;
    return n < 0 ? 0 : n > s.keys ? s.keys : n;
}

// Workgroup b of `units` (heads) x n (slots): the slots of a unit go to as few
// XCDs as can be, since they read the same rows, but in turns, since with causal
// masks the later ones of a sequence have more keys (or the earlier ones more
// rows): those first.
__device__ __forceinline__ bool unit_of(int64_t b, int units, int n, bool later_first, int &unit, int &slot) {
    const int x = (int)(b & 7), i = (int)(b >> 3);
    if (units % 8 == 0) {
        unit = x + 8 * (i / n);
        slot = i % n;
    } else if (8 % units == 0) {
        unit = x % units;
        slot = i * (8 / units) + x / units;
    } else {
        unit = (int)(b % units);
        slot = (int)(b / units);
    }
    if (later_first) slot = n - 1 - slot;
    return slot >= 0 && slot < n && unit < units;
}
// A tile's blocks (of keys, or of rows) are cut into parts of about `share`, at most
// `splits`, so that the longest sequences do not keep a few CUs busy after the
// others are done.  A launch has `splits` workgroups (blockIdx.y) for each tile, of which
// those past its parts end at once.  (Next to each other in blockIdx.x, those that end
// left half of an XCD's shader engines, which are taken in turns, without work.)
struct Cut {
    int64_t share;
    int splits;
};
__device__ __forceinline__ int parts_of(const Cut &c, int64_t blocks) {
    const int64_t n = (blocks + c.share - 1) / c.share;
    return (int)(n < 1 ? 1 : n < c.splits ? n : c.splits);
}
inline int64_t unit_grid(int units, int64_t n) {
    if (units % 8 && 8 % units == 0) return (n + 8 / units - 1) / (8 / units) * 8;
    return units * n;
}

// Rows of DP values in LDS, in chunks of 16 bytes: chunk c of row r lies at
// place c ^ key(r) of the row.  The keys are such that reading one chunk of 16
// rows, and 4 chunks of each of 4 rows (the transposing read), meets every one
// of the 64 banks once.
template <bool BF16, int DP>
struct Rows {
    static constexpr int E = BF16 ? 2 : 4, BYTES = DP * E, CHUNKS = BYTES / 16;
    static constexpr int VEC = BF16 ? 8 : 4;     // values of a chunk
    static constexpr int STEPS = CHUNKS / 2;     // products over a row's channels
    static_assert(CHUNKS >= 4, "head dimension");
    __device__ static __forceinline__ int key(int row) {
        if (CHUNKS == 4) return (row >> 2) & 3;
        if (CHUNKS == 8) return ((row & 2) << 1) | ((row >> 2) & 3);
        if (BF16) return ((row & 3) << 2) | ((row >> 2) & 3);
        return ((row & 4) << 1) | ((row & 8) >> 1) | (row & 3);
    }
    __device__ static __forceinline__ int at(int row, int chunk) { return row * BYTES + ((chunk ^ key(row)) << 4); }
};

template <Type T, int DP>
using RowsOf = Rows<T != F32, DP>;
// Bytes of a tile of `rows` rows, its planes one behind the other.
template <Type T, int DP>
constexpr int tile_bytes(int rows) { return kPlanes<T> * rows * RowsOf<T, DP>::BYTES; }

// acc += a b over 2 x 16 bytes of each row.
template <bool BF16>
__device__ __forceinline__ void mma(const u32x4_t &a, const u32x4_t &b, f32x16_t &acc) {
    if constexpr (BF16) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                      acc, 0, 0, 0);
    } else {
        const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
    }
}

__device__ __forceinline__ void clear(f32x16_t &a) {
#pragma unroll
    for (int e = 0; e < 16; ++e) a[e] = 0.f;
}

// Order of what lies between two sched_barriers: AHEAD reads of LDS, then a product and
// a read in turns (left alone, the compiler waits for each read before its product).
template <int PRODUCTS, int READS, int AHEAD, int I = 0>
__device__ __forceinline__ void read_ahead() {
    if constexpr (I == 0) __builtin_amdgcn_sched_group_barrier(0x100, AHEAD < READS ? AHEAD : READS, 0);
    if constexpr (I < PRODUCTS) {
        // as many a product as keep the distance
        constexpr int PER = (READS + PRODUCTS - 1) / PRODUCTS, DONE = AHEAD + I * PER;
        constexpr int r = DONE >= READS ? 0 : READS - DONE < PER ? READS - DONE : PER;
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
        read_ahead<PRODUCTS, READS, AHEAD, I + 1>();
    }
}

// A row's values as a right operand: this lane's chunks 2 t + lane / 32.
template <Type T, int DP>
struct Fragments {
    u32x4_t v[kPlanes<T>][RowsOf<T, DP>::STEPS];
};

// acc = (rows row0.. of a tile of ROWS) (fragments b)^T.  Of planes the smaller
// products come first.
template <Type T, int DP, int ROWS>
__device__ __forceinline__ void rows_times(const char *tile, int row0, const Fragments<T, DP> &b, f32x16_t &acc) {
    using L = RowsOf<T, DP>;
    constexpr int P = kPlanes<T>;
    const int lane = threadIdx.x & 63, row = row0 + (lane & 31), h = lane >> 5;
#pragma unroll
    for (int t = 0; t < L::STEPS; ++t) {
        u32x4_t a[P];
#pragma unroll
        for (int p = 0; p < P; ++p)
            a[p] = *reinterpret_cast<const u32x4_t *>(tile + p * ROWS * L::BYTES + L::at(row, 2 * t + h));
#pragma unroll
        for (int sum = P - 1; sum >= 0; --sum)
#pragma unroll
            for (int p = 0; p <= sum; ++p) mma<T != F32>(a[p], b.v[sum - p][t], acc);
    }
}

// Three bf16 whose sum is x, of two values at a time: of values below 2^-110 the
// last ones vanish.
__device__ __forceinline__ void planes_of(float x0, float x1, uint32_t &h, uint32_t &m, uint32_t &l) {
    h = pack_bf16(x0, x1);
    const float r0 = x0 - __uint_as_float(h << 16), r1 = x1 - __uint_as_float(h & 0xffff0000u);
    m = pack_bf16(r0, r1);
    l = pack_bf16(r0 - __uint_as_float(m << 16), r1 - __uint_as_float(m & 0xffff0000u));
}

// The right operand made of an accumulator's block: 4 values a register group.
template <Type T>
struct Right {
    u32x4_t v[kPlanes<T>][T == F32 ? 4 : 2];
    __device__ __forceinline__ void set(const f32x16_t &x) {
        if constexpr (T == F32) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[0][g][i] = __float_as_uint(x[4 * g + i]);
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x0 = x[8 * s + 2 * i], x1 = x[8 * s + 2 * i + 1];
                    if constexpr (T == PLANES) {
                        uint32_t h, m, l;
                        planes_of(x0, x1, h, m, l);
                        v[0][s][i] = h, v[1][s][i] = m, v[2][s][i] = l;
                    } else {
                        v[0][s][i] = pack_bf16(x0, x1);
                    }
                }
        }
    }
};

// acc[d] += (channels of rows row0 .. row0 + 31 of a tile of ROWS)^T b, for 32
// channels a block d.
template <Type T, int DP, int ROWS>
__device__ __forceinline__ void columns_times(const char *tile, int row0, const Right<T> &b, f32x16_t (&acc)[DP / 32]) {
    using L = RowsOf<T, DP>;
    constexpr int P = kPlanes<T>;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (T != F32) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const int j = lane & 15, wide = (lane >> 4) & 1;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                const int chunk = 4 * d + 2 * wide + ((j & 3) >> 1);
                u32x4_t a[P];
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    s16x4_t x[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row = row0 + 16 * s + 8 * u + 4 * h + (j >> 2);
                        x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (lds_s16x4 *)(tile + p * ROWS * L::BYTES + L::at(row, chunk) + 8 * (j & 1)));
                    }
                    const s16x8_t both = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    a[p] = __builtin_bit_cast(u32x4_t, both);
                }
#pragma unroll
                for (int sum = P - 1; sum >= 0; --sum)
#pragma unroll
                    for (int p = 0; p <= sum; ++p) mma<true>(a[p], b.v[sum - p][s], acc[d]);
            }
    } else {
        const int c = lane & 31;
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = row0 + 8 * g + 4 * h + i;
                    const float x = *reinterpret_cast<const float *>(tile + L::at(row, 8 * d + (c >> 2)) + 4 * (c & 3));
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, __uint_as_float(b.v[0][g][i]), acc[d], 0, 0, 0);
                }
    }
}

// Fragments of a row of a tensor, zeros past the row's D channels.
template <Type T, int DP>
__device__ __forceinline__ void load_fragments(const View &x, int64_t row, int head, int D, Fragments<T, DP> &f) {
    using L = RowsOf<T, DP>;
    const int h = (threadIdx.x & 63) >> 5;
    const char *from = reinterpret_cast<const char *>(x.p) + (row * x.row + head * x.head) * L::E;
#pragma unroll
    for (int p = 0; p < kPlanes<T>; ++p)
#pragma unroll
        for (int t = 0; t < L::STEPS; ++t) {
            Raw<T != F32, L::VEC> u;
            load_raw<T != F32, L::VEC>(from + p * x.plane, (2 * t + h) * L::VEC, D, u);
            f.v[p][t] = u32x4_t{u.w[0], u.w[1], u.w[2], u.w[3]};
        }
}

// Bring ROWS rows of a tensor into LDS with WAVES wavefronts (this one is number
// `wave` of them): straight (DMA; rows start at multiples of 16 bytes and are
// whole chunks long) or through registers.  Rows past the last one and chunks
// past a row's last stand in for those that are not there: their scores are
// masked, their channels not stored.
template <Type T, int DP, int ROWS, int WAVES, bool DMA>
struct Loader {
    using L = RowsOf<T, DP>;
    static_assert(T != PLANES || DMA, "planes are laid out for direct loads");
    static constexpr int EACH = ROWS * L::CHUNKS / 64;  // wavefronts' loads of a plane, 1 KB each
    static constexpr int ALL = kPlanes<T> * EACH;       // not all wavefronts may have as many
    static constexpr int N = (ALL + WAVES - 1) / WAVES;
    static_assert(ROWS * L::CHUNKS % 64 == 0, "loads of a tile");
    __device__ __forceinline__ bool has(int n) const { return ALL % WAVES == 0 || n * WAVES + wave < ALL; }
    const char *base;
    int64_t stride, plane;  // bytes
    int D, wave;
    uint32_t offset[DMA ? N : 1];  // of this lane's loads from the first row's start
    u32x4_t r[DMA ? 1 : N];

    __device__ __forceinline__ Loader(const View &x, int64_t row0, int head, int D, int wave)
        : base(reinterpret_cast<const char *>(x.p) + (row0 * x.row + head * x.head) * L::E), stride(x.row * L::E),
          plane(x.plane), D(D), wave(wave) {
        if constexpr (DMA)
#pragma unroll
            for (int n = 0; n < N; ++n) offset[n] = offset_of(n, ROWS - 1);
    }
    // Row and chunk of this lane's load n in its plane.
    __device__ __forceinline__ void place(int n, int &row, int &chunk) const {
        const int id = (n * WAVES + wave) % EACH * 64 + (threadIdx.x & 63);
        row = id / L::CHUNKS;
        chunk = (id % L::CHUNKS) ^ L::key(row);
    }
    __device__ __forceinline__ uint32_t offset_of(int n, int last) const {
        int row, chunk;
        place(n, row, chunk);
        const int end = D * L::E / 16 - 1;
        return (uint32_t)(row < last ? row : last) * (uint32_t)stride + (chunk < end ? chunk : end) * 16;
    }
    // Rows first .. of which the tensor has `rows` (more than first).
    __device__ __forceinline__ void fetch(char *tile, int first, int rows) {
        const int last = rows - 1 - first;
        const char *from = base + first * stride;
        if constexpr (DMA) {
            const bool whole = last >= ROWS - 1;
            if constexpr (T == PLANES) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if (!has(n)) continue;
                    const gemm::rsrc_t src = gemm::buffer(uniform(from + (n * WAVES + wave) / EACH * plane));
                    gemm::dma16(src, whole ? offset[n] : offset_of(n, last), 0, tile + (n * WAVES + wave) * 1024);
                }
            } else {
                const gemm::rsrc_t src = gemm::buffer(uniform(from));
                if (whole) {
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (has(n)) gemm::dma16(src, offset[n], 0, tile + (n * WAVES + wave) * 1024);
                } else {
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (has(n)) gemm::dma16(src, offset_of(n, last), 0, tile + (n * WAVES + wave) * 1024);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (!has(n)) continue;
                int row, chunk;
                place(n, row, chunk);
                Raw<T != F32, L::VEC> u;
                load_raw<T != F32, L::VEC>(from + (int64_t)(row < last ? row : last) * stride, chunk * L::VEC, D, u);
                r[n] = u32x4_t{u.w[0], u.w[1], u.w[2], u.w[3]};
            }
        }
    }
    // What fetch() holds in registers goes to the tile.
    __device__ __forceinline__ void commit(char *tile) const {
        if constexpr (!DMA) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (has(n)) *reinterpret_cast<u32x4_t *>(tile + ((n * WAVES + wave) * 64 + lane) * 16) = r[n];
        }
    }
};

// In a branch that few blocks take: keeps the compiler from making selects of it, which all
// blocks would go through.
__device__ __forceinline__ void seldom() { asm volatile(""); }

// The maximum, or the sum, of a value and that of the lane 32 further (or before).
__device__ __forceinline__ float pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Scores of keys from `seen` on (of the block from key0 on) count for nothing.
__device__ __forceinline__ void mask(f32x16_t &s, int key0, int seen) {
    const int n = seen - key0 - 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + (e & 3) >= n) s[e] = -INFINITY;
}

// Store 4 channels c0 .. of a row of D of them.
template <bool BF16>
__device__ __forceinline__ void store4(void *row, int c0, int D, const float *v) {
    if (c0 + 4 <= D) {
        if constexpr (BF16) {
            struct __attribute__((packed, aligned(2))) Two { uint32_t v[2]; };
            *reinterpret_cast<Two *>(reinterpret_cast<uint16_t *>(row) + c0) = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        } else {
            *reinterpret_cast<Words4 *>(reinterpret_cast<float *>(row) + c0) =
                {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i < D) {
                if (BF16)
                    reinterpret_cast<uint16_t *>(row)[c0 + i] = (uint16_t)pack_bf16(v[i], 0.f);
                else
                    reinterpret_cast<float *>(row)[c0 + i] = v[i];
            }
    }
}

// D values of zero.
template <bool BF16>
__device__ __forceinline__ void zero_row(void *row, int D, int lane, int lanes) {
    for (int c = lane; c < D; c += lanes) {
        if (BF16)
            reinterpret_cast<uint16_t *>(row)[c] = 0;
        else
            reinterpret_cast<float *>(row)[c] = 0.f;
    }
}

// -- fp32 tensors as planes of bf16 --

// [3][rows][heads][DP] of up to four tensors, one of blockIdx.y each, channels from D on zeros.
struct PlaneJobs {
    View x[4];
    uint16_t *out[4];
    int64_t rows[4];
    int heads[4];
};
namespace {
__global__ __launch_bounds__(256) void k_planes(PlaneJobs jobs, int D, int DP) {
    const int j = blockIdx.y, parts = DP / 8;
    const View x = jobs.x[j];
    const int64_t all = jobs.rows[j] * jobs.heads[j] * parts;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t rh = i / parts, row = rh / jobs.heads[j];
        const int c0 = (int)(i - rh * parts) * 8, head = (int)(rh - row * jobs.heads[j]);
        Raw<false, 8> u;
        load_raw<false, 8>(reinterpret_cast<const float *>(x.p) + row * x.row + head * x.head, c0, D, u);
        u32x4_t p[3];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h, m, l;
            planes_of(__uint_as_float(u.w[2 * k]), __uint_as_float(u.w[2 * k + 1]), h, m, l);
            p[0][k] = h, p[1][k] = m, p[2][k] = l;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<u32x4_t *>(jobs.out[j] + (k * all + i) * 8) = p[k];
    }
}
}  // namespace
// Lay x out at `at` (its bytes: plane_bytes), and take it from there.
inline void add_planes(PlaneJobs &jobs, int j, View &x, int64_t rows, int heads, int DP, void *at) {
    jobs.x[j] = x;
    jobs.out[j] = static_cast<uint16_t *>(at);
    jobs.rows[j] = rows;
    jobs.heads[j] = heads;
    x = {at, (int64_t)heads * DP, DP, rows * heads * DP * 2};
}
inline int64_t plane_bytes(int64_t rows, int heads, int DP) { return 3 * rows * heads * DP * 2; }
inline hipError_t launch_planes(lattice_dense *D, const PlaneJobs &jobs, int count, int C, int DP) {
    int64_t most = 1;
    for (int j = 0; j < count; ++j) most = std::max(most, jobs.rows[j] * jobs.heads[j] * (DP / 8));
    hipLaunchKernelGGL(k_planes, dim3(grid_for(most, 256, D->cu_count), (unsigned)count), dim3(256), 0, D->stream, jobs, C, DP);
    return hipGetLastError();
}

// -- host side --

// Whether a tensor's rows can go to LDS straight.
inline bool straight(const View &x, int D, int E) {
    return (D * E) % 16 == 0 && (x.row * E) % 16 == 0 && (x.head * E) % 16 == 0 &&
           reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && x.row * E < ((int64_t)1 << 25);
}
// Whether fp32 products go by planes of bf16: where they take the fp32 cores longer than laying
// the planes out, a launch of its own.  4 heads of 32, rows and keys alike, fp32 cores and planes
// in us: forward 600 rows (5e7 of these products) 20 and 23, 1000 (1.3e8) 31 and 25, 2500 67 and 55;
// backward 300 rows (1.2e7) 46 and 40, 2500 193 and 130.  Wider heads are not built so: two
// stages of 64 keys' planes of 128 channels take 192 KB of LDS, more than there is; blocks of 32
// keys would fit, with one wavefront a SIMD, which is what the fp32 cores' kernels have there too.
// (Nor are planes of more than 8 GB made.)
inline bool planes_pay(const AttendArgs &a, int64_t keys, double from) {
    return a.D <= 64 && (double)a.q_rows * a.heads * (double)keys * a.D >= from &&
           ((double)a.q_rows * a.heads + (double)a.kv_rows * a.kv_heads) * 2 * 6 * 64 <= 8e9;
}
inline int padded_dim(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }
// Slots of tiles of R rows, see find().
inline int64_t slots_of(const int32_t *starts, int64_t sequences, int64_t rows, int R) {
    return starts ? rows / R + sequences + 2 : (rows + R - 1) / R;
}
// How the query heads of a key head and the rows of a sequence share the columns
// of a tile.
struct Columns {
    int parts, heads, R;  // parts of the group, query heads of one, rows
    Columns(int group, int columns) {
        parts = (group + columns - 1) / columns;
        heads = (group + parts - 1) / parts;
        parts = (group + heads - 1) / heads;
        R = columns / heads;
    }
};
inline Packing packing_of(const AttendArgs &a) {
    return {a.q_rows, a.kv_rows, a.q_starts, a.kv_starts, a.kv_lengths, (int)a.sequences, a.causal};
}
// Workgroups of a launch; more go in several (the threads along a side have 32 bits).
constexpr int64_t kMostGrid = (int64_t)1 << 22;
template <class Params, class Launch>
hipError_t in_launches(Params p, int64_t grid, Launch launch) {
    for (p.block0 = 0; p.block0 < grid; p.block0 += kMostGrid) {
        const int64_t left = grid - p.block0;
        launch(dim3((unsigned)(left < kMostGrid ? left : kMostGrid), (unsigned)p.cut.splits), p);
        TRY(hipGetLastError());
    }
    return hipSuccess;
}
// How a launch of `grid` workgroups cuts its tiles: `tiles` of them have about `blocks`
// blocks each, and none more than `most`.  A part is what each of `places` workgroups
// that run at once has to do in all, or half of it where there are few tiles for a place
// (whole tiles: 4.5 ms for a training step of 16 objects of 1 to 6411 rows in fp32, halves
// 4.1; with four tiles a place whole ones are better, 0.93 and 1.03 ms for 12 sequences of
// 1 to 3400 rows in bf16).  Room for a sequence four times as long as the mean one;
// `room`: parts whose results are not too large.
inline Cut cut_of(int64_t tiles, int64_t blocks, int64_t most, int64_t grid, int64_t places, int64_t least, int64_t room) {
    Cut c;
    c.share = tiles * blocks / ((tiles < 4 * places ? 2 : 1) * places);
    c.share = c.share < least ? least : c.share;
    most = most < 4 * blocks ? most : 4 * blocks;
    int64_t n = (most + c.share - 1) / c.share;
    const int64_t few = 32 * places / (grid > 0 ? grid : 1);  // workgroups that end at once are not free
    n = n < kMostSplits ? n : kMostSplits;
    n = n < few || n <= 2 ? n : few < 2 ? 2 : few;
    n = n < room ? n : room;
    c.splits = (int)(n < 1 || grid > kMostGrid ? 1 : n);
    return c;
}
// The grid of a join: tiles, their rows by kJoinRows, and what each of these has to do in
// up to `pieces` where there are not workgroups enough.
inline dim3 join_grid(int64_t slots, int R, int64_t pieces) {
    const int64_t y = (R + kJoinRows - 1) / kJoinRows, z = 8192 / (slots * y);
    return dim3((unsigned)slots, (unsigned)y, (unsigned)(z < 1 ? 1 : z < pieces ? z : pieces));
}
// Bytes of partial results that are not too large.
constexpr int64_t kMostParts = (int64_t)1 << 29;

}  // namespace attend
