// Attention among all atoms of a segment: what its forward and backward kernels share.
//
// Rows and tiles.  The query heads that share a key head are stacked: row r of a (segment, key head) is query r / group,
// head r % group of the group.  So keys and values are read once for all of them, one query is a tile like any other, and
// the gradients of a key head come out summed over its query heads.  A wave owns 32 rows (backward over the keys: 32 keys) and
// works with 32 x 32 matrix instructions, transposed: in
//   S^T = K Q^T            lane l holds row l % 32 and the keys 8 (i/4) + 4 (l/32) + i % 4, i = 0..15
// a row's parameters are the lane's own registers, its sums over the keys are additions within the lane (and one exchange
// of the two halves at the end), and the weights need no exchange to become an operand of
//   O^T = V^T P^T
// because the order in which a product's sum runs over the keys is free: operand V^T takes the keys in the order in which
// the weights lie in the lanes.
#pragma once
#include <type_traits>

#include "e2f_block.h"

namespace e2f {

constexpr float LOG2E = 1.4426950408889634f;

// What the score of a pair is formed from, in units of base-2 logarithms (so that the softmax's exponential is exp2).
struct DenseScore {
    float in;            // x = in * (q . k): the argument of the tanh, or without a cap the score itself
    float out, inv_out;  // cap log2(e) and its reciprocal
    float c[8];          // odd polynomial of out * tanh
    int32_t capped, biased;
};

struct DenseParams {
    Rows q, k, v, out;             // out: out, or grad_q
    Rows go, gk, gv;               // backward: dL/dout, grad_k, grad_v
    const int32_t *q_offsets, *k_offsets, *q_lengths, *k_lengths;
    const float *q_pos, *k_pos, *slope;
    int32_t Nq, Nk, S, Hk, group, D, group_shift;
    uint32_t group_magic;
    float scale;
    DenseScore score;
    float *part, *part_sum;        // forward with split keys: [splits][Nq][Hq][D] sums over a part's keys, [splits][Nq][Hq][2] reference, sum
    float4* stats;                 // backward: [Nq][Hq] softmax reference, 1 / sum, delta, reference + log2(sum)
    float* usual;                  // backward: [Nq][Hq] mean distance under a row's weights
    // of the parts of a backward pass: [parts] of [row tiles][Hq], [Hq][Nq][3], [Hk][Nk][3], [Nq][Hq], [Nq][Hq][D], [Nk][Hk][D]
    float *slope_part, *q_pos_part, *k_pos_part;
    float4* stats_part;
    float *gq_part, *gk_part, *gv_part;
    __device__ __forceinline__ int over_group(uint32_t r) const { return (int)((uint64_t)r * group_magic >> group_shift); }
};

// The tokens of segment s that count: first token and number.
__device__ __forceinline__ void segment_range(const int32_t* offsets, const int32_t* lengths, int s, int N, int& first, int& n) {
    first = min(max(offsets[s], 0), N);
    n = min(max(offsets[s + 1], first), N) - first;
    if (lengths) n = min(max(lengths[s], 0), n);
}

// Tiles are numbered so that no table is needed: with rows = tokens * group, segment s starts at tile
// floor(rows before it / BM) + s, which leaves it at least as many tiles as it has rows for, since
// floor(a + b) - floor(a) + 1 >= ceil(b).  The whole wave looks for the segment, 64 candidates at a time.
__device__ __forceinline__ int64_t first_tile(int offset, int s, int N, int group, int BM) {
    return ((int64_t)min(max(offset, 0), N) * group >> (BM == 128 ? 7 : 5)) + s;
}
static inline int64_t dense_tiles(int64_t N, int group, int S, int BM) { return N * group / BM + S; }

struct Segment {
    int q0, nq, k0, nk;            // first query, queries, first key, keys
    int64_t first;                 // first tile
};
// KEYS: tiles of keys instead of rows.  The last round reads all that is wanted of its 63 candidates, so that a workgroup among up to 63
// segments waits for memory once.
template <bool KEYS>
__device__ __forceinline__ Segment segment_of(const DenseParams& A, int BM, int64_t tile) {
    const int32_t* offsets = KEYS ? A.k_offsets : A.q_offsets;
    const int N = KEYS ? A.Nk : A.Nq, group = KEYS ? 1 : A.group, lane = threadIdx.x & 63;
    int lo = 0, n = A.S;           // the answer lies in [lo, lo + n)
    while (n > 63) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        const bool before = lane * step < n && first_tile(offsets[min(at, A.S)], at, N, group, BM) <= tile;
        const int k = __popcll(__ballot(before)), next = lo + (k ? k - 1 : 0) * step;      // candidate 0 always counts
        n = min(step, lo + n - next);
        lo = next;
    }
    const int at = lo + min(lane, n);
    const int q = A.q_offsets[at], k = A.k_offsets[at];
    int lq = INT32_MAX, lk = INT32_MAX;
    if (A.q_lengths) lq = A.q_lengths[min(at, A.S - 1)];
    if (A.k_lengths) lk = A.k_lengths[min(at, A.S - 1)];
    const int64_t first = first_tile(KEYS ? k : q, at, N, group, BM);
    const int found = max(__popcll(__ballot(lane < n && first <= tile)) - 1, 0);
    auto of = [&](int x, int i) { return __builtin_amdgcn_readlane(x, i); };
    Segment s;
    s.q0 = min(max(of(q, found), 0), A.Nq);
    s.nq = min(max(of(lq, found), 0), min(max(of(q, found + 1), s.q0), A.Nq) - s.q0);
    s.k0 = min(max(of(k, found), 0), A.Nk);
    s.nk = min(max(of(lk, found), 0), min(max(of(k, found + 1), s.k0), A.Nk) - s.k0);
    s.first = first_tile(KEYS ? s.k0 : s.q0, __builtin_amdgcn_readfirstlane(lo) + found, N, group, BM);
    return s;
}

// The last segment that starts at or before a token.
__device__ __forceinline__ int token_segment(const int32_t* offsets, int S, int token) {
    int lo = 0, hi = S;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid] <= token) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// the upper halves of two words, the first in the low half
__device__ __forceinline__ uint32_t upper(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

// Matrix instructions and operands of the two feature types.  DP: D rounded up to 32, zero beyond D.  A tile is BN rows of
// features in LDS, LD elements from row to row, a row's 16-byte pieces in the order piece(row, .).
template <typename T, int DP>
struct Mma;

// bf16: v_mfma_f32_32x32x16_bf16, lane l: row l % 32, summands 8 (l/32) .. +7
template <int DP>
struct Mma<uint16_t, DP> {
    using T = uint16_t;      // in memory
    using E = uint16_t;      // in LDS
    // Rows are 16 banks of 64 apart (modulo 64), so that the transposed reads of 4 rows x 32 features meet no bank twice, and pieces
    // are exchanged within groups of four by the row, so that the reads of one piece of 8 rows do not either.
    static constexpr int STEPS = DP / 16, LD = DP == 64 ? 96 : DP == 128 ? 160 : DP;
    static __device__ __forceinline__ int piece(int row, int i) { return i ^ (row >> 2 & 3); }
    static __device__ __forceinline__ void keep(E* tile, int row, int i, u32x4 x) { *reinterpret_cast<u32x4*>(tile + row * LD + piece(row, i) * 8) = x; }
    // a row of features as an operand, for products over the features
    struct Frag {
        bf16x8 x[STEPS];
    };
    static __device__ __forceinline__ void load(Frag& f, const char* row, int D, bool valid, int half) {
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int d = 16 * c + 8 * half;
            u32x4 x = {0, 0, 0, 0};
            if (valid && d < D) x = *reinterpret_cast<const u32x4*>(row + d * 2);
            f.x[c] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // A B^T over the features: A 32 rows of a tile
    static __device__ __forceinline__ f32x16 dot(const T* tile, int row0, const Frag& b, int lane) {
        f32x16 acc = {};
        const T* row = tile + (row0 + (lane & 31)) * LD;
        const T* p[2] = {row + 8 * piece(lane, lane >> 5), row + 8 * piece(lane, 2 + (lane >> 5))};      // row0: a multiple of 32
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(p[c & 1] + 32 * (c >> 1)), b.x[c], acc, 0, 0, 0);
        return acc;
    }
    // weights of 32 tile rows as an operand of products over those rows: the sum of two bf16 each (the first cut, the second what is
    // left, rounded: off by 2^-15 at most).  One bf16 would bring as much error as the rounding of a bf16 result, and more to sums whose
    // terms cancel: errors of 2.4e-3 in place of 1.7e-3, for 10 % less time (10 000 atoms 562 us, with two 620; without cap and bias 322 and 401).
    struct Weights {
        bf16x8 x[2][2];
    };
    static __device__ __forceinline__ Weights weights(const f32x16& p) {
        Weights w;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            u32x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = p[8 * c + 2 * e], b = p[8 * c + 2 * e + 1];
                const uint32_t i = __float_as_uint(a), j = __float_as_uint(b);
                x[e] = upper(i, j);
                y[e] = pack_bf16(a - __uint_as_float(i & 0xFFFF0000u), b - __uint_as_float(j & 0xFFFF0000u));
            }
            w.x[0][c] = __builtin_bit_cast(bf16x8, x);
            w.x[1][c] = __builtin_bit_cast(bf16x8, y);
        }
        return w;
    }
    static constexpr int WEIGHT_VECTORS = 4;      // 16-byte pieces of a lane's weights
    static __device__ __forceinline__ void put(u32x4* to, const Weights& w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) to[64 * i] = __builtin_bit_cast(u32x4, w.x[i / 2][i % 2]);
    }
    static __device__ __forceinline__ Weights get(const u32x4* from) {
        Weights w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w.x[i / 2][i % 2] = __builtin_bit_cast(bf16x8, from[64 * i]);
        return w;
    }
    // Transposed operands: ds_read_b64_tr_b16 turns 4 rows of 16 features in each 16 lanes: lane 4 r + c of them addresses features
    // 4 c .. of row r, lane i gets feature i of the four rows.  p, q: a lane's places in rows 4 half .. and 8 + 4 half .., whose pieces
    // are exchanged by half and 2 + half.
    template <int LINE>
    static __device__ __forceinline__ void turned_rows(const E* tile, int row0, int lane, const E*& p, const E*& q) {
        const int half = lane >> 5, i = (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
        const E* row = tile + (row0 + 4 * half + (lane >> 2 & 3)) * LINE + 4 * (lane & 1);
        p = row + 8 * (i ^ half);
        q = row + 8 * LINE + 8 * (i ^ (2 + half));
    }
    static __device__ __forceinline__ bf16x8 turned(const E* p, const E* q) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)q);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // acc[dt] += (features 32 dt .. of the tile, transposed) W over the 32 tile rows from row0
    template <int NT>
    static __device__ __forceinline__ void accumulate(f32x16 (&acc)[NT], const E* tile, int row0, const Weights& w, int lane) {
        const E *p, *q;
        turned_rows<LD>(tile, row0, lane, p, q);
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const bf16x8 a = turned(p + dt * 32 + 16 * c * LD, q + dt * 32 + 16 * c * LD);
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w.x[1][c], acc[dt], 0, 0, 0);
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w.x[0][c], acc[dt], 0, 0, 0);
            }
    }
};

// binary32 beyond 64 features: v_mfma_f32_32x32x2_f32, lane l: row l % 32, summand l / 32.  The order of the sum over the features is free as
// well: the lower half of the lanes takes the first DP/2 features, so that a lane's operands lie side by side.
template <int DP>
struct MmaNative {
    using T = float;
    using E = float;
    static constexpr int LD = DP + 8, H = DP / 2;
    static __device__ __forceinline__ void keep(E* tile, int row, int i, u32x4 x) { *reinterpret_cast<u32x4*>(tile + row * LD + i * 4) = x; }
    struct Frag {
        float x[H];
    };
    static __device__ __forceinline__ void load(Frag& f, const char* row, int D, bool valid, int half) {
#pragma unroll
        for (int c = 0; c < H; c += 4) {
            const int d = half * H + c;
            f32x4 x = {0, 0, 0, 0};
            if (valid && d < D) x = *reinterpret_cast<const f32x4*>(row + d * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) f.x[c + e] = x[e];
        }
    }
    static __device__ __forceinline__ f32x16 dot(const T* tile, int row0, const Frag& b, int lane) {
        f32x16 acc = {};
        const T* p = tile + (row0 + (lane & 31)) * LD + (lane >> 5) * H;
#pragma unroll
        for (int c = 0; c < H; c += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], b.x[c + e], acc, 0, 0, 0);
        }
        return acc;
    }
    struct Weights {
        f32x16 x;
    };
    static __device__ __forceinline__ Weights weights(const f32x16& p) { return Weights{p}; }
    static constexpr int WEIGHT_VECTORS = 4;
    static __device__ __forceinline__ void put(u32x4* to, const Weights& w) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const f32x4 x = {w.x[4 * c], w.x[4 * c + 1], w.x[4 * c + 2], w.x[4 * c + 3]};
            to[64 * c] = __builtin_bit_cast(u32x4, x);
        }
    }
    static __device__ __forceinline__ Weights get(const u32x4* from) {
        Weights w;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const f32x4 x = __builtin_bit_cast(f32x4, from[64 * c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) w.x[4 * c + e] = x[e];
        }
        return w;
    }
    template <int NT>
    static __device__ __forceinline__ void accumulate(f32x16 (&acc)[NT], const T* tile, int row0, const Weights& w, int lane) {
        const T* p = tile + (row0 + 4 * (lane >> 5)) * LD + (lane & 31);
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(p[(8 * (i / 4) + i % 4) * LD + dt * 32], w.x[i], acc[dt], 0, 0, 0);
    }
};

// binary32 up to 64 features: a value as the sum of three bf16 with 8 bits of its significand each (cut, not rounded, so that the parts
// keep its sign, are exact, and no part of a finite value is infinite), a product as six of its nine partial products, each a bf16 matrix
// instruction with binary32 sums.  The parts are below 2^-7 and 2^-15 of the value's power of two, so that the three left out are below 2^-21 of the
// product (7.8 * 2^-24 at worst, 0.7 * 2^-24 in the mean of random factors) and make it smaller, never larger.  For 16 summands these
// take 6 x 32 cycles where 8 binary32 instructions take 64 each.  (More features would not leave room for the three parts of the
// operands in registers.)
__device__ __forceinline__ void cut(float x, uint32_t (&part)[3]) {
    part[0] = __float_as_uint(x);
    const float r = x - __uint_as_float(part[0] & 0xFFFF0000u);
    part[1] = __float_as_uint(r);
    part[2] = __float_as_uint(r - __uint_as_float(part[1] & 0xFFFF0000u));
}
template <int DP>
struct MmaSplit {
    using T = float;
    using E = uint16_t;
    using Row = Mma<uint16_t, DP>;
    static constexpr int STEPS = DP / 16, LD = DP == 64 ? 224 : 96;      // a row's three parts one after the other, rows 48 banks apart
    static_assert(DP == 32 || DP == 64, "");
    static __device__ __forceinline__ void keep(E* tile, int row, int i, u32x4 x) {
        uint32_t p[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) cut(__uint_as_float(x[e]), p[e]);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            *reinterpret_cast<u32x2*>(tile + row * LD + k * DP + Row::piece(row, i >> 1) * 8 + (i & 1) * 4) = u32x2{upper(p[0][k], p[1][k]), upper(p[2][k], p[3][k])};
    }
    struct Frag {
        bf16x8 x[3][STEPS];
    };
    static __device__ __forceinline__ void cut8(const float (&f)[8], bf16x8 (&x)[3]) {
        uint32_t p[8][3];
#pragma unroll
        for (int e = 0; e < 8; ++e) cut(f[e], p[e]);
#pragma unroll
        for (int k = 0; k < 3; ++k)
            x[k] = __builtin_bit_cast(bf16x8, u32x4{upper(p[0][k], p[1][k]), upper(p[2][k], p[3][k]), upper(p[4][k], p[5][k]), upper(p[6][k], p[7][k])});
    }
    static __device__ __forceinline__ void load(Frag& f, const char* row, int D, bool valid, int half) {
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const int d = 16 * c + 8 * half;
            float x[8] = {};
            if (valid && d < D) {
                const f32x4 a = *reinterpret_cast<const f32x4*>(row + d * 4), b = *reinterpret_cast<const f32x4*>(row + d * 4 + 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = a[e];
                    x[4 + e] = b[e];
                }
            }
            bf16x8 parts[3];
            cut8(x, parts);
#pragma unroll
            for (int k = 0; k < 3; ++k) f.x[k][c] = parts[k];
        }
    }
    // the small partial products first
    static __device__ __forceinline__ f32x16 product(const bf16x8 (&a)[3], const bf16x8& b0, const bf16x8& b1, const bf16x8& b2, f32x16 acc) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2], b0, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b1, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b2, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b0, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b1, acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b0, acc, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 dot(const E* tile, int row0, const Frag& b, int lane) {
        f32x16 acc = {};
        const E* row = tile + (row0 + (lane & 31)) * LD;
        const E* p[2] = {row + 8 * Row::piece(lane, lane >> 5), row + 8 * Row::piece(lane, 2 + (lane >> 5))};
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            bf16x8 a[3];
#pragma unroll
            for (int k = 0; k < 3; ++k) a[k] = *reinterpret_cast<const bf16x8*>(p[c & 1] + 32 * (c >> 1) + k * DP);
            acc = product(a, b.x[0][c], b.x[1][c], b.x[2][c], acc);
        }
        return acc;
    }
    struct Weights {
        bf16x8 x[3][2];
    };
    static __device__ __forceinline__ Weights weights(const f32x16& p) {
        Weights w;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = p[8 * c + e];
            bf16x8 parts[3];
            cut8(f, parts);
#pragma unroll
            for (int k = 0; k < 3; ++k) w.x[k][c] = parts[k];
        }
        return w;
    }
    static constexpr int WEIGHT_VECTORS = 6;
    static __device__ __forceinline__ void put(u32x4* to, const Weights& w) {
#pragma unroll
        for (int i = 0; i < 6; ++i) to[64 * i] = __builtin_bit_cast(u32x4, w.x[i / 2][i % 2]);
    }
    static __device__ __forceinline__ Weights get(const u32x4* from) {
        Weights w;
#pragma unroll
        for (int i = 0; i < 6; ++i) w.x[i / 2][i % 2] = __builtin_bit_cast(bf16x8, from[64 * i]);
        return w;
    }
    template <int NT>
    static __device__ __forceinline__ void accumulate(f32x16 (&acc)[NT], const E* tile, int row0, const Weights& w, int lane) {
        const E *p, *q;
        Row::template turned_rows<LD>(tile, row0, lane, p, q);
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                bf16x8 a[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) a[k] = Row::turned(p + dt * 32 + 16 * c * LD + k * DP, q + dt * 32 + 16 * c * LD + k * DP);
                acc[dt] = product(a, w.x[0][c], w.x[1][c], w.x[2][c], acc[dt]);
            }
    }
};

template <int DP>
struct Mma<float, DP> : std::conditional_t<(DP <= 64), MmaSplit<DP <= 64 ? DP : 64>, MmaNative<DP>> {};

// BN rows of features on their way from memory into a tile, in the registers of THREADS threads: rows and features behind the end as zeros.
// Rows at one stride (below 2^25 bytes): a load's address is the tile's, the same for all threads, and a 32-bit offset that a thread
// forms once, so that the loop has no vector instructions for addresses (2 % of the time of 10 000 atoms).  Rows of several heads: the row's.
template <typename M, int DP, int BN, int THREADS>
struct Transfer {
    using T = typename M::T;
    static constexpr int V = 16 / sizeof(T), VECS = DP / V, EACH = BN * VECS / THREADS;
    static_assert(BN * VECS % THREADS == 0, "whole vectors for each thread");
    u32x4 x[EACH];
    uint32_t offset[EACH];
    __device__ __forceinline__ void place(int tid, int64_t row_bytes) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = tid + j * THREADS;
            offset[j] = (uint32_t)(i / VECS) * (uint32_t)row_bytes + (uint32_t)(i % VECS * 16);
        }
    }
    __device__ __forceinline__ void load(const char* first_row, int tid, int n, int D) {
        if (n >= BN && D == DP) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) x[j] = *reinterpret_cast<const u32x4*>(first_row + offset[j]);
        } else {
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int i = tid + j * THREADS;
                x[j] = u32x4{0, 0, 0, 0};
                if (i / VECS < n && i % VECS * V < D) x[j] = *reinterpret_cast<const u32x4*>(first_row + offset[j]);
            }
        }
    }
    template <class RowAt>
    __device__ __forceinline__ void load_rows(int tid, int n, int D, RowAt row_at) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = tid + j * THREADS, r = i / VECS, d = i % VECS * V;
            x[j] = u32x4{0, 0, 0, 0};
            if (r < n && d < D) x[j] = *reinterpret_cast<const u32x4*>(row_at(r) + d * sizeof(T));
        }
    }
    __device__ __forceinline__ void store(int tid, typename M::E* tile) const {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = tid + j * THREADS;
            M::keep(tile, i / VECS, i % VECS, x[j]);
        }
    }
};

// A coordinate as it counts: within 5e18, so that the squares of a distance, (2 * 5e18)^2 three times, stay below 3.4e38.  Otherwise a key far away
// (a place that says "not there") would have an infinite distance, which its weight of 0, or a slope of 0, turns into a NaN.  NaN stays NaN.
constexpr float MOST_PLACE = 5e18f;
__device__ __forceinline__ float place_of(float x) { return fabsf(x) > MOST_PLACE ? copysignf(MOST_PLACE, x) : x; }

// The places of BN tokens likewise, into three lines of BN.
template <int BN, int THREADS>
struct PlaceTransfer {
    static constexpr int EACH = (3 * BN + THREADS - 1) / THREADS;
    float x[EACH];
    __device__ __forceinline__ void load(int tid, int n, const float* pos) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = tid + j * THREADS;
            x[j] = i < 3 * n ? pos[i] : 0.0f;
        }
    }
    __device__ __forceinline__ void store(int tid, float* place) const {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int i = tid + j * THREADS;
            if (i < 3 * BN) place[i % 3 * BN + i / 3] = place_of(x[j]);
        }
    }
};

// Orders a tile's stores before the reads of it (and those before the next stores): of a whole workgroup, or of one wave alone.
template <bool WORKGROUP>
__device__ __forceinline__ void tile_sync() {
    if constexpr (WORKGROUP) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// p (products q . k) -> scores minus base; SLACK: slack = 1 - tanh^2.  The tanh of an argument x up to 1 is an odd polynomial (relative
// error 8e-8; scores are rarely near their cap), beyond that 1 - 2 / (1 + e^2|x|) with the sign of x, whose absolute error of 1e-7 is then a relative one.
// Which form an element gets goes by the element alone, so that a row's result does not depend on the rows beside it; the
// vote only leaves the second form out where no element of the wave needs it.
// The largest argument's size of a lane; beyond 1 in any lane of the wave (`__any`), FAR is asked for.
__device__ __forceinline__ float cap_arguments(f32x16& p, const DenseScore& A, float far) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        p[i] *= A.in;
        far = fmaxf(far, fabsf(p[i]));
    }
    return far;
}
// p: arguments -> scores minus base.
template <bool SLACK, bool FAR>
__device__ __forceinline__ void cap_values(f32x16& p, f32x16& slack, const DenseScore& A, float base) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float x = p[i], y = x * x;
        float t = A.c[7];
#pragma unroll
        for (int k = 6; k >= 0; --k) t = t * y + A.c[k];
        if (SLACK) {
            const float v = x * t, th = v * A.inv_out;
            slack[i] = 1.0f - th * th;
            p[i] = v - base;
        } else {
            p[i] = x * t - base;
        }
        if (FAR) {
            // from |x|: r is at most 0.12 then, and 1 - r keeps its precision at either sign
            const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(fabsf(x) * (2.0f * LOG2E)));
            if (fabsf(x) > 1.0f) {
                if (SLACK) slack[i] = 4.0f * r * (1.0f - r);       // 1 - (1 - 2 r)^2
                p[i] = copysignf((1.0f - 2.0f * r) * A.out, x) - base;
            }
        }
    }
}
__device__ __forceinline__ void plain_scores(f32x16& p, const DenseScore& A, float base) {
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = p[i] * A.in - base;
}
template <bool SLACK>
__device__ __forceinline__ void cap_scores(f32x16& p, f32x16& slack, const DenseScore& A, float base) {
    if (!A.capped) {
        plain_scores(p, A, base);
        if (SLACK) {
#pragma unroll
            for (int i = 0; i < 16; ++i) slack[i] = 1.0f;
        }
        return;
    }
    if (!__any(cap_arguments(p, A, 0.0f) > 1.0f)) cap_values<SLACK, false>(p, slack, A, base);
    else cap_values<SLACK, true>(p, slack, A, base);
}

// The same with tanh x = 1 - 2 / (1 + e^2x) everywhere: 7 issue slots an element (the exponential and the reciprocal take two each)
// where the polynomial and its vote take 11.  Its absolute error, 2^-23 of the cap whatever the score, shifts a weight by 2^-15 at a cap of
// 128, as the weights' own rounding for the matrix cores does: it is for results in bf16 and caps up to that (at 2^20 it is 10 % of a weight).
constexpr float COARSE_CAP = 128.0f;
__device__ __forceinline__ void cap_scores_coarse(f32x16& p, const DenseScore& A, float base) {
    if (!A.capped) {
        plain_scores(p, A, base);
        return;
    }
    const float in = A.in * (2.0f * LOG2E), out = -2.0f * A.out, over = A.out - base;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(p[i] * in)) * out + over;
}

// The running reference of a row's softmax moves to the first tile's maximum, and later when scores pass it by 2^8 (sums of weights up to
// 2^8 lose nothing in binary32 or bf16), so that the sums are rescaled rarely.  p holds scores minus base and gets those minus the new
// reference.  Returns whether any row's moved; `shrink` is then the factor of what a row has summed so far.
__device__ __forceinline__ float reference_base(float top) { return top > -INFINITY ? top : 0.0f; }
__device__ __forceinline__ bool move_reference(f32x16& p, float& top, float& shrink) {
    float most = p[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, p[i]);
    most = fmaxf(most, other_half(most));
    const bool unset = top == -INFINITY, moves = unset ? most > -INFINITY : most > 8.0f;
    if (!__any(moves)) return false;
    const float up = moves ? most : 0.0f;
    shrink = !moves ? 1.0f : unset ? 0.0f : __builtin_amdgcn_exp2f(-up);
    if (moves) top = reference_base(top) + up;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] -= up;
    return true;
}

// Distances of a lane's row to the tile's keys `at` .. `at` + 3, whose places lie in three lines of BN.
template <int BN>
__device__ __forceinline__ f32x4 key_distances(float x, float y, float z, const float* place, int at) {
    const f32x4 px = *reinterpret_cast<const f32x4*>(place + at), py = *reinterpret_cast<const f32x4*>(place + BN + at),
                pz = *reinterpret_cast<const f32x4*>(place + 2 * BN + at);
    f32x4 d;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float dx = x - px[e], dy = y - py[e], dz = z - pz[e];
        d[e] = __builtin_amdgcn_sqrtf(dx * dx + dy * dy + dz * dz);
    }
    return d;
}

// p -= slope * distance; `at`: the lane's first key.
template <int BN>
__device__ __forceinline__ void bias_scores(f32x16& p, float x, float y, float z, float slope, const float* place, int at) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const f32x4 d = key_distances<BN>(x, y, z, place, at + 8 * b);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * b + e] -= slope * d[e];
    }
}

// 32 x 32 features of a wave's accumulators, transposed: lane l holds row l % 32, features 8 (i/4) + 4 (l/32) + i % 4.
// The first of the features is d0 of the row's D.
template <typename T, int DP>
__device__ __forceinline__ void store_row(char* row, const f32x16 (&acc)[DP / 32], float factor, int D, int half, int d0 = 0) {
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int d = d0 + dt * 32 + 8 * b + 4 * half;
            if (d >= D) continue;
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[dt][4 * b + e] * factor;
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<f32x4*>(row + d * 4) = x;
            } else {
                const u32x2 y = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
                *reinterpret_cast<u32x2*>(row + d * 2) = y;
            }
        }
}


}  // namespace e2f
