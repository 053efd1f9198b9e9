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
#include "e2f_block.h"

namespace e2f {

constexpr int DENSE_THREADS = 256;
constexpr int DENSE_BM = 128;      // rows of a workgroup
constexpr float LOG2E = 1.4426950408889634f;

struct DenseParams {
    Rows q, k, v, out;             // out: out, or grad_q
    Rows go, gk, gv;               // backward: dL/dout, grad_k, grad_v
    const int32_t *q_offsets, *k_offsets, *q_lengths, *k_lengths;
    const float *q_pos, *k_pos, *slope;
    int32_t Nq, Nk, S, Hk, group, D;
    float scale, cap;
    float4* stats;                 // backward: [Nq][Hq] softmax reference (base 2), 1 / sum, delta
    float *slope_part;             // [Nq][Hq]
    float *q_pos_part, *k_pos_part;   // [Hq][Nq][3], [Hk][Nk][3]
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
__device__ __forceinline__ int64_t first_tile(const int32_t* offsets, int s, int N, int group, int BM) {
    return (int64_t)min(max(offsets[s], 0), N) * group / BM + s;
}
static inline int64_t dense_tiles(int64_t N, int group, int S, int BM) { return N * group / BM + S; }

__device__ __forceinline__ int segment_of(const int32_t* offsets, int S, int N, int group, int BM, int64_t tile) {
    int lo = 0, n = S;             // the answer lies in [lo, lo + n)
    const int lane = threadIdx.x & 63;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        const bool before = lane * step < n && first_tile(offsets, at, N, group, BM) <= tile;
        const int k = __popcll(__ballot(before));          // candidate 0 always counts
        const int next = lo + (k ? k - 1 : 0) * step;
        n = min(step, lo + n - next);
        lo = next;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Matrix instructions and operands of the two feature types.  DP: D rounded up to 32, zero beyond D.
template <typename T, int DP>
struct Mma;

// bf16: v_mfma_f32_32x32x16_bf16, lane l: row l % 32, summands 8 (l/32) .. +7
template <int DP>
struct Mma<uint16_t, DP> {
    using T = uint16_t;
    static constexpr int STEPS = DP / 16, BN = 64, LD = DP + 8, LDT = BN + 8;
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
    // C += A B^T over the features: A 32 rows of a tile in LDS
    static __device__ __forceinline__ f32x16 dot(const T* tile, int row0, const Frag& b, int lane) {
        f32x16 acc = {};
        const T* p = tile + (row0 + (lane & 31)) * LD + 8 * (lane >> 5);
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(p + 16 * c), b.x[c], acc, 0, 0, 0);
        return acc;
    }
    // weights of 32 tile rows as an operand of products over those rows
    struct Weights {
        bf16x8 x[2];
    };
    static __device__ __forceinline__ Weights weights(const f32x16& p) {
        Weights w;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            u32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = pack_bf16(p[8 * c + 2 * e], p[8 * c + 2 * e + 1]);
            w.x[c] = __builtin_bit_cast(bf16x8, x);
        }
        return w;
    }
    // acc[dt] += (features dt*32.. of the tile, transposed) W over the 32 tile rows from row0; `turned` is the transposed tile
    static __device__ __forceinline__ void accumulate(f32x16 (&acc)[DP / 32], const T*, const T* turned, int row0, const Weights& w, int lane) {
        const T* p = turned + (lane & 31) * LDT + row0 + 4 * (lane >> 5);
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const u32x2 a = *reinterpret_cast<const u32x2*>(p + dt * 32 * LDT + 16 * c);
                const u32x2 b = *reinterpret_cast<const u32x2*>(p + dt * 32 * LDT + 16 * c + 8);
                const u32x4 ab = {a[0], a[1], b[0], b[1]};
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ab), w.x[c], acc[dt], 0, 0, 0);
            }
    }
    static constexpr int TILE = BN * LD, TURNED = DP * LDT;
    // four rows of eight features to the transposed tile
    static __device__ __forceinline__ void turn(T* turned, int row, int d, const u32x4 (&r)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // two features of four rows each
            const u32x2 even = {__builtin_amdgcn_perm(r[1][e], r[0][e], 0x05040100), __builtin_amdgcn_perm(r[3][e], r[2][e], 0x05040100)};
            const u32x2 odd = {__builtin_amdgcn_perm(r[1][e], r[0][e], 0x07060302), __builtin_amdgcn_perm(r[3][e], r[2][e], 0x07060302)};
            *reinterpret_cast<u32x2*>(turned + (d + 2 * e) * LDT + row) = even;
            *reinterpret_cast<u32x2*>(turned + (d + 2 * e + 1) * LDT + row) = odd;
        }
    }
};

// binary32: v_mfma_f32_32x32x2_f32, lane l: row l % 32, summand l / 32.  The order of the sum over the features is free as
// well: the lower half of the lanes takes the first DP/2 features, so that a lane's operands lie side by side.
template <int DP>
struct Mma<float, DP> {
    using T = float;
    static constexpr int BN = 32, LD = DP + 8, LDT = 0, H = DP / 2;
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
    static __device__ __forceinline__ void accumulate(f32x16 (&acc)[DP / 32], const T* tile, const T*, int row0, const Weights& w, int lane) {
        const T* p = tile + (row0 + 4 * (lane >> 5)) * LD + (lane & 31);
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(p[(8 * (i / 4) + i % 4) * LD + dt * 32], w.x[i], acc[dt], 0, 0, 0);
    }
    static constexpr int TILE = BN * LD, TURNED = 0;
};

// BN rows of a tile from memory into LDS, rows and features behind the end as zeros; PLAIN, TURNED: which of the two forms.
// row_at(r): the row's memory.
template <typename M, int DP, bool PLAIN, bool TURNED, class RowAt>
__device__ __forceinline__ void stage(typename M::T* plain, typename M::T* turned, int n, int D, RowAt row_at) {
    using T = typename M::T;
    constexpr int V = 16 / sizeof(T);
    if constexpr (sizeof(T) == 4 || !TURNED) {
        constexpr int VECS = DP / V;
        for (int i = threadIdx.x; i < M::BN * VECS; i += DENSE_THREADS) {
            const int r = i / VECS, d = i % VECS * V;
            u32x4 x = {0, 0, 0, 0};
            if (r < n && d < D) x = *reinterpret_cast<const u32x4*>(row_at(r) + d * sizeof(T));
            *reinterpret_cast<u32x4*>(plain + r * M::LD + d) = x;
        }
    } else {
        constexpr int VECS = DP / 8;
        for (int i = threadIdx.x; i < M::BN / 4 * VECS; i += DENSE_THREADS) {
            const int r = i / VECS * 4, d = i % VECS * 8;
            u32x4 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = u32x4{0, 0, 0, 0};
                if (r + e < n && d < D) x[e] = *reinterpret_cast<const u32x4*>(row_at(r + e) + d * 2);
                if (PLAIN) *reinterpret_cast<u32x4*>(plain + (r + e) * M::LD + d) = x[e];
            }
            M::turn(turned, r, d, x);
        }
    }
}

// Places of BN tokens, as three lines.
template <int BN>
__device__ __forceinline__ void stage_places(float* s, const float* pos, int64_t first, int n) {
    for (int i = threadIdx.x; i < 3 * BN; i += DENSE_THREADS) {
        const int r = i / 3, c = i % 3;
        s[c * BN + r] = r < n ? pos[first * 3 + i] : 0.0f;
    }
}

// 32 x 32 features of a wave's accumulators, transposed: lane l holds row l % 32, features 8 (i/4) + 4 (l/32) + i % 4.
template <typename T, int DP>
__device__ __forceinline__ void store_row(char* row, const f32x16 (&acc)[DP / 32], float factor, int D, int half) {
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int d = dt * 32 + 8 * b + 4 * half;
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

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

}  // namespace e2f
