// Attention among all atoms of a segment, forward: one pass over the keys with the running maximum and sum of the softmax.
#include <initializer_list>
#include <type_traits>

#include "e2f_dense_api.h"

namespace {

using namespace e2f;

// ROWW waves of a workgroup own 32 rows each and share a tile of keys; or KEYW waves own the same 32 rows, take turns at
// the tiles (each with LDS of its own) and join at the end.  Workgroups with the same blockIdx.x and another blockIdx.y take
// parts of the keys, joined by k_dense_join.
template <typename T, int DP, int ROWW, int KEYW>
struct FwdShape {
    using M = Mma<T, DP>;
    static constexpr int BN = ROWW > 1 && sizeof(T) == 2 ? 64 : 32, BM = 32 * ROWW, THREADS = 64 * ROWW * KEYW, STAGERS = 64 * ROWW;
    struct Tile {
        typename M::E k[BN * M::LD], v[BN * M::LD];
        float place[3 * BN];
    };
};

// COARSE: the tanh by exponential and reciprocal, for results in bf16 (see cap_scores_coarse).
template <typename T, int DP, int ROWW, int KEYW, bool COARSE>
__global__ __launch_bounds__(64 * ROWW * KEYW, ROWW == 1 && DP * sizeof(T) > 128 ? 1 : 2) void k_dense_fwd(DenseParams A) {
    using F = FwdShape<T, DP, ROWW, KEYW>;
    using M = typename F::M;
    constexpr int BN = F::BN;
    __shared__ __align__(16) typename F::Tile tiles[KEYW];
    __shared__ float joint[KEYW > 1 ? KEYW : 1][2][32];
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int roww = ROWW > 1 ? wave : 0, keyw = KEYW > 1 ? wave : 0, tid = KEYW > 1 ? lane : threadIdx.x;
    typename F::Tile& tile = tiles[keyw];
    const int head_k = blockIdx.x % A.Hk;
    const int64_t t_index = blockIdx.x / A.Hk;
    const Segment segment = segment_of<false>(A, F::BM, t_index);
    const int q0 = segment.q0, nq = segment.nq, k0 = segment.k0, nk = segment.nk;
    const int64_t row0 = (t_index - segment.first) * F::BM, rows = (int64_t)nq * A.group;
    if (row0 < 0 || row0 >= rows) return;
    const int64_t row = row0 + roww * 32 + (lane & 31);
    const bool valid = row < rows, busy = row0 + roww * 32 < rows;
    const int in_segment = valid ? A.over_group((uint32_t)row) : 0;
    const int query = q0 + in_segment, head = head_k * A.group + (valid ? (int)row - in_segment * A.group : 0);
    // this workgroup's part of the keys, in whole tiles
    const int parts = gridDim.y, n_tiles = (nk + BN - 1) / BN, each = (n_tiles + parts - 1) / parts;
    const int begin = min((int64_t)nk, (int64_t)blockIdx.y * each * BN), end = min((int64_t)nk, (int64_t)begin + (int64_t)each * BN);
    typename M::Frag qf;
    M::load(qf, A.q.row(query, head), A.D, valid, half);
    float x = 0, y = 0, z = 0, slope = 0;
    if (A.score.biased) {
        x = place_of(A.q_pos[(int64_t)query * 3]);
        y = place_of(A.q_pos[(int64_t)query * 3 + 1]);
        z = place_of(A.q_pos[(int64_t)query * 3 + 2]);
        slope = A.slope[head] * LOG2E;
    }
    f32x16 acc[DP / 32] = {};
    float top = -INFINITY, sum = 0;
    Transfer<M, DP, BN, F::STAGERS> tk, tv;
    PlaceTransfer<BN, F::STAGERS> tp;
    tk.place(tid, A.k.token_bytes);
    tv.place(tid, A.v.token_bytes);
    auto fetch = [&](int t) {
        const int n = end - t;
        tk.load(A.k.row(k0 + t, head_k), tid, n, A.D);
        tv.load(A.v.row(k0 + t, head_k), tid, n, A.D);
        if (A.score.biased) tp.load(tid, min(n, BN), A.k_pos + (int64_t)(k0 + t) * 3);
    };
    const int first = begin + keyw * BN;
    if (first < end) fetch(first);
    for (int t = first; t < end; t += KEYW * BN) {
        tile_sync<(ROWW > 1)>();
        tk.store(tid, tile.k);
        tv.store(tid, tile.v);
        if (A.score.biased) tp.store(tid, tile.place);
        tile_sync<(ROWW > 1)>();
        if (t + KEYW * BN < end) fetch(t + KEYW * BN);
        if (!busy) continue;
        const int n = min(BN, end - t);
        for (int m = 0; m < n; m += 32) {
            f32x16 p = M::dot(tile.k, m, qf, lane);
            if constexpr (COARSE) cap_scores_coarse(p, A.score, reference_base(top));
            else cap_scores<false>(p, p, A.score, reference_base(top));
            if (A.score.biased) bias_scores<BN>(p, x, y, z, slope, tile.place, m + 4 * half);
            if (n - m < 32) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (m + 8 * (i / 4) + 4 * half + i % 4 >= n) p[i] = -INFINITY;
            }
            float shrink;
            if (move_reference(p, top, shrink)) {
                sum *= shrink;
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt) acc[dt] *= shrink;
            }
            float add = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(p[i]);
                add += p[i];
            }
            sum += add;
            M::accumulate(acc, tile.v, m, M::weights(p), lane);
        }
    }
    sum += other_half(sum);
    if constexpr (KEYW > 1) {
        // over the waves, in order; a wave without keys has a reference of -inf and a sum of 0
        joint[keyw][0][lane & 31] = top;
        joint[keyw][1][lane & 31] = sum;
        __syncthreads();
        float best = -INFINITY;
#pragma unroll
        for (int w = 0; w < KEYW; ++w) best = fmaxf(best, joint[w][0][lane & 31]);
        const float mine = best > -INFINITY ? __builtin_amdgcn_exp2f(top - best) : 0.0f;
        float total = 0;
#pragma unroll
        for (int w = 0; w < KEYW; ++w)
            total += joint[w][1][lane & 31] * (best > -INFINITY ? __builtin_amdgcn_exp2f(joint[w][0][lane & 31] - best) : 0.0f);
        float* all = reinterpret_cast<float*>(tiles);       // [KEYW][16][64] of one 32 x 32 block at a time
        static_assert(sizeof(tiles) >= KEYW * 1024 * 4, "room for a block of every wave");
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 16; ++i) all[(keyw * 16 + i) * 64 + lane] = acc[dt][i] * mine;
            __syncthreads();
            if (keyw == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float a = all[i * 64 + lane];
#pragma unroll
                    for (int w = 1; w < KEYW; ++w) a += all[(w * 16 + i) * 64 + lane];
                    acc[dt][i] = a;
                }
            }
        }
        top = best;
        sum = total;
        if (keyw != 0) return;
    }
    if (!valid) return;
    if (parts == 1) {
        store_row<T, DP>(A.out.row(query, head), acc, nk > 0 ? 1.0f / sum : 0.0f, A.D, half);
    } else {
        const int64_t at = ((int64_t)blockIdx.y * A.Nq + query) * (A.Hk * A.group) + head;
        if (begin < end) store_row<float, DP>(reinterpret_cast<char*>(A.part + at * A.D), acc, 1.0f, A.D, half);
        if (half == 0) {
            A.part_sum[at * 2] = begin < end ? top : -INFINITY;
            A.part_sum[at * 2 + 1] = begin < end ? sum : 0.0f;
        }
    }
}

// Joins the parts of a row: out = sum_p 2^(top_p - top) part_p / sum_p 2^(top_p - top) sum_p.  For a few parts of many rows, a thread
// for four features of a row: 2 parts of 80 000 rows of 64 features, 53 MB with the result, in 21 us.
template <typename T>
__global__ __launch_bounds__(256) void k_dense_join_few(DenseParams A, int parts) {
    const int Hq = A.Hk * A.group, quads = A.D / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / quads, stride = (int64_t)A.Nq * Hq;
    if (row >= stride) return;
    const int d = (int)(i % quads) * 4, query = (int)(row / Hq);
    const int s = token_segment(A.q_offsets, A.S, query);
    int first, n, k_first, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, first, n);
    if (query < first || query >= first + n) return;
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k_first, nk);
    const f32x2* of = reinterpret_cast<const f32x2*>(A.part_sum) + row;
    float top = -INFINITY, sum = 0;
    for (int p = 0; p < parts; ++p) top = fmaxf(top, of[p * stride][0]);
    f32x4 a = {0, 0, 0, 0};
    for (int p = 0; p < parts; ++p) {
        const f32x2 r = of[p * stride];
        if (!(r[1] != 0.0f)) continue;       // no keys in this part, which then left nothing to read
        const float f = __builtin_amdgcn_exp2f(r[0] - top);
        sum += f * r[1];
        a += f * *reinterpret_cast<const f32x4*>(A.part + (p * stride + row) * A.D + d);
    }
    a = nk > 0 ? a / sum : f32x4{0, 0, 0, 0};
    char* to = A.out.row(query, row % Hq) + d * sizeof(T);
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(to) = a;
    else *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
}

// For more than JOIN_FEW parts of fewer than JOIN_ROWS rows, which do not fill the chip so, a workgroup for a row; its waves share the parts, a lane
// forms a part's factor, then all lanes walk over the features of the wave's parts, whose loads do not wait for each other.  Both ways, by rows
// and by threads: 8 rows of 64 features over 1 600 keys (6 parts) 14.2 and 13.3 us, 2 100 keys (8 parts) 14.0 and 14.3, 4 500 keys 14.4 and
// 18.3; over 60 000 keys 1 280 rows of 64 features 119 and 121, 1 600 rows 139 and 133 (of 32 or 128 features: 1 024 rows 91 and 103, 117
// and 129, 1 600 rows 128 and 122, 163 and 157), 2 400 rows 195 and 165.
constexpr int JOIN_WAVES = 16, JOIN_FEW = 8, JOIN_ROWS = 1400;
template <typename T>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_dense_join(DenseParams A, int parts) {
    __shared__ float sums[JOIN_WAVES][128], weight[JOIN_WAVES], best[JOIN_WAVES];
    const int Hq = A.Hk * A.group, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x, stride = (int64_t)A.Nq * Hq;
    const int query = (int)(row / Hq);
    const int s = token_segment(A.q_offsets, A.S, query);
    int first, n, k_first, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, first, n);
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k_first, nk);
    if (query < first || query >= first + n) return;
    const int each = (parts + JOIN_WAVES - 1) / JOIN_WAVES, p0 = wave * each, p1 = min(parts, p0 + each);
    float top = -INFINITY;
    for (int p = p0 + lane; p < p1; p += 64) top = fmaxf(top, A.part_sum[(p * stride + row) * 2]);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) best[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < JOIN_WAVES; ++w) top = fmaxf(top, best[w]);
    float a0 = 0, a1 = 0, sum = 0;
    for (int q = p0; q < p1; q += 64) {
        float f = 0;
        if (q + lane < p1) {
            const float* of = A.part_sum + ((q + lane) * stride + row) * 2;
            // a part without keys has a sum of 0 and left nothing to read
            f = of[1] != 0.0f ? __builtin_amdgcn_exp2f(of[0] - top) : -1.0f;
            if (f >= 0.0f || f != f) sum += f * of[1];
        }
        const int m = min(64, p1 - q);
        for (int i = 0; i < m; i += 16) {
            float x[16], y[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float* part = A.part + ((q + i + j) * stride + row) * A.D;
                const bool in = i + j < m && !(__shfl(f, i + j) < 0.0f);
                x[j] = in && lane < A.D ? part[lane] : 0.0f;
                y[j] = in && lane + 64 < A.D ? part[lane + 64] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float g = i + j < m ? __shfl(f, i + j) : -1.0f;
                a0 += g < 0.0f ? 0.0f : g * x[j];
                a1 += g < 0.0f ? 0.0f : g * y[j];
            }
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    sums[wave][lane] = a0;
    sums[wave][lane + 64] = a1;
    if (lane == 0) weight[wave] = sum;
    __syncthreads();
    if (threadIdx.x >= (unsigned)A.D) return;
    sum = 0;
    float a = 0;
#pragma unroll
    for (int w = 0; w < JOIN_WAVES; ++w) {
        sum += weight[w];
        a += sums[w][threadIdx.x];
    }
    a = nk > 0 ? a / sum : 0.0f;
    char* out = A.out.row(query, row % Hq);
    if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(out)[threadIdx.x] = a;
    else reinterpret_cast<uint16_t*>(out)[threadIdx.x] = (uint16_t)pack_bf16(a, 0.0f);
}

// Which form runs, from the sizes that the host knows.
struct FwdPlan {
    int roww, keyw, parts;
    int64_t tiles;
    bool coarse;
};
FwdPlan fwd_plan(const e2f_dense_args* a) {
    FwdPlan P = {4, 1, 1, 0, a->cap <= COARSE_CAP};
    const int group = a->Hq / a->Hk;
    const int64_t rows = (int64_t)a->Nq * group, S = a->S > 0 ? a->S : 1;
    if (rows <= 32 * S) {
        P.roww = 1;
        P.keyw = a->Nk > 128 * S ? 4 : 1;
    }
    P.tiles = dense_tiles(a->Nq, group, a->S, 32 * P.roww);
    if (P.tiles == 0) return P;
    const int64_t blocks = P.tiles * a->Hk, keys = a->Nk / S;
    if (P.roww == 4) {
        // two workgroups to a compute unit; a round over 10 000 keys with 64 (128) features takes 390 (590) us in bf16, 800 (1 500) in
        // fp32.  Parts instead of one: 10 000 atoms, 8 heads, 632 workgroups 776 -> 654 us with two (687 with three); 4 000 atoms in fp32,
        // 264 workgroups, 304 -> 243 with three; 40 (100) queries over 60 000 keys on 2 key heads 317 (315) us with eight parts, 58 (86)
        // with up to 64
        const double per_key = a->dtype == E2F_BF16 ? 0.02 + 0.0003 * a->D : 0.02 + 0.001 * a->D;
        P.parts = best_parts(blocks, 512, keys * per_key, rows * a->Hk * (a->D * 8.0) / 4.5e6, rows * a->Hk * (a->D / 4), keys / 256);
    } else {
        // a few rows: their keys over 2048 waves, each with two tiles at least
        int64_t parts = 2048 / (blocks * P.keyw);
        const int64_t most = keys / (64 * P.keyw);
        if (parts > most) parts = most;
        P.parts = parts > 1 ? (int)(parts < 1024 ? parts : 1024) : 1;
    }
    return P;
}

bool launches(const e2f_dense_args* a, const FwdPlan& P) { return e2f::launches(P.tiles * a->Hk, 64 * P.roww * P.keyw); }

template <typename T, int DP>
void launch_dp(const DenseParams& A, const FwdPlan& P, hipStream_t st) {
    const dim3 grid((unsigned)(P.tiles * A.Hk), (unsigned)P.parts);
    auto go = [&](auto coarse) {
        constexpr bool COARSE = decltype(coarse)::value;
        if (P.roww == 4) k_dense_fwd<T, DP, 4, 1, COARSE><<<grid, 256, 0, st>>>(A);
        else if (P.keyw == 4) k_dense_fwd<T, DP, 1, 4, COARSE><<<grid, 256, 0, st>>>(A);
        else k_dense_fwd<T, DP, 1, 1, COARSE><<<grid, 64, 0, st>>>(A);
    };
    if constexpr (sizeof(T) == 2) {
        if (P.coarse) go(std::true_type{});
        else go(std::false_type{});
    } else {
        go(std::false_type{});
    }
    const int64_t rows = (int64_t)A.Nq * A.Hk * A.group;
    if (P.parts > JOIN_FEW && rows < JOIN_ROWS) k_dense_join<T><<<(unsigned)rows, 64 * JOIN_WAVES, 0, st>>>(A, P.parts);
    else if (P.parts > 1) k_dense_join_few<T><<<(unsigned)((rows * (A.D / 4) + 255) / 256), 256, 0, st>>>(A, P.parts);
}

template <typename T>
void launch(const DenseParams& A, const FwdPlan& P, hipStream_t st) {
    if (A.D <= 32) launch_dp<T, 32>(A, P, st);
    else if (A.D <= 64) launch_dp<T, 64>(A, P, st);
    else if (A.D <= 96) launch_dp<T, 96>(A, P, st);
    else launch_dp<T, 128>(A, P, st);
}

size_t layout(const e2f_dense_args* a, const FwdPlan& P, char* ws, DenseParams* A) {
    if (P.parts == 1) return 0;
    const size_t rows = (size_t)P.parts * a->Nq * a->Hq, sums = e2f_align_up(rows * 2 * sizeof(float));
    if (A) {
        A->part_sum = reinterpret_cast<float*>(ws);
        A->part = reinterpret_cast<float*>(ws + sums);
    }
    return sums + e2f_align_up(rows * a->D * sizeof(float));
}

}  // namespace

namespace e2f {

e2f_status dense_check_sizes(const e2f_dense_args* a) {
    if (!a || (a->dtype != E2F_F32 && a->dtype != E2F_BF16) || a->Nq < 0 || a->Nk < 0 || a->S < 0 || a->Hq <= 0 || a->Hk <= 0 ||
        a->D <= 0 || a->Hq % a->Hk || !isfinite(a->scale) || !(a->cap >= 0.0f) || !isfinite(a->cap))
        return E2F_ERR_INVALID_ARG;
    if (a->D % 8 || a->D > 128 || a->Hq > 1024) return E2F_ERR_UNSUPPORTED;
    // far from where the constants of the tanh leave binary32
    if (a->cap > 0.0f && (a->cap < 0x1p-20f || a->cap > 0x1p20f)) return E2F_ERR_UNSUPPORTED;
    // the grid of either direction and the stacked rows of a segment are 31-bit numbers, and so are the counters that walk over rows and
    // keys by tiles, a step beyond their end
    const int64_t most = INT32_MAX / a->Hk;
    if ((int64_t)a->Nq * (a->Hq / a->Hk) > INT32_MAX - 1024 || a->Nk > INT32_MAX - 1024) return E2F_ERR_UNSUPPORTED;
    if (dense_tiles(a->Nq, a->Hq / a->Hk, a->S, 32) > most || dense_tiles(a->Nk, 1, a->S, 32) > most)
        return E2F_ERR_UNSUPPORTED;
    return E2F_OK;
}

e2f_status dense_check(const e2f_dense_args* a) {
    const e2f_status rc = dense_check_sizes(a);
    if (rc != E2F_OK) return rc;
    if (a->slope ? (a->Nq > 0 && !a->q_pos) || (a->Nk > 0 && !a->k_pos) : a->q_pos || a->k_pos) return E2F_ERR_INVALID_ARG;
    if (a->S > 0 && (!a->q_offsets || !a->k_offsets)) return E2F_ERR_INVALID_ARG;
    for (const void* p : {(const void*)a->q_offsets, (const void*)a->k_offsets, (const void*)a->q_lengths, (const void*)a->k_lengths,
                          (const void*)a->q_pos, (const void*)a->k_pos, (const void*)a->slope})
        if (!word_aligned(p)) return E2F_ERR_INVALID_ARG;
    return E2F_OK;
}

void dense_fill(DenseParams& A, const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v) {
    A = DenseParams{};
    A.q = rows_of(q, a->dtype);
    A.k = rows_of(k, a->dtype);
    A.v = rows_of(v, a->dtype);
    A.q_offsets = a->q_offsets;
    A.k_offsets = a->k_offsets;
    A.q_lengths = a->q_lengths;
    A.k_lengths = a->k_lengths;
    A.q_pos = a->q_pos;
    A.k_pos = a->k_pos;
    A.slope = a->slope;
    A.Nq = a->Nq;
    A.Nk = a->Nk;
    A.S = a->S;
    A.Hk = a->Hk;
    A.group = a->Hq / a->Hk;
    // r / group = r magic >> (31 + ceil(log2 group)) for 0 <= r < 2^31
    int bits = 0;
    while ((1 << bits) < A.group) ++bits;
    A.group_shift = 31 + bits;
    A.group_magic = (uint32_t)((1ull << A.group_shift) / A.group + 1);
    A.D = a->D;
    A.scale = a->scale;
    DenseScore& s = A.score;
    s.capped = a->cap > 0.0f;
    s.biased = a->slope != nullptr;
    s.in = s.capped ? a->scale / a->cap : (float)((double)a->scale * 1.4426950408889634);
    const double out = (double)a->cap * 1.4426950408889634;
    s.out = (float)out;
    s.inv_out = s.capped ? (float)(1.0 / out) : 0.0f;
    // tanh x / x as a polynomial of x^2 on [0, 1], its relative error 4e-9 at most (minimised over the interval)
    static const double tanh_c[8] = {0.99999999577764732,   -0.33333278673333597, 0.13332159672365009,    -0.053870912721773931,
                                     0.021464820153790358, -0.0079174443902042118, 0.0022822293973515737, -0.00035334546706570396};
    for (int i = 0; i < 8; ++i) s.c[i] = (float)(out * tanh_c[i]);
}

}  // namespace e2f

extern "C" {

size_t e2f_dense_attn_workspace_bytes(const e2f_dense_args* a) {
    if (dense_check_sizes(a) != E2F_OK) return 0;
    const FwdPlan P = fwd_plan(a);
    return launches(a, P) ? layout(a, P, nullptr, nullptr) : 0;
}

e2f_status e2f_dense_attn_forward(const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v,
                                  const e2f_heads* out, void* ws, size_t ws_bytes, void* hip_stream) {
    e2f_status rc = dense_check(a);
    if (rc != E2F_OK) return rc;
    if ((rc = check_rows(q, a->dtype, a->Nq, a->Hq)) != E2F_OK || (rc = check_rows(k, a->dtype, a->Nk, a->Hk)) != E2F_OK ||
        (rc = check_rows(v, a->dtype, a->Nk, a->Hk)) != E2F_OK ||
        (rc = check_result_rows(out, a->dtype, a->Nq, a->Hq, a->D)) != E2F_OK)
        return rc;
    const FwdPlan P = fwd_plan(a);
    if (!launches(a, P)) return E2F_ERR_UNSUPPORTED;
    const size_t need = layout(a, P, nullptr, nullptr);
    if (need && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < need) return E2F_ERR_WORKSPACE_TOO_SMALL;
    if (a->Nq == 0 || a->S == 0) return E2F_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    DenseParams A;
    dense_fill(A, a, q, k, v);
    A.out = rows_of(out, a->dtype);
    layout(a, P, static_cast<char*>(ws), &A);
    if (a->dtype == E2F_BF16) launch<uint16_t>(A, P, st);
    else launch<float>(A, P, st);
    E2F_HIP_CHECK(hipGetLastError());
    return E2F_OK;
}

}  // extern "C"
