// Attention among all atoms of a segment, backward.  With p the softmax weights, dp_ij = dout_i . v_j, th = tanh(x / cap):
//   delta_i = sum_j p dp;  ds = p (dp - delta);  dx = ds (1 - th^2)
//   dv_j = sum_i p dout_i;  dq_i = scale sum_j dx k_j;  dk_j = scale sum_i dx q_i
//   dslope_h = - sum ds d;  dr_i = - sum_{h,j} slope_h ds (r_i - r_j) / d,  dr_j the opposite
// Nothing of a pair is stored: a kernel over rows forms the softmax statistics and delta, a second one dq, a kernel over keys
// dk and dv.  Each sum is formed by the workgroup that owns its row or key, so no atomics are needed; where these are too few to
// fill the chip the other side is cut into parts, whose sums are joined in their order.  delta comes from the binary32 products
// and weights (not from the rounded result of the forward pass): the gradients of slope and places are binary32 and keep their
// precision.
#include <type_traits>

#include "e2f_dense_api.h"

namespace {

using namespace e2f;

constexpr int SUM_THREADS = 256;

// A distance and its reciprocal.  d^2 is kept from 0, so that a pair at one place has a finite reciprocal that the components of
// the difference, zero, annul.
__device__ __forceinline__ void distance(float dx, float dy, float dz, float& d, float& inv) {
    const float d2 = fmaxf(dx * dx + dy * dy + dz * dz, 1e-36f);
    inv = __builtin_amdgcn_rsqf(d2);
    d = d2 * inv;
}

// A workgroup's 32 ROWW rows of a (segment, key head), its part of the segment's keys (blockIdx.y), and the walk over them.  SHARE
// waves to a group of 32 rows: they take 32 keys of a tile each.
template <typename T, int DP, int ROWW, int SHARE>
struct RowWalk {
    using M = Mma<T, DP>;
    static constexpr int BN = SHARE > 1 ? 32 * SHARE : ROWW > 1 && sizeof(T) == 2 ? 64 : 32, BM = 32 * ROWW, THREADS = 64 * ROWW * SHARE;
    struct Tile {
        typename M::E k[BN * M::LD], v[BN * M::LD];
        float place[3 * BN];
    };
    int lane, half, group, share, head_k, k0, begin, end, query, head, first_head;
    int64_t at;            // of the row among [Nq][Hq]
    bool any, valid, busy;
    float x, y, z, slope;
    typename M::Frag qf, gf;

    __device__ __forceinline__ RowWalk(const DenseParams& A) {
        lane = threadIdx.x & 63;
        half = lane >> 5;
        group = (threadIdx.x >> 6) % ROWW;
        share = (threadIdx.x >> 6) / ROWW;
        head_k = blockIdx.x % A.Hk;
        const int64_t tile = blockIdx.x / A.Hk;
        const Segment segment = segment_of<false>(A, BM, tile);
        const int q0 = segment.q0, nq = segment.nq, nk = segment.nk;
        k0 = segment.k0;
        const int64_t row0 = (tile - segment.first) * BM, rows = (int64_t)nq * A.group;
        any = row0 >= 0 && row0 < rows;
        if (!any) return;
        first_head = (int)(row0 % A.group);
        const int64_t row = row0 + group * 32 + (lane & 31);
        valid = row < rows;
        busy = row0 + group * 32 < rows;
        const int in_segment = valid ? A.over_group((uint32_t)row) : 0;
        query = q0 + in_segment;
        head = head_k * A.group + (valid ? (int)row - in_segment * A.group : 0);
        at = (int64_t)query * (A.Hk * A.group) + head;
        const int tiles = (nk + BN - 1) / BN, each = (tiles + (int)gridDim.y - 1) / (int)gridDim.y;
        begin = (int)min((int64_t)nk, (int64_t)blockIdx.y * each * BN);
        end = (int)min((int64_t)nk, (int64_t)begin + (int64_t)each * BN);
        M::load(qf, A.q.row(query, head), A.D, valid, half);
        M::load(gf, A.go.row(query, head), A.D, valid, half);
        x = y = z = slope = 0;
        if (A.score.biased) {
            x = place_of(A.q_pos[(int64_t)query * 3]);
            y = place_of(A.q_pos[(int64_t)query * 3 + 1]);
            z = place_of(A.q_pos[(int64_t)query * 3 + 2]);
            slope = A.slope[head];
        }
    }
    // body(first row of 32 keys in the tile, how many of them count); with SHARE, body(whether the wave's rows count, ...) for each wave
    template <class Body>
    __device__ __forceinline__ void walk(const DenseParams& A, Tile& tile, Body body) {
        const int tid = threadIdx.x;
        Transfer<M, DP, BN, THREADS> tk, tv;
        PlaceTransfer<BN, THREADS> tp;
        tk.place(tid, A.k.token_bytes);
        tv.place(tid, A.v.token_bytes);
        auto fetch = [&](int t) {
            const int n = end - t;
            tk.load(A.k.row(k0 + t, head_k), tid, n, A.D);
            tv.load(A.v.row(k0 + t, head_k), tid, n, A.D);
            if (A.score.biased) tp.load(tid, min(n, BN), A.k_pos + (int64_t)(k0 + t) * 3);
        };
        if (begin < end) fetch(begin);
        for (int t = begin; t < end; t += BN) {
            __syncthreads();
            tk.store(tid, tile.k);
            tv.store(tid, tile.v);
            if (A.score.biased) tp.store(tid, tile.place);
            __syncthreads();
            if (t + BN < end) fetch(t + BN);
            const int n = min(BN, end - t);
            if constexpr (SHARE > 1) {
                body(32 * share, n - 32 * share);
            } else {
                if (!busy) continue;
                for (int m = 0; m < n; m += 32) body(m, n - m);
            }
        }
    }
    // keys behind the end: weight 0
    __device__ __forceinline__ void mask(f32x16& p, int n) const {
        if (n >= 32) return;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i / 4) + 4 * half + i % 4 >= n) p[i] = -INFINITY;
    }
};

// Softmax statistics of the rows: reference, sum, sum of p dp, sum of p d.  With parts of the keys each leaves its own, [parts][Nq][Hq].
// Workgroups of one wave get the registers of a SIMD from 256 bytes of features on, where two waves spill (1 000 x 30 atoms, 64 fp32 features:
// 531 us with two waves, 416 with one; 300 x 40 atoms in bf16 with 128 features 218 and 213, with 96 features 184 and 195).
template <typename T, int DP, int ROWW>
__global__ __launch_bounds__(64 * ROWW, ROWW == 1 && DP * sizeof(T) >= 256 ? 1 : 2) void k_dense_bwd_stats(DenseParams A) {
    using R = RowWalk<T, DP, ROWW, 1>;
    using M = typename R::M;
    __shared__ __align__(16) typename R::Tile tile;
    R w(A);
    if (!w.any) return;
    float top = -INFINITY, sum = 0, delta = 0, usual = 0;
    w.walk(A, tile, [&](int m, int n) {
        f32x16 p = M::dot(tile.k, m, w.qf, w.lane), d;
        const f32x16 dp = M::dot(tile.v, m, w.gf, w.lane);
        cap_scores<false>(p, p, A.score, reference_base(top));
        if (A.score.biased) {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 of = key_distances<R::BN>(w.x, w.y, w.z, tile.place, m + 4 * w.half + 8 * b);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[4 * b + e] = of[e];
                    p[4 * b + e] -= w.slope * LOG2E * of[e];
                }
            }
        }
        w.mask(p, n);
        float shrink;
        if (move_reference(p, top, shrink)) {
            sum *= shrink;
            delta *= shrink;
            usual *= shrink;
        }
        float add = 0, dot = 0, far = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = __builtin_amdgcn_exp2f(p[i]);
            add += p[i];
            dot += p[i] * dp[i];
        }
        if (A.score.biased) {
#pragma unroll
            for (int i = 0; i < 16; ++i) far += p[i] * d[i];
        }
        sum += add;
        delta += dot;
        usual += far;
    });
    sum += other_half(sum);
    delta += other_half(delta);
    usual += other_half(usual);
    if (!w.valid || w.half) return;
    if (gridDim.y == 1) {
        const float inv = w.begin < w.end ? 1.0f / sum : 0.0f;
        A.stats[w.at] = make_float4(top, inv, delta * inv, top - __builtin_amdgcn_logf(inv));
        if (A.score.biased) A.usual[w.at] = usual * inv;
    } else {
        A.stats_part[(int64_t)blockIdx.y * A.Nq * (A.Hk * A.group) + w.at] = make_float4(top, sum, delta, usual);
    }
}

// Joins the parts' statistics.  Rows that no segment covers hold anything and are not read by anyone.
__global__ __launch_bounds__(SUM_THREADS) void k_dense_bwd_join_stats(DenseParams A, int parts) {
    const int64_t rows = (int64_t)A.Nq * (A.Hk * A.group), row = (int64_t)blockIdx.x * SUM_THREADS + threadIdx.x;
    if (row >= rows) return;
    float top = -INFINITY, sum = 0, delta = 0, usual = 0;
    for (int p = 0; p < parts; ++p) top = fmaxf(top, A.stats_part[p * rows + row].x);
    for (int p = 0; p < parts; ++p) {
        const float4 s = A.stats_part[p * rows + row];
        const float f = top > -INFINITY ? __builtin_amdgcn_exp2f(s.x - top) : 1.0f;
        sum += f * s.y;
        delta += f * s.z;
        usual += f * s.w;
    }
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;      // no keys: no weights
    A.stats[row] = make_float4(top, inv, delta * inv, top - __builtin_amdgcn_logf(inv));
    if (A.score.biased) A.usual[row] = usual * inv;
}

// dq and a row's shares of the gradients of slope and place, from the statistics.  SHARE waves to a group of rows pass each other the weights and
// keep the sums of DP / SHARE features each, as in the kernel over keys.
template <typename T, int DP, int ROWW, int SHARE>
__global__ __launch_bounds__(64 * ROWW * SHARE, ROWW == 1 && DP * sizeof(T) > 128 ? 1 : 2) void k_dense_bwd_rows(DenseParams A) {
    using R = RowWalk<T, DP, ROWW, SHARE>;
    using M = typename R::M;
    constexpr int BN = R::BN, NT = DP / SHARE / 32;
    __shared__ __align__(16) typename R::Tile tile;
    __shared__ __align__(16) u32x4 passed[SHARE > 1 ? ROWW * SHARE : 1][SHARE > 1 ? M::WEIGHT_VECTORS * 64 : 1];
    R w(A);
    const int Hq = A.Hk * A.group;
    float* slopes = A.slope_part ? A.slope_part + ((int64_t)blockIdx.y * (gridDim.x / A.Hk) + blockIdx.x / A.Hk) * Hq + w.head_k * A.group : nullptr;
    if (!w.any) {
        if (slopes)
            for (int g = threadIdx.x; g < A.group; g += R::THREADS) slopes[g] = 0.0f;
        return;
    }
    const float4 st = A.stats[w.at];
    const float top = st.x, inv = st.y, delta = st.z, slope2 = w.slope * LOG2E;
    // weights stay without 1 / sum: a row's sums get it at the end
    float dslope = 0, gx = 0, gy = 0, gz = 0;
    // a row's ds sum up to nothing, so that any distance may be taken off all of its distances: with the mean distance under the row's
    // weights the rounding of delta, a multiple of those weights in ds, drops out of the sum of ds d
    const float usual = A.score.biased ? A.usual[w.at] : 0.0f;
    f32x16 acc[NT] = {};
    auto weigh = [&](int m, int n) {
        f32x16 p = M::dot(tile.k, m, w.qf, w.lane), slack;
        const f32x16 dp = M::dot(tile.v, m, w.gf, w.lane);
        cap_scores<true>(p, slack, A.score, top);
        w.mask(p, n);
        if (A.score.biased) {
            float ts = 0, tx = 0, ty = 0, tz = 0;      // a tile's sums by themselves: shorter sums, smaller errors
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float* at = tile.place + m + 4 * w.half + 8 * b;
                const f32x4 px = *reinterpret_cast<const f32x4*>(at), py = *reinterpret_cast<const f32x4*>(at + BN),
                            pz = *reinterpret_cast<const f32x4*>(at + 2 * BN);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * b + e;
                    const float dx = w.x - px[e], dy = w.y - py[e], dz = w.z - pz[e];
                    float d, id;
                    distance(dx, dy, dz, d, id);
                    p[i] = __builtin_amdgcn_exp2f(p[i] - slope2 * d) * (dp[i] - delta);
                    ts += p[i] * (d - usual);
                    const float f = p[i] * id;
                    tx += f * dx;
                    ty += f * dy;
                    tz += f * dz;
                }
            }
            dslope += ts;
            gx += tx;
            gy += ty;
            gz += tz;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(p[i]) * (dp[i] - delta);
        }
        if (A.score.capped) {
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] *= slack[i];
        }
        return M::weights(p);
    };
    if constexpr (SHARE == 1) {
        w.walk(A, tile, [&](int m, int n) { M::accumulate(acc, tile.k, m, weigh(m, n), w.lane); });
    } else {
        w.walk(A, tile, [&](int m, int n) {
            if (w.busy) M::put(&passed[w.share * ROWW + w.group][w.lane], weigh(m, n));
            __syncthreads();
            if (w.busy) {
#pragma unroll
                for (int u = 0; u < SHARE; ++u)
                    M::accumulate(acc, tile.k + w.share * NT * 32, 32 * u, M::get(&passed[u * ROWW + w.group][w.lane]), w.lane);
            }
        });
    }
    dslope += other_half(dslope);
    gx += other_half(gx);
    gy += other_half(gy);
    gz += other_half(gz);
    float* sums = reinterpret_cast<float*>(&tile);      // [SHARE][4][BM]
    static_assert(sizeof(tile) >= SHARE * 4 * R::BM * 4, "room for the rows' sums");
    if (SHARE > 1 || slopes) {
        __syncthreads();
        if (!w.half) {
            float* to = sums + w.share * 4 * R::BM + w.group * 32 + w.lane;
            to[0] = w.valid ? -dslope * inv : 0.0f;
            to[R::BM] = gx;
            to[2 * R::BM] = gy;
            to[3 * R::BM] = gz;
        }
        __syncthreads();
    }
    if (SHARE > 1 && w.share == 0 && !w.half) {
#pragma unroll
        for (int u = 1; u < SHARE; ++u) {
            const float* from = sums + u * 4 * R::BM + w.group * 32 + w.lane;
            gx += from[R::BM];
            gy += from[2 * R::BM];
            gz += from[3 * R::BM];
        }
    }
    if (slopes) {
        // over the workgroup's rows, for each head of the group, in their order
        for (int g = threadIdx.x; g < A.group; g += R::THREADS) {
            float sum = 0;
            for (int u = 0; u < SHARE; ++u)
                for (int r = g >= w.first_head ? g - w.first_head : g - w.first_head + A.group; r < R::BM; r += A.group) sum += sums[u * 4 * R::BM + r];
            slopes[g] = sum;
        }
    }
    if (!w.valid) return;
    const int64_t at = (int64_t)blockIdx.y * A.Nq * Hq + w.at;
    const int d0 = w.share * NT * 32;
    if (gridDim.y == 1) store_row<T, NT * 32>(A.out.row(w.query, w.head), acc, A.scale * inv, A.D, w.half, d0);
    else store_row<float, NT * 32>(reinterpret_cast<char*>(A.gq_part + at * A.D), acc, A.scale * inv, A.D, w.half, d0);
    if (w.half || w.share) return;
    if (A.q_pos_part) {
        float* g = A.q_pos_part + (((int64_t)blockIdx.y * Hq + w.head) * A.Nq + w.query) * 3;
        g[0] = -w.slope * inv * gx;
        g[1] = -w.slope * inv * gy;
        g[2] = -w.slope * inv * gz;
    }
}

// What the kernel over keys needs of a row, as lines of BN in LDS: place, slope in base-2 units, and with lse = reference + log2(sum) the
// weight is one exponential (the rounding of lse, 2^-24 of it, scales a row's weights alike).
enum { ROW_X, ROW_Y, ROW_Z, ROW_SLOPE, ROW_LSE, ROW_DELTA, ROW_LINES };

// CAP, BIAS: what the scores have.  KEYW groups of 32 keys a workgroup, SHARE waves to a group: they take a block of 32 rows each of a
// tile, pass each other the weights through LDS and keep the sums of DP / SHARE features each.  With 128 features one wave's operands and sums
// take more registers than leave room for a second wave on its SIMD.
template <typename T, int DP, int KEYW, int SHARE, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * KEYW * SHARE, KEYW == 1 && DP * sizeof(T) > 128 ? 1 : 2) void k_dense_bwd_keys(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = SHARE > 1 ? 32 * SHARE : KEYW > 1 && sizeof(T) == 2 ? 64 : 32, BM = 32 * KEYW, THREADS = 64 * KEYW * SHARE;
    constexpr int NT = DP / SHARE / 32;
    __shared__ __align__(16) typename M::E qs[BN * M::LD];
    __shared__ __align__(16) typename M::E gs[BN * M::LD];
    __shared__ __align__(16) float par[ROW_LINES][BN];
    __shared__ __align__(16) u32x4 passed[SHARE > 1 ? KEYW * SHARE : 1][2][SHARE > 1 ? M::WEIGHT_VECTORS * 64 : 1];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = (tid >> 6) % KEYW, share = (tid >> 6) / KEYW;
    const int head_k = blockIdx.x % A.Hk, Hq = A.Hk * A.group;
    const int64_t tile = blockIdx.x / A.Hk;
    const Segment segment = segment_of<true>(A, BM, tile);
    const int q0 = segment.q0, nq = segment.nq, k0 = segment.k0, nk = segment.nk;
    const int64_t first = (tile - segment.first) * BM;
    const int rows = nq * A.group;
    if (first < 0 || first >= nk) return;
    const int mine = (int)first + wave * 32 + (lane & 31);
    const bool valid = mine < nk, busy = (int)first + wave * 32 < nk;
    const int key = k0 + (valid ? mine : 0);
    typename M::Frag kf, vf;
    M::load(kf, A.k.row(key, head_k), A.D, valid, half);
    M::load(vf, A.v.row(key, head_k), A.D, valid, half);
    float x = 0, y = 0, z = 0;
    if (BIAS) {
        x = place_of(A.k_pos[(int64_t)key * 3]);
        y = place_of(A.k_pos[(int64_t)key * 3 + 1]);
        z = place_of(A.k_pos[(int64_t)key * 3 + 2]);
    }
    // this workgroup's part of the rows
    const int row_tiles = (rows + BN - 1) / BN, each = (row_tiles + (int)gridDim.y - 1) / (int)gridDim.y;
    const int begin = (int)min((int64_t)rows, (int64_t)blockIdx.y * each * BN), end = (int)min((int64_t)rows, (int64_t)begin + (int64_t)each * BN);
    Transfer<M, DP, BN, THREADS> tq, tg;
    float4 st;
    float rx = 0, ry = 0, rz = 0, rs = 0;
    auto fetch = [&](int t) {
        const int n = end - t;
        auto at = [&](const Rows& R, int r) {
            const int query = A.over_group((uint32_t)(t + r));
            return R.row(q0 + query, head_k * A.group + (t + r - query * A.group));
        };
        tq.load_rows(tid, n, A.D, [&](int r) { return at(A.q, r); });
        tg.load_rows(tid, n, A.D, [&](int r) { return at(A.go, r); });
        st = make_float4(0, 0, 0, INFINITY);        // rows behind the end: weight 0
        if (tid < n && tid < BN) {
            const int in_segment = A.over_group((uint32_t)(t + tid)), head = head_k * A.group + (t + tid - in_segment * A.group);
            const int64_t query = q0 + in_segment;
            st = A.stats[query * Hq + head];
            if (BIAS) {
                rx = A.q_pos[query * 3];
                ry = A.q_pos[query * 3 + 1];
                rz = A.q_pos[query * 3 + 2];
                rs = A.slope[head] * LOG2E;
            }
        }
    };
    float gx = 0, gy = 0, gz = 0;
    f32x16 dk[NT] = {}, dv[NT] = {};
    // weights of 32 rows from row m of the tile, left in p (for dv) and ds (for dk)
    auto weigh = [&](int m, f32x16& p, f32x16& ds) {
        p = M::dot(qs, m, kf, lane);
        ds = M::dot(gs, m, vf, lane);
        f32x16 slack;
        if (CAP) cap_scores<true>(p, slack, A.score, 0.0f);
        else plain_scores(p, A.score, 0.0f);
        float tx = 0, ty = 0, tz = 0;      // a tile's sums by themselves: shorter sums, smaller errors
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            auto line = [&](int l) { return *reinterpret_cast<const f32x4*>(&par[l][m + 4 * half + 8 * b]); };
            const f32x4 lse = line(ROW_LSE), delta = line(ROW_DELTA);
            f32x4 px, py, pz, slope;
            if (BIAS) {
                px = line(ROW_X);
                py = line(ROW_Y);
                pz = line(ROW_Z);
                slope = line(ROW_SLOPE);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 4 * b + e;
                float s = p[i] - lse[e], dx, dy, dz, d, id;
                if (BIAS) {
                    dx = px[e] - x;
                    dy = py[e] - y;
                    dz = pz[e] - z;
                    distance(dx, dy, dz, d, id);
                    s -= slope[e] * d;
                }
                p[i] = __builtin_amdgcn_exp2f(s);
                const float g = p[i] * (ds[i] - delta[e]);
                if (BIAS) {
                    const float f = g * slope[e] * id;
                    tx += f * dx;
                    ty += f * dy;
                    tz += f * dz;
                }
                ds[i] = CAP ? g * slack[i] : g;
            }
        }
        gx += tx;
        gy += ty;
        gz += tz;
    };
    if (begin < end) fetch(begin);
    for (int t = begin; t < end; t += BN) {
        __syncthreads();
        tq.store(tid, qs);
        tg.store(tid, gs);
        if (tid < BN) {
            par[ROW_X][tid] = place_of(rx);
            par[ROW_Y][tid] = place_of(ry);
            par[ROW_Z][tid] = place_of(rz);
            par[ROW_SLOPE][tid] = rs;
            par[ROW_LSE][tid] = st.w;
            par[ROW_DELTA][tid] = st.z;
        }
        __syncthreads();
        if (t + BN < end) fetch(t + BN);
        if constexpr (SHARE == 1) {
            if (!busy) continue;
            const int n = min(BN, end - t);
#pragma unroll 1
            for (int m = 0; m < n; m += 32) {
                f32x16 p, ds;
                weigh(m, p, ds);
                M::accumulate(dv, gs, m, M::weights(p), lane);
                M::accumulate(dk, qs, m, M::weights(ds), lane);
            }
        } else {
            if (busy) {
                f32x16 p, ds;
                weigh(32 * share, p, ds);
                M::put(&passed[share * KEYW + wave][0][lane], M::weights(p));
                M::put(&passed[share * KEYW + wave][1][lane], M::weights(ds));
            }
            __syncthreads();
            if (busy) {
#pragma unroll
                for (int u = 0; u < SHARE; ++u) {
                    M::accumulate(dv, gs + share * NT * 32, 32 * u, M::get(&passed[u * KEYW + wave][0][lane]), lane);
                    M::accumulate(dk, qs + share * NT * 32, 32 * u, M::get(&passed[u * KEYW + wave][1][lane]), lane);
                }
            }
        }
    }
    gx += other_half(gx);
    gy += other_half(gy);
    gz += other_half(gz);
    if constexpr (SHARE > 1 && BIAS) {
        // the sharing waves' rows together, in their order
        float* g = reinterpret_cast<float*>(passed);
        __syncthreads();
        if (!half) {
            g[(share * KEYW + wave) * 96 + lane] = gx;
            g[(share * KEYW + wave) * 96 + 32 + lane] = gy;
            g[(share * KEYW + wave) * 96 + 64 + lane] = gz;
        }
        __syncthreads();
        if (!half && share == 0) {
#pragma unroll
            for (int u = 1; u < SHARE; ++u) {
                gx += g[(u * KEYW + wave) * 96 + lane];
                gy += g[(u * KEYW + wave) * 96 + 32 + lane];
                gz += g[(u * KEYW + wave) * 96 + 64 + lane];
            }
        }
    }
    if (!valid) return;
    const int d0 = share * NT * 32;
    if (gridDim.y == 1) {
        store_row<T, NT * 32>(A.gk.row(key, head_k), dk, A.scale, A.D, half, d0);
        store_row<T, NT * 32>(A.gv.row(key, head_k), dv, 1.0f, A.D, half, d0);
    } else {
        const int64_t at = (((int64_t)blockIdx.y * A.Nk + key) * A.Hk + head_k) * A.D;
        store_row<float, NT * 32>(reinterpret_cast<char*>(A.gk_part + at), dk, A.scale, A.D, half, d0);
        store_row<float, NT * 32>(reinterpret_cast<char*>(A.gv_part + at), dv, 1.0f, A.D, half, d0);
    }
    if (BIAS && A.k_pos_part && !half && share == 0) {
        float* g = A.k_pos_part + (((int64_t)blockIdx.y * A.Hk + head_k) * A.Nk + key) * 3;
        g[0] = gx * (1.0f / LOG2E);
        g[1] = gy * (1.0f / LOG2E);
        g[2] = gz * (1.0f / LOG2E);
    }
}

// Whether a segment's length covers a token.
__device__ __forceinline__ bool covered(const int32_t* offsets, const int32_t* lengths, int S, int N, int token) {
    int first, n;
    segment_range(offsets, lengths, token_segment(offsets, S, token), N, first, n);
    return token >= first && token < first + n;
}

// Sums of what parts and heads left of the gradients of places, for the covered tokens, and of the slopes' over the workgroups.
// Workgroups: first those of the queries, then of the keys (a thread for a token), then one for each slope.
__global__ __launch_bounds__(SUM_THREADS) void k_dense_bwd_sums(DenseParams A, float* gq, float* gk, float* gslope, int q_blocks, int k_blocks,
                                                                int row_parts, int key_parts, int64_t slope_lines) {
    const int Hq = A.Hk * A.group;
    int b = blockIdx.x;
    if (b < q_blocks + k_blocks) {
        const bool keys = b >= q_blocks;
        if (keys) b -= q_blocks;
        const int N = keys ? A.Nk : A.Nq, planes = keys ? A.Hk * key_parts : Hq * row_parts;
        const float* part = keys ? A.k_pos_part : A.q_pos_part;
        float* g = keys ? gk : gq;
        const int64_t token = (int64_t)b * SUM_THREADS + threadIdx.x;
        if (token >= N) return;
        if (!covered(keys ? A.k_offsets : A.q_offsets, keys ? A.k_lengths : A.q_lengths, A.S, N, (int)token)) return;
        float sum[3] = {0, 0, 0};
        for (int h = 0; h < planes; ++h)
            for (int c = 0; c < 3; ++c) sum[c] += part[((int64_t)h * N + token) * 3 + c];
        for (int c = 0; c < 3; ++c) g[token * 3 + c] = sum[c];
        return;
    }
    const int h = b - q_blocks - k_blocks;
    __shared__ double s[SUM_THREADS];
    double sum = 0;
    for (int64_t i = threadIdx.x; i < slope_lines; i += SUM_THREADS) sum += (double)A.slope_part[i * Hq + h];
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int o = SUM_THREADS / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) gslope[h] = (float)s[0];
}

// Sums of the parts' rows, for the covered tokens: a thread for four features.
template <typename T>
__global__ __launch_bounds__(SUM_THREADS) void k_dense_bwd_join(Rows out, const float* part, int parts, const int32_t* offsets,
                                                                const int32_t* lengths, int S, int N, int H, int D) {
    const int quads = D / 4;
    const int64_t i = (int64_t)blockIdx.x * SUM_THREADS + threadIdx.x, row = i / quads;
    if (row >= (int64_t)N * H) return;
    const int d = (int)(i % quads) * 4, token = (int)(row / H);
    if (!covered(offsets, lengths, S, N, token)) return;
    f32x4 sum = {0, 0, 0, 0};
    for (int p = 0; p < parts; ++p) sum += *reinterpret_cast<const f32x4*>(part + ((int64_t)p * N * H + row) * D + d);
    char* to = out.row(token, row % H) + d * sizeof(T);
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(to) = sum;
    else *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
}

// Workgroups of 128 rows (keys), or of 32 where a segment has no more than 64 of them on average; and parts of the other side
// where the workgroups do not fill the chip evenly: two of four waves to a compute unit, or one of eight.
struct BwdPlan {
    int row_waves, key_waves, stat_parts, row_parts, key_parts;
    int64_t row_tiles, key_tiles;
};
BwdPlan bwd_plan(const e2f_dense_args* a) {
    const int group = a->Hq / a->Hk;
    const int64_t S = a->S, rows = (int64_t)a->Nq * group;
    BwdPlan P = {1, 1, 1, 1, 1, 0, 0};
    if (S == 0) return P;
    P.row_waves = rows > 64 * S ? 4 : 1;
    P.key_waves = a->Nk > 64 * S ? 4 : 1;
    P.row_tiles = a->Nq ? dense_tiles(a->Nq, group, a->S, 32 * P.row_waves) : 0;
    P.key_tiles = a->Nk ? dense_tiles(a->Nk, 1, a->S, 32 * P.key_waves) : 0;
    // times of a round for a step along the other side, and of a part's sums, written and read at 4.5 TB/s.  At 5 003 keys of 2 heads and
    // 128 bf16 features, 314 workgroups over rows take 589 us in one part, 466 in three and 456 in four; 80 over keys, 20 012 rows, take
    // 1 605 us in one part, 646 in three, 638 in four and 649 in thirteen
    const double step = a->dtype == E2F_BF16 ? 0.03 + 0.0004 * a->D : 0.05 + 0.004 * a->D;
    const int row_slots = a->D > 64 ? 256 : 512, key_slots = a->D * elem_bytes(a->dtype) > 128 ? 256 : 512;
    if (P.row_tiles) {
        const int64_t blocks = P.row_tiles * a->Hk * P.row_waves / 4 + 1, most = a->Nk / S / 256;
        P.stat_parts = best_parts(blocks, 512, a->Nk / S * step, rows * a->Hk * 32.0 / 4.5e6, rows * a->Hk, most);
        P.row_parts = best_parts(blocks, row_slots, a->Nk / S * step, rows * a->Hk * a->D * 8.0 / 4.5e6, rows * a->Hk * (a->D / 4), most);
    }
    if (P.key_tiles)
        P.key_parts = best_parts(P.key_tiles * a->Hk * P.key_waves / 4 + 1, key_slots, rows / S * step, (double)a->Nk * a->Hk * a->D * 16.0 / 4.5e6,
                                 (int64_t)a->Nk * a->Hk * (a->D / 4), rows / S / 256);
    return P;
}

// Workgroups have up to two waves to a group of rows or keys, see launch_dp.
bool launches(const e2f_dense_args* a, const BwdPlan& P) {
    return e2f::launches(P.row_tiles * a->Hk, P.row_waves == 4 ? 512 : 64) && e2f::launches(P.key_tiles * a->Hk, P.key_waves == 4 ? 512 : 64);
}

template <typename T, int DP>
void launch_dp(const DenseParams& A, const BwdPlan& P, hipStream_t st) {
    const dim3 stats((unsigned)(P.row_tiles * A.Hk), (unsigned)P.stat_parts), rows(stats.x, (unsigned)P.row_parts),
        keys((unsigned)(P.key_tiles * A.Hk), (unsigned)P.key_parts);
    const int64_t n = (int64_t)A.Nq * A.Hk * A.group;
    // workgroups of many rows or keys with more than 64 features: two waves to a group of 32; of keys also beyond 32 features in fp32 (48
    // features, 4 x 1 000 atoms: rows 215 us with two waves and 147 with one, keys 197 and 245).  Workgroups of one wave have the
    // registers for all of it, and its LDS would leave a compute unit one workgroup
    constexpr int KD = DP > 64 ? 128 : DP, SHARE = DP > 64 ? 2 : 1, KEY_SHARE = DP * sizeof(T) > 128 ? 2 : 1;
    if (rows.x) {
        if (P.row_waves == 4) k_dense_bwd_stats<T, DP, 4><<<stats, 256, 0, st>>>(A);
        else k_dense_bwd_stats<T, DP, 1><<<stats, 64, 0, st>>>(A);
        if (P.stat_parts > 1) k_dense_bwd_join_stats<<<(unsigned)((n + SUM_THREADS - 1) / SUM_THREADS), SUM_THREADS, 0, st>>>(A, P.stat_parts);
        if (P.row_waves == 4) k_dense_bwd_rows<T, KD, 4, SHARE><<<rows, 256 * SHARE, 0, st>>>(A);
        else k_dense_bwd_rows<T, DP, 1, 1><<<rows, 64, 0, st>>>(A);
    }
    if (keys.x) {
        auto go = [&](auto cap, auto bias) {
            constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
            if (P.key_waves == 4) k_dense_bwd_keys<T, KD, 4, KEY_SHARE, CAP, BIAS><<<keys, 256 * KEY_SHARE, 0, st>>>(A);
            else k_dense_bwd_keys<T, DP, 1, 1, CAP, BIAS><<<keys, 64, 0, st>>>(A);
        };
        const std::true_type yes;
        const std::false_type no;
        if (A.score.capped) A.score.biased ? go(yes, yes) : go(yes, no);
        else A.score.biased ? go(no, yes) : go(no, no);
    }
    auto join = [&](const Rows& out, const float* part, int parts, const int32_t* offsets, const int32_t* lengths, int N, int H) {
        const int64_t threads = (int64_t)N * H * (A.D / 4);
        k_dense_bwd_join<T><<<(unsigned)((threads + SUM_THREADS - 1) / SUM_THREADS), SUM_THREADS, 0, st>>>(out, part, parts, offsets, lengths, A.S, N, H, A.D);
    };
    if (rows.x && P.row_parts > 1) join(A.out, A.gq_part, P.row_parts, A.q_offsets, A.q_lengths, A.Nq, A.Hk * A.group);
    if (keys.x && P.key_parts > 1) {
        join(A.gk, A.gk_part, P.key_parts, A.k_offsets, A.k_lengths, A.Nk, A.Hk);
        join(A.gv, A.gv_part, P.key_parts, A.k_offsets, A.k_lengths, A.Nk, A.Hk);
    }
}

template <typename T>
void launch(const DenseParams& A, const BwdPlan& P, hipStream_t st) {
    if (A.D <= 32) launch_dp<T, 32>(A, P, st);
    else if (A.D <= 64) launch_dp<T, 64>(A, P, st);
    else if (A.D <= 96) launch_dp<T, 96>(A, P, st);
    else launch_dp<T, 128>(A, P, st);
}

// Workspace: statistics of the rows, what the three sums need (always, so that the size does not depend on which are asked for),
// and the parts' rows.
size_t layout(const e2f_dense_args* a, const BwdPlan& P, char* ws, DenseParams* A) {
    size_t off = 0;
    auto take = [&](size_t floats) {
        char* p = ws ? ws + off : nullptr;
        off += e2f_align_up(floats * sizeof(float));
        return reinterpret_cast<float*>(p);
    };
    const size_t rows = (size_t)a->Nq * a->Hq, keys = (size_t)a->Nk * a->Hk, sp = P.stat_parts, rp = P.row_parts, kp = P.key_parts;
    float* stats = take(rows * 4);
    float* usual = take(a->slope ? rows : 0);
    float* slope = take(a->slope ? rp * P.row_tiles * a->Hq : 0);
    float* qp = take(a->slope ? rp * rows * 3 : 0);
    float* kpos = take(a->slope ? kp * keys * 3 : 0);
    float* stats_part = take(sp > 1 ? sp * rows * 4 : 0);
    float* gq = take(rp > 1 ? rp * rows * a->D : 0);
    float* gk = take(kp > 1 ? kp * keys * a->D : 0);
    float* gv = take(kp > 1 ? kp * keys * a->D : 0);
    if (A) {
        A->stats = reinterpret_cast<float4*>(stats);
        A->usual = usual;
        A->slope_part = slope;
        A->q_pos_part = qp;
        A->k_pos_part = kpos;
        A->stats_part = reinterpret_cast<float4*>(stats_part);
        A->gq_part = gq;
        A->gk_part = gk;
        A->gv_part = gv;
    }
    return off;
}

}  // namespace

extern "C" {

size_t e2f_dense_attn_backward_workspace_bytes(const e2f_dense_args* a) {
    if (dense_check_sizes(a) != E2F_OK) return 0;
    const BwdPlan P = bwd_plan(a);
    return launches(a, P) ? layout(a, P, nullptr, nullptr) : 0;
}

e2f_status e2f_dense_attn_backward(const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v,
                                   const e2f_heads* grad_out, const e2f_heads* grad_q, const e2f_heads* grad_k,
                                   const e2f_heads* grad_v, float* grad_slope, float* grad_q_pos, float* grad_k_pos,
                                   void* ws, size_t ws_bytes, void* hip_stream) {
    e2f_status rc = dense_check(a);
    if (rc != E2F_OK) return rc;
    if ((rc = check_rows(q, a->dtype, a->Nq, a->Hq)) != E2F_OK || (rc = check_rows(k, a->dtype, a->Nk, a->Hk)) != E2F_OK ||
        (rc = check_rows(v, a->dtype, a->Nk, a->Hk)) != E2F_OK || (rc = check_rows(grad_out, a->dtype, a->Nq, a->Hq)) != E2F_OK ||
        (rc = check_result_rows(grad_q, a->dtype, a->Nq, a->Hq, a->D)) != E2F_OK ||
        (rc = check_result_rows(grad_k, a->dtype, a->Nk, a->Hk, a->D)) != E2F_OK ||
        (rc = check_result_rows(grad_v, a->dtype, a->Nk, a->Hk, a->D)) != E2F_OK)
        return rc;
    if ((grad_slope || grad_q_pos || grad_k_pos) && !a->slope) return E2F_ERR_INVALID_ARG;
    if (!word_aligned(grad_slope) || !word_aligned(grad_q_pos) || !word_aligned(grad_k_pos)) return E2F_ERR_INVALID_ARG;
    const BwdPlan P = bwd_plan(a);
    if (!launches(a, P)) return E2F_ERR_UNSUPPORTED;
    const size_t need = layout(a, P, nullptr, nullptr);
    if (need && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < need) return E2F_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    DenseParams A;
    dense_fill(A, a, q, k, v);
    layout(a, P, static_cast<char*>(ws), &A);
    A.out = rows_of(grad_q, a->dtype);
    A.go = rows_of(grad_out, a->dtype);
    A.gk = rows_of(grad_k, a->dtype);
    A.gv = rows_of(grad_v, a->dtype);
    if (!grad_slope) A.slope_part = nullptr;
    if (!grad_q_pos) A.q_pos_part = nullptr;
    if (!grad_k_pos) A.k_pos_part = nullptr;
    if (P.row_tiles || P.key_tiles) {
        if (a->dtype == E2F_BF16) launch<uint16_t>(A, P, st);
        else launch<float>(A, P, st);
        E2F_HIP_CHECK(hipGetLastError());
    }
    const int q_blocks = grad_q_pos && P.row_tiles ? (a->Nq + SUM_THREADS - 1) / SUM_THREADS : 0;
    const int k_blocks = grad_k_pos && P.key_tiles ? (a->Nk + SUM_THREADS - 1) / SUM_THREADS : 0;
    const int blocks = q_blocks + k_blocks + (grad_slope ? a->Hq : 0);
    if (blocks) {
        k_dense_bwd_sums<<<blocks, SUM_THREADS, 0, st>>>(A, grad_q_pos, grad_k_pos, grad_slope, q_blocks, k_blocks, P.row_parts, P.key_parts, P.row_tiles * P.row_parts);
        E2F_HIP_CHECK(hipGetLastError());
    }
    return E2F_OK;
}

}  // extern "C"
