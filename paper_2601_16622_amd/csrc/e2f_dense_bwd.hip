// Attention among all atoms of a segment, backward.  With p the softmax weights, dp_ij = dout_i . v_j, th = tanh(x / cap):
//   delta_i = sum_j p dp;  ds = p (dp - delta);  dx = ds (1 - th^2)
//   dv_j = sum_i p dout_i;  dq_i = scale sum_j dx k_j;  dk_j = scale sum_i dx q_i
//   dslope_h = - sum ds d;  dr_i = - sum_{h,j} slope_h ds (r_i - r_j) / d,  dr_j the opposite
// Nothing of a pair is stored: a kernel over rows forms the softmax statistics and delta in a first pass over the keys and
// dq in a second one, a kernel over keys forms dk and dv, and each sum is formed by the workgroup that owns its row or key, so no
// atomics are needed.  delta comes from the binary32 products and weights (not from the rounded result of the forward pass):
// the gradients of slope and places are binary32 and keep their precision.
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

template <typename T, int DP, int ROWW>
__global__ __launch_bounds__(64 * ROWW) void k_dense_bwd_rows(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = ROWW > 1 && sizeof(T) == 2 ? 64 : 32, BM = 32 * ROWW, THREADS = 64 * ROWW;
    __shared__ __align__(16) T ks[BN * M::LD];
    __shared__ __align__(16) T vs[BN * M::LD];
    __shared__ __align__(16) float place[3 * BN];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = tid >> 6;
    const int head_k = blockIdx.x % A.Hk;
    const int64_t tile = blockIdx.x / A.Hk;
    const int s = segment_of(A.q_offsets, A.S, A.Nq, A.group, BM, tile);
    int q0, nq, k0, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, q0, nq);
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k0, nk);
    const int64_t row0 = (tile - first_tile(A.q_offsets, s, A.Nq, A.group, BM)) * BM, rows = (int64_t)nq * A.group;
    if (row0 < 0 || row0 >= rows) return;
    const int64_t row = row0 + wave * 32 + (lane & 31);
    const bool valid = row < rows, busy = row0 + wave * 32 < rows;
    const int in_segment = valid ? A.over_group((uint32_t)row) : 0;
    const int query = q0 + in_segment, head = head_k * A.group + (valid ? (int)row - in_segment * A.group : 0);
    typename M::Frag qf, gf;
    M::load(qf, A.q.row(query, head), A.D, valid, half);
    M::load(gf, A.go.row(query, head), A.D, valid, half);
    float x = 0, y = 0, z = 0, slope = 0;
    if (A.score.biased) {
        x = A.q_pos[(int64_t)query * 3];
        y = A.q_pos[(int64_t)query * 3 + 1];
        z = A.q_pos[(int64_t)query * 3 + 2];
        slope = A.slope[head];
    }
    const float slope2 = slope * LOG2E;
    Transfer<M, DP, BN, THREADS> tk, tv;
    PlaceTransfer<BN, THREADS> tp;
    auto fetch = [&](int t) {
        const int n = nk - t;
        tk.load(tid, n, A.D, [&](int r) { return A.k.row(k0 + t + r, head_k); });
        tv.load(tid, n, A.D, [&](int r) { return A.v.row(k0 + t + r, head_k); });
        if (A.score.biased) tp.load(tid, min(n, BN), A.k_pos + (int64_t)(k0 + t) * 3);
    };
    // walks over the keys: body(first row of 32 in the tile, how many count)
    auto walk = [&](auto body) {
        if (nk > 0) fetch(0);
        for (int t = 0; t < nk; t += BN) {
            tile_sync<(ROWW > 1)>();
            tk.store(tid, ks);
            tv.store(tid, vs);
            if (A.score.biased) tp.store(tid, place);
            tile_sync<(ROWW > 1)>();
            if (t + BN < nk) fetch(t + BN);
            if (!busy) continue;
            const int n = min(BN, nk - t);
            for (int m = 0; m < n; m += 32) body(m, n - m);
        }
    };
    auto behind = [&](f32x16& p, int n) {
        if (n >= 32) return;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i / 4) + 4 * half + i % 4 >= n) p[i] = -INFINITY;
    };
    float top = -INFINITY, sum = 0, delta = 0;
    walk([&](int m, int n) {
        f32x16 p = M::dot(ks, m, qf, lane);
        const f32x16 dp = M::dot(vs, m, gf, lane);
        cap_scores<false>(p, p, A.score, reference_base(top));
        if (A.score.biased) bias_scores<BN>(p, x, y, z, slope2, place, m + 4 * half);
        behind(p, n);
        float shrink;
        if (move_reference(p, top, shrink)) {
            sum *= shrink;
            delta *= shrink;
        }
        float add = 0, dot = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float w = __builtin_amdgcn_exp2f(p[i]);
            add += w;
            dot += w * dp[i];
        }
        sum += add;
        delta += dot;
    });
    sum += other_half(sum);
    delta += other_half(delta);
    const float inv = nk > 0 ? 1.0f / sum : 0.0f;
    delta *= inv;
    // weights stay without 1 / sum here: a row's sums get it at the end
    float dslope = 0, gx = 0, gy = 0, gz = 0;
    f32x16 acc[DP / 32] = {};
    walk([&](int m, int n) {
        f32x16 p = M::dot(ks, m, qf, lane), slack;
        const f32x16 dp = M::dot(vs, m, gf, lane);
        cap_scores<true>(p, slack, A.score, top);
        behind(p, n);
        if (A.score.biased) {
            float ts = 0, tx = 0, ty = 0, tz = 0;      // a tile's sums by themselves: shorter sums, smaller errors
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float* at = place + m + 4 * half + 8 * b;
                const f32x4 px = *reinterpret_cast<const f32x4*>(at), py = *reinterpret_cast<const f32x4*>(at + BN),
                            pz = *reinterpret_cast<const f32x4*>(at + 2 * BN);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * b + e;
                    const float dx = x - px[e], dy = y - py[e], dz = z - pz[e];
                    float d, id;
                    distance(dx, dy, dz, d, id);
                    p[i] = __builtin_amdgcn_exp2f(p[i] - slope2 * d) * (dp[i] - delta);
                    ts += p[i] * d;
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
        M::accumulate(acc, ks, m, M::weights(p), lane);
    });
    dslope += other_half(dslope);
    gx += other_half(gx);
    gy += other_half(gy);
    gz += other_half(gz);
    if (!valid) return;
    store_row<T, DP>(A.out.row(query, head), acc, A.scale * inv, A.D, half);
    if (half) return;
    const int64_t at = (int64_t)query * (A.Hk * A.group) + head;
    A.stats[at] = make_float4(top, inv, delta, 0.0f);
    if (A.slope_part) A.slope_part[at] = -dslope * inv;
    if (A.q_pos_part) {
        float* g = A.q_pos_part + ((int64_t)head * A.Nq + query) * 3;
        g[0] = -slope * inv * gx;
        g[1] = -slope * inv * gy;
        g[2] = -slope * inv * gz;
    }
}

// What the kernel over keys needs of a row, as lines of BN in LDS.
enum { ROW_X, ROW_Y, ROW_Z, ROW_SLOPE, ROW_TOP, ROW_INV, ROW_DELTA, ROW_LINES };

template <typename T, int DP, int ROWW>
__global__ __launch_bounds__(64 * ROWW) void k_dense_bwd_keys(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = ROWW > 1 && sizeof(T) == 2 ? 64 : 32, BM = 32 * ROWW, THREADS = 64 * ROWW;
    __shared__ __align__(16) T qs[BN * M::LD];
    __shared__ __align__(16) T gs[BN * M::LD];
    __shared__ __align__(16) float par[ROW_LINES][BN];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = tid >> 6;
    const int head_k = blockIdx.x % A.Hk, Hq = A.Hk * A.group;
    const int64_t tile = blockIdx.x / A.Hk;
    const int s = segment_of(A.k_offsets, A.S, A.Nk, 1, BM, tile);
    int q0, nq, k0, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, q0, nq);
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k0, nk);
    const int64_t first = (tile - first_tile(A.k_offsets, s, A.Nk, 1, BM)) * BM;
    const int rows = nq * A.group;
    if (first < 0 || first >= nk) return;
    const int mine = (int)first + wave * 32 + (lane & 31);
    const bool valid = mine < nk, busy = (int)first + wave * 32 < nk;
    const int key = k0 + (valid ? mine : 0);
    typename M::Frag kf, vf;
    M::load(kf, A.k.row(key, head_k), A.D, valid, half);
    M::load(vf, A.v.row(key, head_k), A.D, valid, half);
    float x = 0, y = 0, z = 0;
    if (A.score.biased) {
        x = A.k_pos[(int64_t)key * 3];
        y = A.k_pos[(int64_t)key * 3 + 1];
        z = A.k_pos[(int64_t)key * 3 + 2];
    }
    Transfer<M, DP, BN, THREADS> tq, tg;
    float4 st;
    float rx = 0, ry = 0, rz = 0, rs = 0;
    auto fetch = [&](int t) {
        const int n = rows - t;
        auto at = [&](const Rows& R, int r) {
            const int query = A.over_group((uint32_t)(t + r));
            return R.row(q0 + query, head_k * A.group + (t + r - query * A.group));
        };
        tq.load(tid, n, A.D, [&](int r) { return at(A.q, r); });
        tg.load(tid, n, A.D, [&](int r) { return at(A.go, r); });
        st = make_float4(INFINITY, 0, 0, 0);        // rows behind the end: weight 0
        if (tid < n && tid < BN) {
            const int in_segment = A.over_group((uint32_t)(t + tid)), head = head_k * A.group + (t + tid - in_segment * A.group);
            const int64_t query = q0 + in_segment;
            st = A.stats[query * Hq + head];
            if (A.score.biased) {
                rx = A.q_pos[query * 3];
                ry = A.q_pos[query * 3 + 1];
                rz = A.q_pos[query * 3 + 2];
                rs = A.slope[head];
            }
        }
    };
    float gx = 0, gy = 0, gz = 0;
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    if (rows > 0) fetch(0);
    for (int t = 0; t < rows; t += BN) {
        tile_sync<(ROWW > 1)>();
        tq.store(tid, qs);
        tg.store(tid, gs);
        if (tid < BN) {
            par[ROW_X][tid] = rx;
            par[ROW_Y][tid] = ry;
            par[ROW_Z][tid] = rz;
            par[ROW_SLOPE][tid] = rs;
            par[ROW_TOP][tid] = st.x;
            par[ROW_INV][tid] = st.y;
            par[ROW_DELTA][tid] = st.z;
        }
        tile_sync<(ROWW > 1)>();
        if (t + BN < rows) fetch(t + BN);
        if (!busy) continue;
        const int n = min(BN, rows - t);
        for (int m = 0; m < n; m += 32) {
            f32x16 p = M::dot(qs, m, kf, lane), ds = M::dot(gs, m, vf, lane), slack;
            cap_scores<true>(p, slack, A.score, 0.0f);
            float tx = 0, ty = 0, tz = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                auto line = [&](int l) { return *reinterpret_cast<const f32x4*>(&par[l][m + 4 * half + 8 * b]); };
                const f32x4 top = line(ROW_TOP), inv = line(ROW_INV), delta = line(ROW_DELTA);
                if (A.score.biased) {
                    const f32x4 px = line(ROW_X), py = line(ROW_Y), pz = line(ROW_Z), slope = line(ROW_SLOPE);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * b + e;
                        const float dx = px[e] - x, dy = py[e] - y, dz = pz[e] - z;
                        float d, id;
                        distance(dx, dy, dz, d, id);
                        p[i] = __builtin_amdgcn_exp2f((p[i] - top[e]) - slope[e] * LOG2E * d) * inv[e];
                        const float g = p[i] * (ds[i] - delta[e]), f = g * slope[e] * id;
                        tx += f * dx;
                        ty += f * dy;
                        tz += f * dz;
                        ds[i] = g;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * b + e;
                        p[i] = __builtin_amdgcn_exp2f(p[i] - top[e]) * inv[e];
                        ds[i] = p[i] * (ds[i] - delta[e]);
                    }
                }
            }
            gx += tx;
            gy += ty;
            gz += tz;
            if (A.score.capped) {
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[i] *= slack[i];
            }
            M::accumulate(dv, gs, m, M::weights(p), lane);
            M::accumulate(dk, qs, m, M::weights(ds), lane);
        }
    }
    gx += other_half(gx);
    gy += other_half(gy);
    gz += other_half(gz);
    if (!valid) return;
    store_row<T, DP>(A.gk.row(key, head_k), dk, A.scale, A.D, half);
    store_row<T, DP>(A.gv.row(key, head_k), dv, 1.0f, A.D, half);
    if (A.k_pos_part && !half) {
        float* g = A.k_pos_part + ((int64_t)head_k * A.Nk + key) * 3;
        g[0] = gx;
        g[1] = gy;
        g[2] = gz;
    }
}

// Sums of the partial place gradients over the heads, for the tokens that a segment's length covers, and of the slopes'
// over the rows.  Workgroups: first those of the queries, then of the keys (a thread for a token), then one for each slope.
__global__ __launch_bounds__(SUM_THREADS) void k_dense_bwd_sums(DenseParams A, float* gq, float* gk, float* gslope, int q_blocks, int k_blocks) {
    const int Hq = A.Hk * A.group;
    int b = blockIdx.x;
    if (b < q_blocks + k_blocks) {
        const bool keys = b >= q_blocks;
        if (keys) b -= q_blocks;
        const int N = keys ? A.Nk : A.Nq, H = keys ? A.Hk : Hq;
        const int32_t* offsets = keys ? A.k_offsets : A.q_offsets;
        const float* part = keys ? A.k_pos_part : A.q_pos_part;
        float* g = keys ? gk : gq;
        const int64_t token = (int64_t)b * SUM_THREADS + threadIdx.x;
        if (token >= N) return;
        int first, n;
        segment_range(offsets, keys ? A.k_lengths : A.q_lengths, token_segment(offsets, A.S, (int)token), N, first, n);
        if (token < first || token >= first + n) return;
        float sum[3] = {0, 0, 0};
        for (int h = 0; h < H; ++h)
            for (int c = 0; c < 3; ++c) sum[c] += part[((int64_t)h * N + token) * 3 + c];
        for (int c = 0; c < 3; ++c) g[token * 3 + c] = sum[c];
        return;
    }
    const int h = b - q_blocks - k_blocks;
    __shared__ double s[SUM_THREADS];
    double sum = 0;
    for (int seg = 0; seg < A.S; ++seg) {
        int first, n;
        segment_range(A.q_offsets, A.q_lengths, seg, A.Nq, first, n);
        for (int i = threadIdx.x; i < n; i += SUM_THREADS) sum += (double)A.slope_part[(int64_t)(first + i) * Hq + h];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int o = SUM_THREADS / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) gslope[h] = (float)s[0];
}

// Workgroups of four waves and 128 rows (keys), or of one wave where a segment has no more than 64 of them on average.
struct BwdPlan {
    int row_waves, key_waves;
    int64_t row_tiles, key_tiles;
};
BwdPlan bwd_plan(const e2f_dense_args* a) {
    const int group = a->Hq / a->Hk;
    const int64_t S = a->S;
    BwdPlan P;
    P.row_waves = (int64_t)a->Nq * group > 64 * S ? 4 : 1;
    P.key_waves = a->Nk > 64 * S ? 4 : 1;
    P.row_tiles = a->Nq && S ? dense_tiles(a->Nq, group, a->S, 32 * P.row_waves) : 0;
    P.key_tiles = a->Nk && S ? dense_tiles(a->Nk, 1, a->S, 32 * P.key_waves) : 0;
    return P;
}

template <typename T, int DP>
void launch_dp(const DenseParams& A, const BwdPlan& P, hipStream_t st) {
    const unsigned rows = (unsigned)(P.row_tiles * A.Hk), keys = (unsigned)(P.key_tiles * A.Hk);
    if (rows && P.row_waves == 4) k_dense_bwd_rows<T, DP, 4><<<rows, 256, 0, st>>>(A);
    else if (rows) k_dense_bwd_rows<T, DP, 1><<<rows, 64, 0, st>>>(A);
    if (keys && P.key_waves == 4) k_dense_bwd_keys<T, DP, 4><<<keys, 256, 0, st>>>(A);
    else if (keys) k_dense_bwd_keys<T, DP, 1><<<keys, 64, 0, st>>>(A);
}

template <typename T>
void launch(const DenseParams& A, const BwdPlan& P, hipStream_t st) {
    if (A.D <= 32) launch_dp<T, 32>(A, P, st);
    else if (A.D <= 64) launch_dp<T, 64>(A, P, st);
    else if (A.D <= 96) launch_dp<T, 96>(A, P, st);
    else launch_dp<T, 128>(A, P, st);
}

// Workspace: statistics of the rows, then what the three sums need (always, so that the size does not depend on what is asked for).
size_t layout(const e2f_dense_args* a, char* ws, DenseParams* A) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* p = ws ? ws + off : nullptr;
        off += e2f_align_up(bytes);
        return p;
    };
    const size_t rows = (size_t)a->Nq * a->Hq;
    char* stats = take(rows * sizeof(float4));
    char* slope = a->slope ? take(rows * sizeof(float)) : nullptr;
    char* qp = a->slope ? take(rows * 3 * sizeof(float)) : nullptr;
    char* kp = a->slope ? take((size_t)a->Nk * a->Hk * 3 * sizeof(float)) : nullptr;
    if (A) {
        A->stats = reinterpret_cast<float4*>(stats);
        A->slope_part = reinterpret_cast<float*>(slope);
        A->q_pos_part = reinterpret_cast<float*>(qp);
        A->k_pos_part = reinterpret_cast<float*>(kp);
    }
    return off;
}

}  // namespace

extern "C" {

size_t e2f_dense_attn_backward_workspace_bytes(const e2f_dense_args* a) {
    return dense_check_sizes(a) == E2F_OK ? layout(a, nullptr, nullptr) : 0;
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
    const size_t need = layout(a, nullptr, nullptr);
    if (need && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < need) return E2F_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    DenseParams A;
    dense_fill(A, a, q, k, v);
    layout(a, static_cast<char*>(ws), &A);
    A.out = rows_of(grad_q, a->dtype);
    A.go = rows_of(grad_out, a->dtype);
    A.gk = rows_of(grad_k, a->dtype);
    A.gv = rows_of(grad_v, a->dtype);
    if (!grad_slope) A.slope_part = nullptr;
    if (!grad_q_pos) A.q_pos_part = nullptr;
    if (!grad_k_pos) A.k_pos_part = nullptr;
    const BwdPlan P = bwd_plan(a);
    if (P.row_tiles || P.key_tiles) {
        if (a->dtype == E2F_BF16) launch<uint16_t>(A, P, st);
        else launch<float>(A, P, st);
        E2F_HIP_CHECK(hipGetLastError());
    }
    const int q_blocks = grad_q_pos && P.row_tiles ? (a->Nq + SUM_THREADS - 1) / SUM_THREADS : 0;
    const int k_blocks = grad_k_pos && P.key_tiles ? (a->Nk + SUM_THREADS - 1) / SUM_THREADS : 0;
    const int blocks = q_blocks + k_blocks + (grad_slope ? a->Hq : 0);
    if (blocks) {
        k_dense_bwd_sums<<<blocks, SUM_THREADS, 0, st>>>(A, grad_q_pos, grad_k_pos, grad_slope, q_blocks, k_blocks);
        E2F_HIP_CHECK(hipGetLastError());
    }
    return E2F_OK;
}

}  // extern "C"
