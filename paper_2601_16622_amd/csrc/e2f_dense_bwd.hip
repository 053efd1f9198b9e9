// Attention among all atoms of a segment, backward.  With p the softmax weights, dp_ij = dout_i . v_j, th = tanh(x / cap):
//   delta_i = sum_j p dp;  ds = p (dp - delta);  dx = ds (1 - th^2)
//   dv_j = sum_i p dout_i;  dq_i = scale sum_j dx k_j;  dk_j = scale sum_i dx q_i
//   dslope_h = - sum ds d;  dr_i = - sum_{h,j} slope_h ds (r_i - r_j) / d,  dr_j the opposite
// Nothing of a pair is stored: a kernel over rows forms the softmax statistics and delta in a first pass over the keys and
// dq in a second one, a kernel over keys forms dk and dv, and each sum is formed by the workgroup that owns its row or key, so no
// atomics are needed.  delta comes from the binary32 products and weights (not from the rounded result of the forward pass):
// the gradients of slope and places are binary32 and keep their precision.
#include "e2f_dense_api.h"
#include "e2f_dense.h"

namespace {

using namespace e2f;


template <typename T, int DP>
__global__ __launch_bounds__(DENSE_THREADS) void k_dense_bwd_rows(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = M::BN;
    __shared__ __align__(16) T ks[M::TILE];
    __shared__ __align__(16) T vs[M::TILE];
    __shared__ __align__(16) T kt[M::TURNED > 0 ? M::TURNED : 8];
    __shared__ __align__(16) float place[3 * BN];
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int head_k = blockIdx.x % A.Hk;
    const int64_t tile = blockIdx.x / A.Hk;
    const int s = segment_of(A.q_offsets, A.S, A.Nq, A.group, DENSE_BM, tile);
    int q0, nq, k0, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, q0, nq);
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k0, nk);
    const int64_t row0 = (tile - first_tile(A.q_offsets, s, A.Nq, A.group, DENSE_BM)) * DENSE_BM, rows = (int64_t)nq * A.group;
    if (row0 < 0 || row0 >= rows) return;
    const int64_t row = row0 + wave * 32 + (lane & 31);
    const bool valid = row < rows, busy = row0 + wave * 32 < rows;
    const int query = q0 + (valid ? (int)(row / A.group) : 0), head = head_k * A.group + (valid ? (int)(row % A.group) : 0);
    typename M::Frag qf, gf;
    M::load(qf, A.q.row(query, head), A.D, valid, half);
    M::load(gf, A.go.row(query, head), A.D, valid, half);
    float x = 0, y = 0, z = 0, slope = 0;
    if (A.slope) {
        x = A.q_pos[(int64_t)query * 3];
        y = A.q_pos[(int64_t)query * 3 + 1];
        z = A.q_pos[(int64_t)query * 3 + 2];
        slope = A.slope[head];
    }
    const float in = A.cap > 0 ? A.scale / A.cap : A.scale * LOG2E, out = A.cap * LOG2E;
    float top = -INFINITY, sum = 0, delta = 0, dslope = 0, gx = 0, gy = 0, gz = 0;
    f32x16 acc[DP / 32] = {};
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            sum += other_half(sum);
            delta += other_half(delta);
            sum = nk > 0 ? 1.0f / sum : 0.0f;
            delta *= sum;
        }
        for (int t = 0; t < nk; t += BN) {
            const int n = min(BN, nk - t);
            __syncthreads();
            if (pass == 0) stage<M, DP, true, false>(ks, nullptr, n, A.D, [&](int r) { return A.k.row(k0 + t + r, head_k); });
            else stage<M, DP, true, true>(ks, kt, n, A.D, [&](int r) { return A.k.row(k0 + t + r, head_k); });
            stage<M, DP, true, false>(vs, nullptr, n, A.D, [&](int r) { return A.v.row(k0 + t + r, head_k); });
            if (A.slope) stage_places<BN>(place, A.k_pos, k0 + t, n);
            __syncthreads();
            if (!busy) continue;
            for (int m = 0; m < n; m += 32) {
                f32x16 p = M::dot(ks, m, qf, lane);
                const f32x16 dp = M::dot(vs, m, gf, lane);
                float most = -INFINITY;
                f32x16 slack;      // 1 - tanh^2
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = m + 8 * (i / 4) + 4 * half + i % 4;
                    float v = p[i] * in;
                    slack[i] = 1.0f;
                    if (A.cap > 0) {
                        const float th = tanhf(v);
                        v = th * out;
                        slack[i] = 1.0f - th * th;
                    }
                    if (A.slope) {
                        const float dx = x - place[key], dy = y - place[BN + key], dz = z - place[2 * BN + key];
                        v -= slope * LOG2E * sqrtf(dx * dx + dy * dy + dz * dz);
                    }
                    p[i] = key < n ? v : -INFINITY;
                    most = fmaxf(most, p[i]);
                }
                if (pass == 0) {
                    most = fmaxf(most, other_half(most));
                    const float now = fmaxf(top, most), shrink = exp2f(top - now);
                    top = now;
                    sum *= shrink;
                    delta *= shrink;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float w = exp2f(p[i] - top);
                        sum += w;
                        delta += w * dp[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = m + 8 * (i / 4) + 4 * half + i % 4;
                        const float ds = exp2f(p[i] - top) * sum * (dp[i] - delta);
                        if (A.slope) {
                            const float dx = x - place[key], dy = y - place[BN + key], dz = z - place[2 * BN + key];
                            const float d = sqrtf(dx * dx + dy * dy + dz * dz);
                            dslope -= ds * d;
                            const float f = d > 0 ? ds / d : 0.0f;
                            gx -= f * dx;
                            gy -= f * dy;
                            gz -= f * dz;
                        }
                        p[i] = ds * slack[i];
                    }
                    M::accumulate(acc, ks, kt, m, M::weights(p), lane);
                }
            }
        }
    }
    dslope += other_half(dslope);
    gx += other_half(gx);
    gy += other_half(gy);
    gz += other_half(gz);
    if (!valid) return;
    store_row<T, DP>(A.out.row(query, head), acc, A.scale, A.D, half);
    if (half) return;
    const int64_t at = (int64_t)query * (A.Hk * A.group) + head;
    A.stats[at] = make_float4(top, sum, delta, 0.0f);
    if (A.slope_part) A.slope_part[at] = dslope;
    if (A.q_pos_part) {
        float* g = A.q_pos_part + ((int64_t)head * A.Nq + query) * 3;
        g[0] = slope * gx;
        g[1] = slope * gy;
        g[2] = slope * gz;
    }
}

template <typename T, int DP>
__global__ __launch_bounds__(DENSE_THREADS) void k_dense_bwd_keys(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = M::BN;
    __shared__ __align__(16) T qs[M::TILE];
    __shared__ __align__(16) T gs[M::TILE];
    __shared__ __align__(16) T qt[M::TURNED > 0 ? M::TURNED : 8];
    __shared__ __align__(16) T gt[M::TURNED > 0 ? M::TURNED : 8];
    __shared__ __align__(16) float par[7][BN];      // place, slope, softmax reference, 1 / sum, delta of the rows
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int head_k = blockIdx.x % A.Hk;
    const int64_t tile = blockIdx.x / A.Hk;
    const int s = segment_of(A.k_offsets, A.S, A.Nk, 1, DENSE_BM, tile);
    int q0, nq, k0, nk;
    segment_range(A.q_offsets, A.q_lengths, s, A.Nq, q0, nq);
    segment_range(A.k_offsets, A.k_lengths, s, A.Nk, k0, nk);
    const int64_t first = (tile - first_tile(A.k_offsets, s, A.Nk, 1, DENSE_BM)) * DENSE_BM, rows = (int64_t)nq * A.group;
    if (first < 0 || first >= nk) return;
    const int mine = (int)first + wave * 32 + (lane & 31);
    const bool valid = mine < nk, busy = (int)first + wave * 32 < nk;
    const int key = k0 + (valid ? mine : 0);
    typename M::Frag kf, vf;
    M::load(kf, A.k.row(key, head_k), A.D, valid, half);
    M::load(vf, A.v.row(key, head_k), A.D, valid, half);
    float x = 0, y = 0, z = 0;
    if (A.slope) {
        x = A.k_pos[(int64_t)key * 3];
        y = A.k_pos[(int64_t)key * 3 + 1];
        z = A.k_pos[(int64_t)key * 3 + 2];
    }
    const float in = A.cap > 0 ? A.scale / A.cap : A.scale * LOG2E, out = A.cap * LOG2E;
    float gx = 0, gy = 0, gz = 0;
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    for (int64_t t = 0; t < rows; t += BN) {
        const int n = (int)min((int64_t)BN, rows - t);
        auto at = [&](const Rows& R, int r) { return R.row(q0 + (t + r) / A.group, head_k * A.group + (t + r) % A.group); };
        __syncthreads();
        stage<M, DP, true, true>(qs, qt, n, A.D, [&](int r) { return at(A.q, r); });
        stage<M, DP, true, true>(gs, gt, n, A.D, [&](int r) { return at(A.go, r); });
        for (int r = threadIdx.x; r < BN; r += DENSE_THREADS) {
            float4 st = make_float4(0, 0, 0, 0);
            float px = 0, py = 0, pz = 0, sl = 0;
            if (r < n) {
                const int64_t query = q0 + (t + r) / A.group;
                const int head = head_k * A.group + (int)((t + r) % A.group);
                st = A.stats[query * (A.Hk * A.group) + head];
                if (A.slope) {
                    px = A.q_pos[query * 3];
                    py = A.q_pos[query * 3 + 1];
                    pz = A.q_pos[query * 3 + 2];
                    sl = A.slope[head];
                }
            }
            par[0][r] = px;
            par[1][r] = py;
            par[2][r] = pz;
            par[3][r] = sl;
            par[4][r] = r < n ? st.x : INFINITY;   // rows behind the end: weight 0
            par[5][r] = st.y;
            par[6][r] = st.z;
        }
        __syncthreads();
        if (!busy) continue;
        for (int m = 0; m < n; m += 32) {
            f32x16 p = M::dot(qs, m, kf, lane);
            f32x16 ds = M::dot(gs, m, vf, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = m + 8 * (i / 4) + 4 * half + i % 4;
                float v = p[i] * in, slack = 1.0f, d = 0, dx = 0, dy = 0, dz = 0;
                if (A.cap > 0) {
                    const float th = tanhf(v);
                    v = th * out;
                    slack = 1.0f - th * th;
                }
                if (A.slope) {
                    dx = par[0][r] - x;
                    dy = par[1][r] - y;
                    dz = par[2][r] - z;
                    d = sqrtf(dx * dx + dy * dy + dz * dz);
                    v -= par[3][r] * LOG2E * d;
                }
                p[i] = exp2f(v - par[4][r]) * par[5][r];
                const float g = p[i] * (ds[i] - par[6][r]);
                if (A.slope) {
                    const float f = d > 0 ? par[3][r] * g / d : 0.0f;
                    gx += f * dx;
                    gy += f * dy;
                    gz += f * dz;
                }
                ds[i] = g * slack;
            }
            M::accumulate(dv, gs, gt, m, M::weights(p), lane);
            M::accumulate(dk, qs, qt, m, M::weights(ds), lane);
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
__global__ __launch_bounds__(DENSE_THREADS) void k_dense_bwd_sums(DenseParams A, float* gq, float* gk, float* gslope, int q_blocks, int k_blocks) {
    const int Hq = A.Hk * A.group;
    int b = blockIdx.x;
    if (b < q_blocks + k_blocks) {
        const bool keys = b >= q_blocks;
        if (keys) b -= q_blocks;
        const int N = keys ? A.Nk : A.Nq, H = keys ? A.Hk : Hq;
        const int32_t* offsets = keys ? A.k_offsets : A.q_offsets;
        const float* part = keys ? A.k_pos_part : A.q_pos_part;
        float* g = keys ? gk : gq;
        const int64_t token = (int64_t)b * DENSE_THREADS + threadIdx.x;
        if (token >= N) return;
        int lo = 0, hi = A.S;      // the last segment that starts at or before the token
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (offsets[mid] <= token) lo = mid; else hi = mid;
        }
        int first, n;
        segment_range(offsets, keys ? A.k_lengths : A.q_lengths, lo, N, first, n);
        if (token < first || token >= first + n) return;
        float sum[3] = {0, 0, 0};
        for (int h = 0; h < H; ++h)
            for (int c = 0; c < 3; ++c) sum[c] += part[((int64_t)h * N + token) * 3 + c];
        for (int c = 0; c < 3; ++c) g[token * 3 + c] = sum[c];
        return;
    }
    const int h = b - q_blocks - k_blocks;
    __shared__ double s[DENSE_THREADS];
    double sum = 0;
    for (int seg = 0; seg < A.S; ++seg) {
        int first, n;
        segment_range(A.q_offsets, A.q_lengths, seg, A.Nq, first, n);
        for (int i = threadIdx.x; i < n; i += DENSE_THREADS) sum += (double)A.slope_part[(int64_t)(first + i) * Hq + h];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int o = DENSE_THREADS / 2; o; o >>= 1) {
        if ((int)threadIdx.x < o) s[threadIdx.x] += s[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) gslope[h] = (float)s[0];
}

template <typename T, int DP>
void launch_dp(const DenseParams& A, unsigned row_blocks, unsigned key_blocks, hipStream_t st) {
    if (row_blocks) k_dense_bwd_rows<T, DP><<<row_blocks, DENSE_THREADS, 0, st>>>(A);
    if (key_blocks) k_dense_bwd_keys<T, DP><<<key_blocks, DENSE_THREADS, 0, st>>>(A);
}

template <typename T>
void launch(const DenseParams& A, unsigned row_blocks, unsigned key_blocks, hipStream_t st) {
    if (A.D <= 32) launch_dp<T, 32>(A, row_blocks, key_blocks, st);
    else if (A.D <= 64) launch_dp<T, 64>(A, row_blocks, key_blocks, st);
    else if (A.D <= 96) launch_dp<T, 96>(A, row_blocks, key_blocks, st);
    else launch_dp<T, 128>(A, row_blocks, key_blocks, st);
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
    const unsigned row_blocks = a->Nq && a->S ? (unsigned)(dense_tiles(a->Nq, A.group, a->S, DENSE_BM) * a->Hk) : 0;
    const unsigned key_blocks = a->Nk && a->S ? (unsigned)(dense_tiles(a->Nk, 1, a->S, DENSE_BM) * a->Hk) : 0;
    if (row_blocks || key_blocks) {
        if (a->dtype == E2F_BF16) launch<uint16_t>(A, row_blocks, key_blocks, st);
        else launch<float>(A, row_blocks, key_blocks, st);
        E2F_HIP_CHECK(hipGetLastError());
    }
    const int q_blocks = grad_q_pos && row_blocks ? (a->Nq + DENSE_THREADS - 1) / DENSE_THREADS : 0;
    const int k_blocks = grad_k_pos && key_blocks ? (a->Nk + DENSE_THREADS - 1) / DENSE_THREADS : 0;
    const int blocks = q_blocks + k_blocks + (grad_slope ? a->Hq : 0);
    if (blocks) {
        k_dense_bwd_sums<<<blocks, DENSE_THREADS, 0, st>>>(A, grad_q_pos, grad_k_pos, grad_slope, q_blocks, k_blocks);
        E2F_HIP_CHECK(hipGetLastError());
    }
    return E2F_OK;
}

}  // extern "C"
