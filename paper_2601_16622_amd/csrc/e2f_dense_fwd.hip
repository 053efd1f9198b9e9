// Attention among all atoms of a segment, forward: one pass over the keys with the running maximum and sum of the softmax.
#include "e2f_dense_api.h"
#include "e2f_dense.h"

namespace {

using namespace e2f;

template <typename T, int DP>
__global__ __launch_bounds__(DENSE_THREADS) void k_dense_fwd(DenseParams A) {
    using M = Mma<T, DP>;
    constexpr int BN = M::BN;
    __shared__ __align__(16) T ks[M::TILE];
    __shared__ __align__(16) T vs[sizeof(T) == 4 ? M::TILE : M::TURNED];
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
    typename M::Frag qf;
    M::load(qf, A.q.row(query, head), A.D, valid, half);
    float x = 0, y = 0, z = 0, slope = 0;
    if (A.slope) {
        x = A.q_pos[(int64_t)query * 3];
        y = A.q_pos[(int64_t)query * 3 + 1];
        z = A.q_pos[(int64_t)query * 3 + 2];
        slope = A.slope[head] * LOG2E;
    }
    const float in = A.cap > 0 ? A.scale / A.cap : A.scale * LOG2E, out = A.cap * LOG2E;
    f32x16 acc[DP / 32] = {};
    float top = -INFINITY, sum = 0;
    for (int t = 0; t < nk; t += BN) {
        const int n = min(BN, nk - t);
        __syncthreads();
        stage<M, DP, true, false>(ks, nullptr, n, A.D, [&](int r) { return A.k.row(k0 + t + r, head_k); });
        if constexpr (sizeof(T) == 4) stage<M, DP, true, false>(vs, nullptr, n, A.D, [&](int r) { return A.v.row(k0 + t + r, head_k); });
        else stage<M, DP, false, true>(nullptr, vs, n, A.D, [&](int r) { return A.v.row(k0 + t + r, head_k); });
        if (A.slope) stage_places<BN>(place, A.k_pos, k0 + t, n);
        __syncthreads();
        if (!busy) continue;
        for (int m = 0; m < n; m += 32) {
            f32x16 p = M::dot(ks, m, qf, lane);
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = m + 8 * (i / 4) + 4 * half + i % 4;
                float v = p[i] * in;
                if (A.cap > 0) v = tanhf(v) * out;
                if (A.slope) {
                    const float dx = x - place[key], dy = y - place[BN + key], dz = z - place[2 * BN + key];
                    v -= slope * sqrtf(dx * dx + dy * dy + dz * dz);
                }
                p[i] = key < n ? v : -INFINITY;
                most = fmaxf(most, p[i]);
            }
            most = fmaxf(most, other_half(most));
            const float now = fmaxf(top, most), shrink = exp2f(top - now);
            top = now;
            sum *= shrink;
#pragma unroll
            for (int dt = 0; dt < DP / 32; ++dt) acc[dt] *= shrink;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = exp2f(p[i] - top);
                sum += p[i];
            }
            M::accumulate(acc, vs, vs, m, M::weights(p), lane);
        }
    }
    sum += other_half(sum);
    if (valid) store_row<T, DP>(A.out.row(query, head), acc, nk > 0 ? 1.0f / sum : 0.0f, A.D, half);
}

template <typename T>
void launch(const DenseParams& A, unsigned blocks, hipStream_t st) {
    if (A.D <= 32) k_dense_fwd<T, 32><<<blocks, DENSE_THREADS, 0, st>>>(A);
    else if (A.D <= 64) k_dense_fwd<T, 64><<<blocks, DENSE_THREADS, 0, st>>>(A);
    else if (A.D <= 96) k_dense_fwd<T, 96><<<blocks, DENSE_THREADS, 0, st>>>(A);
    else k_dense_fwd<T, 128><<<blocks, DENSE_THREADS, 0, st>>>(A);
}

}  // namespace

namespace e2f {

e2f_status dense_check_sizes(const e2f_dense_args* a) {
    if (!a || (a->dtype != E2F_F32 && a->dtype != E2F_BF16) || a->Nq < 0 || a->Nk < 0 || a->S < 0 || a->Hq <= 0 || a->Hk <= 0 ||
        a->D <= 0 || a->Hq % a->Hk || !isfinite(a->scale) || !(a->cap >= 0.0f) || !isfinite(a->cap))
        return E2F_ERR_INVALID_ARG;
    if (a->D % 8 || a->D > 128 || a->Hq > 1024) return E2F_ERR_UNSUPPORTED;
    // the grid of either direction is a 31-bit number
    const int64_t most = INT32_MAX / a->Hk;
    if (dense_tiles(a->Nq, a->Hq / a->Hk, a->S, DENSE_BM) > most || dense_tiles(a->Nk, 1, a->S, DENSE_BM) > most)
        return E2F_ERR_UNSUPPORTED;
    return E2F_OK;
}

e2f_status dense_check(const e2f_dense_args* a) {
    const e2f_status rc = dense_check_sizes(a);
    if (rc != E2F_OK) return rc;
    if (a->slope ? (a->Nq > 0 && !a->q_pos) || (a->Nk > 0 && !a->k_pos) : a->q_pos || a->k_pos) return E2F_ERR_INVALID_ARG;
    if (a->S > 0 && (!a->q_offsets || !a->k_offsets)) return E2F_ERR_INVALID_ARG;
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
    A.D = a->D;
    A.scale = a->scale;
    A.cap = a->cap;
}

}  // namespace e2f

extern "C" {

size_t e2f_dense_attn_workspace_bytes(const e2f_dense_args* a) {
    (void)a;
    return 0;
}

e2f_status e2f_dense_attn_forward(const e2f_dense_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* v,
                                  const e2f_heads* out, void* ws, size_t ws_bytes, void* hip_stream) {
    e2f_status rc = dense_check(a);
    if (rc != E2F_OK) return rc;
    if ((rc = check_rows(q, a->dtype, a->Nq, a->Hq)) != E2F_OK || (rc = check_rows(k, a->dtype, a->Nk, a->Hk)) != E2F_OK ||
        (rc = check_rows(v, a->dtype, a->Nk, a->Hk)) != E2F_OK ||
        (rc = check_result_rows(out, a->dtype, a->Nq, a->Hq, a->D)) != E2F_OK)
        return rc;
    const size_t need = e2f_dense_attn_workspace_bytes(a);
    if (need && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < need) return E2F_ERR_WORKSPACE_TOO_SMALL;
    if (a->Nq == 0 || a->S == 0) return E2F_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    DenseParams A;
    dense_fill(A, a, q, k, v);
    A.out = rows_of(out, a->dtype);
    const unsigned blocks = (unsigned)(dense_tiles(a->Nq, A.group, a->S, DENSE_BM) * a->Hk);
    if (a->dtype == E2F_BF16) launch<uint16_t>(A, blocks, st);
    else launch<float>(A, blocks, st);
    E2F_HIP_CHECK(hipGetLastError());
    return E2F_OK;
}

}  // extern "C"
