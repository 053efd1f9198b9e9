// Norms of queries and keys for each head with the rotation by the position along a chain, and their backward pass.
//   u = w x r, r = (mean x^2 + eps)^(-1/2);  y = Rot(f) u
//   g = Rot(-f) dy;  dw = sum g x r;  dx = r (w g - n mean(n w g)), n = x r
// Bound by memory: a row is read once and written once, everything between stays in registers.
//
// A row of D features lies in LANES = D features / 16 bytes lanes, rounded up to a power of two, so that its sums are a few lane
// exchanges; a wave holds 64 / LANES tokens and walks over heads, so that a token's angles (formed in binary64) serve all heads of
// its wave.  A feature's partner in the rotation lies in the same lane (interleaved), in another lane's same place (half, if
// rotary_dim/2 is a multiple of what a lane holds), or anywhere: then it is read from memory again, out of the L1.
#include "e2f_block.h"

namespace {

using namespace e2f;

constexpr int THREADS = 256;
constexpr int MAX_D = 256;
constexpr int MAX_PARTS = 1024;   // workgroups of the backward pass along the tokens: rows of partial sums of dw

struct QkParams {
    Rows x[2], dy[2], out[2];     // queries, keys
    const float* w[2];
    const int32_t* position;
    float* partial;               // [parts][2][D]
    int32_t N, H[2], D, rot, heads_per_wave;
    float eps;
    double turns[MAX_D / 2];      // turns of pair i for each step of the position
};

enum Partner { IN_LANE, OTHER_LANE, FROM_MEMORY };

// cos and signed sin of a lane's features: y_e = c_e u_e + s_e u_partner(e).  For bf16 by the instructions for turns, whose absolute
// error (1.25e-7 = 2^-22.9 at most over 4 M angles of a turn, 3.4e-8 in the mean) is far below a result's rounding, 2^-8, and about one of binary32
// in the gradients of the weights; with the library's functions the angles were 40 % of the instructions (backward pass of 10 000 tokens 4 % slower).
template <typename T, int V, Partner P>
__device__ __forceinline__ void angles(const QkParams& A, int e0, int position, float (&c)[V], float (&s)[V]) {
    const int half = A.rot >> 1;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int e = e0 + u;
        c[u] = 1.0f;
        s[u] = 0.0f;
        if (P == IN_LANE && (u & 1)) {   // the pair's second feature
            c[u] = c[u - 1];
            s[u] = -s[u - 1];
            continue;
        }
        if (e < A.rot) {
            const int pair = P == IN_LANE ? e >> 1 : (e < half ? e : e - half);
            double t = (double)position * A.turns[pair];
            t -= rint(t);
            float sn, cs;
            if constexpr (sizeof(T) == 2) {
                sn = __builtin_amdgcn_sinf((float)t);
                cs = __builtin_amdgcn_cosf((float)t);
            } else {
                sincospif(2.0f * (float)t, &sn, &cs);
            }
            c[u] = cs;
            s[u] = (P == IN_LANE || e < half) ? -sn : sn;
        }
    }
}

// The partners' values of u (or dy), given this lane's; `again(e)` reads and forms one of them from memory.
template <int V, Partner P, class Again>
__device__ __forceinline__ void partners(const float (&mine)[V], float (&theirs)[V], int e0, int rot, int lanes_half, Again again) {
    if constexpr (P == IN_LANE) {
#pragma unroll
        for (int u = 0; u < V; ++u) theirs[u] = mine[u ^ 1];
    } else if constexpr (P == OTHER_LANE) {
        const int lane = threadIdx.x & 63, from = e0 < (rot >> 1) ? lane + lanes_half : (e0 < rot ? lane - lanes_half : lane);
#pragma unroll
        for (int u = 0; u < V; ++u) theirs[u] = __shfl(mine[u], from);
    } else {
        const int half = rot >> 1;
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const int e = e0 + u;
            theirs[u] = e < rot ? again(e < half ? e + half : e - half) : 0.0f;
        }
    }
}

template <typename T>
__device__ __forceinline__ float one(const char* row, int e) {
    if constexpr (sizeof(T) == 4) return reinterpret_cast<const float*>(row)[e];
    else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[e] << 16);
}

template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

template <typename T, int LANES, Partner P>
__global__ __launch_bounds__(THREADS) void k_qk(QkParams A) {
    constexpr int V = Vec<T>::V, ROWS = THREADS / LANES;
    const int e0 = (threadIdx.x % LANES) * V;
    const int64_t token = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    const bool in = token < A.N && e0 < A.D;
    float c[V], s[V], w[2][V];
    angles<T, V, P>(A, e0, A.rot && token < A.N ? A.position[token] : 0, c, s);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int u = 0; u < V; ++u) w[k][u] = e0 < A.D && A.w[k] ? A.w[k][e0 + u] : 1.0f;
    const int h0 = blockIdx.y * A.heads_per_wave, h1 = min(h0 + A.heads_per_wave, A.H[0] + A.H[1]);
    auto row_of = [&](int hh) { return hh >= A.H[0] ? A.x[1].row(token, hh - A.H[0]) : A.x[0].row(token, hh); };
    auto fetch = [&](int hh) { return in && hh < h1 ? *reinterpret_cast<const u32x4*>(row_of(hh) + e0 * sizeof(T)) : u32x4{0, 0, 0, 0}; };
    u32x4 next = fetch(h0);
    for (int hh = h0; hh < h1; ++hh) {
        const int k = hh >= A.H[0], h = hh - (k ? A.H[0] : 0);
        const char* row = row_of(hh);
        const u32x4 raw = next;
        next = fetch(hh + 1);
        float x[V], sum = 0.0f, t[V], y[V];
        Vec<T>::unpack(raw, x);
#pragma unroll
        for (int u = 0; u < V; ++u) sum += x[u] * x[u];
        const float r = 1.0f / sqrtf(row_sum<LANES>(sum) / (float)A.D + A.eps);
#pragma unroll
        for (int u = 0; u < V; ++u) x[u] *= r * (k ? w[1][u] : w[0][u]);
        partners<V, P>(x, t, e0, A.rot, (A.rot >> 1) / V,
                       [&](int e) { return in ? one<T>(row, e) * (r * (A.w[k] ? A.w[k][e] : 1.0f)) : 0.0f; });
#pragma unroll
        for (int u = 0; u < V; ++u) y[u] = x[u] * c[u] + t[u] * s[u];
        if (in) *reinterpret_cast<u32x4*>(A.out[k].row(token, h) + e0 * sizeof(T)) = Vec<T>::pack(y);
    }
}

template <typename T, int LANES, Partner P>
__global__ __launch_bounds__(THREADS) void k_qk_bwd(QkParams A) {
    constexpr int V = Vec<T>::V, ROWS = THREADS / LANES, PAD = V + 1;
    __shared__ float part[THREADS * PAD];
    const int lane_in_row = threadIdx.x % LANES, e0 = lane_in_row * V;
    float w[2][V], dw[2][V];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int u = 0; u < V; ++u) {
            w[k][u] = e0 < A.D && A.w[k] ? A.w[k][e0 + u] : 1.0f;
            dw[k][u] = 0.0f;
        }
    const int h0 = blockIdx.y * A.heads_per_wave, h1 = min(h0 + A.heads_per_wave, A.H[0] + A.H[1]);
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < A.N; base += (int64_t)gridDim.x * ROWS) {
        const int64_t token = base + threadIdx.x / LANES;
        const bool in = token < A.N && e0 < A.D;
        float c[V], s[V];
        angles<T, V, P>(A, e0, A.rot && token < A.N ? A.position[token] : 0, c, s);
        auto row_of = [&](const Rows (&R)[2], int hh) { return hh >= A.H[0] ? R[1].row(token, hh - A.H[0]) : R[0].row(token, hh); };
        auto fetch = [&](const Rows (&R)[2], int hh) {
            return in && hh < h1 ? *reinterpret_cast<const u32x4*>(row_of(R, hh) + e0 * sizeof(T)) : u32x4{0, 0, 0, 0};
        };
        u32x4 next = fetch(A.x, h0), gnext = fetch(A.dy, h0);
        for (int hh = h0; hh < h1; ++hh) {
            const int k = hh >= A.H[0], h = hh - (k ? A.H[0] : 0);
            const char* grow = row_of(A.dy, hh);
            const u32x4 raw = next, graw = gnext;
            next = fetch(A.x, hh + 1);
            gnext = fetch(A.dy, hh + 1);
            float x[V], y[V], t[V], sum = 0.0f, dot = 0.0f;
            Vec<T>::unpack(raw, x);
            Vec<T>::unpack(graw, y);
            partners<V, P>(y, t, e0, A.rot, (A.rot >> 1) / V, [&](int e) { return in ? one<T>(grow, e) : 0.0f; });
#pragma unroll
            for (int u = 0; u < V; ++u) sum += x[u] * x[u];
            const float r = 1.0f / sqrtf(row_sum<LANES>(sum) / (float)A.D + A.eps);
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const float g = y[u] * c[u] - t[u] * s[u];
                x[u] *= r;
                const float gx = g * x[u];
                if (k) dw[1][u] += gx; else dw[0][u] += gx;
                y[u] = g * (k ? w[1][u] : w[0][u]);
                dot += x[u] * y[u];
            }
            const float mean = row_sum<LANES>(dot) / (float)A.D;
#pragma unroll
            for (int u = 0; u < V; ++u) y[u] = r * (y[u] - x[u] * mean);
            if (in) *reinterpret_cast<u32x4*>(A.out[k].row(token, h) + e0 * sizeof(T)) = Vec<T>::pack(y);
        }
    }
    if (!A.partial) return;
    // over the workgroup's rows, in a fixed order
    const int64_t line = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < V; ++u) part[threadIdx.x * PAD + u] = dw[k][u];
        __syncthreads();
        for (int e = threadIdx.x; e < A.D; e += THREADS) {
            float sum = 0.0f;
            for (int r = 0; r < ROWS; ++r) sum += part[(r * LANES + e / V) * PAD + e % V];
            A.partial[(line * 2 + k) * A.D + e] = sum;
        }
    }
}

// Sums of the partial rows: a workgroup for 16 columns, 64 threads down each.
constexpr int SUM_THREADS = 1024;
__global__ __launch_bounds__(SUM_THREADS) void k_qk_weight_sums(const float* partial, int lines, int D, float* gq, float* gk) {
    constexpr int DOWN = SUM_THREADS / 16;
    __shared__ double s[DOWN][16];
    const int col = blockIdx.x * 16 + threadIdx.x % 16, down = threadIdx.x / 16;
    double sum = 0;
    if (col < 2 * D) {
#pragma unroll 4
        for (int l = down; l < lines; l += DOWN) sum += (double)partial[(int64_t)l * 2 * D + col];
    }
    s[down][threadIdx.x % 16] = sum;
    for (int o = DOWN / 2; o; o >>= 1) {
        __syncthreads();
        if (down < o) s[down][threadIdx.x % 16] += s[down + o][threadIdx.x % 16];
    }
    if (down == 0 && col < 2 * D) {
        float* g = col < D ? gq : gk;
        if (g) g[col < D ? col : col - D] = (float)s[0][threadIdx.x];
    }
}

e2f_status check(const e2f_qk_args* a) {
    if (!a || (a->dtype != E2F_F32 && a->dtype != E2F_BF16) || a->N < 0 || a->Hq < 0 || a->Hk < 0 || a->D <= 0)
        return E2F_ERR_INVALID_ARG;
    if (a->rotary_dim < 0 || a->rotary_dim > a->D || (a->rotary_dim & 1)) return E2F_ERR_INVALID_ARG;
    if (a->layout != E2F_ROTARY_HALF && a->layout != E2F_ROTARY_INTERLEAVED) return E2F_ERR_INVALID_ARG;
    if (!(a->eps > 0.0f) || !isfinite(a->eps) || !(a->theta > 0.0) || !isfinite(a->theta) || !isfinite(a->position_scale))
        return E2F_ERR_INVALID_ARG;
    // every pair's angle at a position of up to 2^31 has to be a binary64 number; the rates are 1 and, at the last pair, theta^(2/rotary_dim - 1)
    const double rate = a->rotary_dim ? fmax(1.0, pow(a->theta, 2.0 / a->rotary_dim - 1.0)) : 1.0;
    if (!isfinite(fabs(a->position_scale) * rate * 0x1p31)) return E2F_ERR_INVALID_ARG;
    if (a->D % 8 || a->D > MAX_D || a->Hq > 1024 || a->Hk > 1024) return E2F_ERR_UNSUPPORTED;
    if (a->N > 0 && a->rotary_dim > 0 && !a->position) return E2F_ERR_INVALID_ARG;
    if (!word_aligned(a->position) || !word_aligned(a->weight_q) || !word_aligned(a->weight_k)) return E2F_ERR_INVALID_ARG;
    return E2F_OK;
}

int lanes_of(const e2f_qk_args* a) {
    int lanes = 1;
    while (lanes * 16 < a->D * elem_bytes(a->dtype)) lanes *= 2;
    return lanes;
}

void fill(QkParams& A, const e2f_qk_args* a) {
    A.w[0] = a->weight_q;
    A.w[1] = a->weight_k;
    A.position = a->position;
    A.partial = nullptr;
    A.N = a->N;
    A.H[0] = a->Hq;
    A.H[1] = a->Hk;
    A.D = a->D;
    A.rot = a->rotary_dim;
    A.eps = a->eps;
    for (int i = 0; i < a->rotary_dim / 2; ++i)
        A.turns[i] = a->position_scale * pow(a->theta, -2.0 * i / a->rotary_dim) / 6.283185307179586476925286766559;
}

// Grid along the tokens and the heads.  Heads of a token share its angles, so a wave takes all of them where the tokens alone make
// enough workgroups, and fewer heads where they do not.  For 640 workgroups or more, from both sides (a training step, 16 heads, with
// 320 / 640 / 1 280 workgroups): 3 000 tokens of 64 bf16 features 22.9 / 22.4 / 22.0 us, 10 000 37.6 / 36.6 / 41.3, 30 000 77.2 / 77.3 / 88.1; in
// fp32 30.6 / 24.1 / 25.8, 63.4 / 54.1 / 58.2, 138 / 139 / 146; 10 000 tokens of 16 bf16 features 21.9 / 22.5 / 31.0, 3 000 of 128 37.5 / 34.1 /
// 41.5.  One share of the heads takes 37 us for 300 tokens in place of 12.
struct Grid {
    unsigned x, y;
    int heads_per_wave;
};
Grid grid_of(const e2f_qk_args* a, int64_t most_x) {
    const int rows = THREADS / lanes_of(a), heads = a->Hq + a->Hk;
    int64_t x = ((int64_t)a->N + rows - 1) / rows;
    if (x > most_x) x = most_x;
    int64_t split = (640 + x - 1) / x;
    if (split > heads) split = heads;
    const int per = (heads + (int)split - 1) / (int)split;
    return Grid{(unsigned)x, (unsigned)((heads + per - 1) / per), per};
}

Partner partner_of(const e2f_qk_args* a) {
    if (a->layout == E2F_ROTARY_INTERLEAVED) return IN_LANE;
    return (a->rotary_dim / 2) % (16 / elem_bytes(a->dtype)) == 0 ? OTHER_LANE : FROM_MEMORY;
}

template <bool BWD, typename T, int LANES>
void launch_partner(const e2f_qk_args* a, const QkParams& A, const Grid& g, hipStream_t st) {
    auto go = [&](auto fwd, auto bwd) {
        if constexpr (BWD) bwd<<<dim3(g.x, g.y), THREADS, 0, st>>>(A);
        else fwd<<<dim3(g.x, g.y), THREADS, 0, st>>>(A);
    };
    switch (partner_of(a)) {
        case IN_LANE: go(k_qk<T, LANES, IN_LANE>, k_qk_bwd<T, LANES, IN_LANE>); break;
        case OTHER_LANE: go(k_qk<T, LANES, OTHER_LANE>, k_qk_bwd<T, LANES, OTHER_LANE>); break;
        default: go(k_qk<T, LANES, FROM_MEMORY>, k_qk_bwd<T, LANES, FROM_MEMORY>); break;
    }
}

template <bool BWD>
void launch(const e2f_qk_args* a, const QkParams& A, const Grid& g, hipStream_t st) {
    const int lanes = lanes_of(a);
    if (a->dtype == E2F_BF16) {
        switch (lanes) {
            case 1: launch_partner<BWD, uint16_t, 1>(a, A, g, st); break;
            case 2: launch_partner<BWD, uint16_t, 2>(a, A, g, st); break;
            case 4: launch_partner<BWD, uint16_t, 4>(a, A, g, st); break;
            case 8: launch_partner<BWD, uint16_t, 8>(a, A, g, st); break;
            case 16: launch_partner<BWD, uint16_t, 16>(a, A, g, st); break;
            default: launch_partner<BWD, uint16_t, 32>(a, A, g, st); break;
        }
    } else {
        switch (lanes) {
            case 2: launch_partner<BWD, float, 2>(a, A, g, st); break;
            case 4: launch_partner<BWD, float, 4>(a, A, g, st); break;
            case 8: launch_partner<BWD, float, 8>(a, A, g, st); break;
            case 16: launch_partner<BWD, float, 16>(a, A, g, st); break;
            case 32: launch_partner<BWD, float, 32>(a, A, g, st); break;
            default: launch_partner<BWD, float, 64>(a, A, g, st); break;
        }
    }
}

}  // namespace

extern "C" {

e2f_status e2f_qk_norm_rotate(const e2f_qk_args* a, const e2f_heads* q, const e2f_heads* k, const e2f_heads* q_out,
                              const e2f_heads* k_out, void* hip_stream) {
    e2f_status rc = check(a);
    if (rc != E2F_OK) return rc;
    if ((rc = check_rows(q, a->dtype, a->N, a->Hq)) != E2F_OK || (rc = check_rows(k, a->dtype, a->N, a->Hk)) != E2F_OK ||
        (rc = check_result_rows(q_out, a->dtype, a->N, a->Hq, a->D)) != E2F_OK ||
        (rc = check_result_rows(k_out, a->dtype, a->N, a->Hk, a->D)) != E2F_OK)
        return rc;
    if (a->N == 0 || a->Hq + a->Hk == 0) return E2F_OK;
    QkParams A;
    fill(A, a);
    A.x[0] = rows_of(q, a->dtype);
    A.x[1] = rows_of(k, a->dtype);
    A.dy[0] = A.dy[1] = Rows{nullptr, 0, 0};
    A.out[0] = rows_of(q_out, a->dtype);
    A.out[1] = rows_of(k_out, a->dtype);
    // as many tokens at a time as one launch has threads for
    const int rows = THREADS / lanes_of(a);
    const int64_t most = (MOST_THREADS / THREADS - 1) * rows;
    for (int64_t first = 0; first < a->N; first += most) {
        e2f_qk_args part = *a;
        part.N = A.N = (int32_t)(a->N - first < most ? a->N - first : most);
        const Grid g = grid_of(&part, INT32_MAX);
        A.heads_per_wave = g.heads_per_wave;
        launch<false>(a, A, g, static_cast<hipStream_t>(hip_stream));
        E2F_HIP_CHECK(hipGetLastError());
        if (A.position) A.position += A.N;
        for (int k = 0; k < 2; ++k) {
            if (A.x[k].ptr) A.x[k].ptr += A.N * A.x[k].token_bytes;
            if (A.out[k].ptr) A.out[k].ptr += A.N * A.out[k].token_bytes;
        }
    }
    return E2F_OK;
}

size_t e2f_qk_norm_rotate_backward_workspace_bytes(const e2f_qk_args* a) {
    if (check(a) != E2F_OK || a->N == 0 || a->Hq + a->Hk == 0) return 0;
    const Grid g = grid_of(a, MAX_PARTS);
    return (size_t)g.x * g.y * 2 * a->D * sizeof(float);
}

e2f_status e2f_qk_norm_rotate_backward(const e2f_qk_args* a, const e2f_heads* q, const e2f_heads* k,
                                       const e2f_heads* grad_q_out, const e2f_heads* grad_k_out, const e2f_heads* grad_q,
                                       const e2f_heads* grad_k, float* grad_weight_q, float* grad_weight_k, void* ws,
                                       size_t ws_bytes, void* hip_stream) {
    e2f_status rc = check(a);
    if (rc != E2F_OK) return rc;
    if ((rc = check_rows(q, a->dtype, a->N, a->Hq)) != E2F_OK || (rc = check_rows(k, a->dtype, a->N, a->Hk)) != E2F_OK ||
        (rc = check_rows(grad_q_out, a->dtype, a->N, a->Hq)) != E2F_OK ||
        (rc = check_rows(grad_k_out, a->dtype, a->N, a->Hk)) != E2F_OK ||
        (rc = check_result_rows(grad_q, a->dtype, a->N, a->Hq, a->D)) != E2F_OK ||
        (rc = check_result_rows(grad_k, a->dtype, a->N, a->Hk, a->D)) != E2F_OK)
        return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool empty = a->N == 0 || a->Hq + a->Hk == 0, sums = grad_weight_q || grad_weight_k;
    if (!word_aligned(grad_weight_q) || !word_aligned(grad_weight_k)) return E2F_ERR_INVALID_ARG;
    const size_t need = e2f_qk_norm_rotate_backward_workspace_bytes(a);
    if (need && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < need) return E2F_ERR_WORKSPACE_TOO_SMALL;
    Grid g = {0, 0, 0};
    if (!empty) {
        QkParams A;
        fill(A, a);
        A.x[0] = rows_of(q, a->dtype);
        A.x[1] = rows_of(k, a->dtype);
        A.dy[0] = rows_of(grad_q_out, a->dtype);
        A.dy[1] = rows_of(grad_k_out, a->dtype);
        A.out[0] = rows_of(grad_q, a->dtype);
        A.out[1] = rows_of(grad_k, a->dtype);
        A.partial = sums ? static_cast<float*>(ws) : nullptr;
        g = grid_of(a, MAX_PARTS);
        A.heads_per_wave = g.heads_per_wave;
        launch<true>(a, A, g, st);
        E2F_HIP_CHECK(hipGetLastError());
    }
    if (sums) {   // without rows: zeros
        k_qk_weight_sums<<<(2 * a->D + 15) / 16, SUM_THREADS, 0, st>>>(static_cast<float*>(ws), (int)(g.x * g.y), a->D,
                                                                  grad_weight_q, grad_weight_k);
        E2F_HIP_CHECK(hipGetLastError());
    }
    return E2F_OK;
}

}  // extern "C"
