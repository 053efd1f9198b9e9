// Global norm of many gradient tensors and clipping by it: norm = (sum g^2)^(1/2), out = g min(1, max / (norm + 1e-6)).
// Bound by memory: every element is read for the norm, read again and written for the scaling.
//
// The tensors are cut into chunks of one length, a workgroup each, so that a few large and many tiny tensors load the
// chip alike.  A chunk's sum of squares is a binary64 partial sum in the workspace; the scaling kernel's workgroups each
// sum all of these (out of the L2) in the same order, which saves the launch and the wait of a reduction of its own and gives every workgroup
// the same factor.  They are about 2 000, and one for each tensor at least: with thousands of small tensors every workgroup sums thousands
// (1 000 tensors of 2 000 elements take 79 us, 3 000 277 us, 10 000 1 315 us).  Tensors travel in the kernel's arguments, TENSORS of
// them a launch, so that a captured graph needs no table in device memory.
#include <float.h>

#include "e2f_block.h"

namespace {

using namespace e2f;

constexpr int TENSORS = 112;     // 28 bytes each: within the 4 KB that kernel arguments may have
constexpr int THREADS = 256;
constexpr int64_t MIN_CHUNK = 4096, TARGET_CHUNKS = 2048;

struct Batch {
    const void* in[TENSORS];
    void* out[TENSORS];
    int64_t count[TENSORS];
    int32_t first[TENSORS];      // the tensor's first workgroup of this launch; bit 31: bf16
    int32_t n, chunks;
    int64_t chunk;
};
static_assert(sizeof(Batch) <= 4096 - 64, "kernel arguments");

// 16 bytes at any element.
template <typename T>
using Loose = u32x4 __attribute__((aligned(sizeof(T))));

__device__ __forceinline__ double block_sum(double x, double* s) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) t += s[w];
    __syncthreads();
    return t;
}

// The tensor that workgroup b works on: the last one whose first workgroup is at most b.
__device__ __forceinline__ int tensor_of(const Batch& B, int b) {
    int lo = 0, hi = B.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((B.first[mid] & 0x7FFFFFFF) <= b) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Whole vectors of a chunk, AHEAD of them on their way at once for each thread: body(first element, the vector).
constexpr int AHEAD = 4;
template <typename T, class Body>
__device__ __forceinline__ void vectors(const T* p, int64_t whole, Body body) {
    constexpr int V = Vec<T>::V;
    int64_t i = (int64_t)threadIdx.x * V;
    for (; i + (AHEAD - 1) * THREADS * V < whole; i += AHEAD * THREADS * V) {
        u32x4 x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) x[j] = *reinterpret_cast<const Loose<T>*>(p + i + j * THREADS * V);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) body(i + j * THREADS * V, x[j]);
    }
    for (; i < whole; i += THREADS * V) body(i, *reinterpret_cast<const Loose<T>*>(p + i));
}

template <typename T>
__device__ __forceinline__ double squares(const T* p, int64_t n) {
    constexpr int V = Vec<T>::V;
    double sum = 0;
    const int64_t whole = n / V * V;
    vectors(p, whole, [&](int64_t, u32x4 x) {
        float f[V];
        Vec<T>::unpack(x, f);
#pragma unroll
        for (int u = 0; u < V; ++u) sum += (double)f[u] * (double)f[u];
    });
    for (int64_t i = whole + threadIdx.x; i < n; i += THREADS) {
        float f;
        if constexpr (sizeof(T) == 4) f = p[i]; else f = __uint_as_float((uint32_t)p[i] << 16);
        sum += (double)f * (double)f;
    }
    return sum;
}

__global__ __launch_bounds__(THREADS) void k_clip_squares(Batch B, double* partial) {
    __shared__ double s[THREADS / 64];
    const int b = blockIdx.x, t = tensor_of(B, b), first = B.first[t];
    const int64_t at = (int64_t)(b - (first & 0x7FFFFFFF)) * B.chunk, n = min(B.chunk, B.count[t] - at);
    double sum;
    if (first < 0) sum = squares(static_cast<const uint16_t*>(B.in[t]) + at, n);
    else sum = squares(static_cast<const float*>(B.in[t]) + at, n);
    sum = block_sum(sum, s);
    if (threadIdx.x == 0) partial[b] = sum;
}

// F: float, or double where the factor is below binary32's normal numbers and would lose its last bits there.
template <typename T, typename F>
__device__ __forceinline__ void scaled(const T* p, T* q, int64_t n, F factor) {
    constexpr int V = Vec<T>::V;
    const int64_t whole = n / V * V;
    vectors(p, whole, [&](int64_t i, u32x4 x) {
        float f[V];
        Vec<T>::unpack(x, f);
#pragma unroll
        for (int u = 0; u < V; ++u) f[u] = (float)(f[u] * factor);
        *reinterpret_cast<Loose<T>*>(q + i) = Vec<T>::pack(f);
    });
    for (int64_t i = whole + threadIdx.x; i < n; i += THREADS) {
        if constexpr (sizeof(T) == 4) q[i] = (float)(p[i] * factor);
        else q[i] = (uint16_t)pack_bf16((float)(__uint_as_float((uint32_t)p[i] << 16) * factor), 0.0f);
    }
}

// Bits unchanged, as out = g asks for (a multiplication by 1 would quieten a NaN).
template <typename T>
__device__ __forceinline__ void copied(const T* p, T* q, int64_t n) {
    if (p == q) return;
    constexpr int V = Vec<T>::V;
    const int64_t whole = n / V * V;
    vectors(p, whole, [&](int64_t i, u32x4 x) { *reinterpret_cast<Loose<T>*>(q + i) = x; });
    for (int64_t i = whole + threadIdx.x; i < n; i += THREADS) q[i] = p[i];
}

// n_partial: of all launches, not of this one alone.  B.n == 0: the norm alone.
__global__ __launch_bounds__(THREADS) void k_clip_scale(Batch B, const double* partial, int n_partial, float max_norm,
                                                        float* norm) {
    __shared__ double s[THREADS / 64];
    double sum = 0;
    for (int i = threadIdx.x; i < n_partial; i += THREADS) sum += partial[i];
    sum = block_sum(sum, s);
    const double root = sqrt(sum), ratio = (double)max_norm / (root + 1e-6);
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm) *norm = (float)root;
    if (!B.n) return;
    const int b = gridDim.x - 1 - blockIdx.x;      // the last chunks first: the pass before has just read them
    const int t = tensor_of(B, b), first = B.first[t];
    const int64_t at = (int64_t)(b - (first & 0x7FFFFFFF)) * B.chunk, n = min(B.chunk, B.count[t] - at);
    const bool clip = ratio < 1.0 && root < (double)INFINITY;   // false for a NaN too
    auto chunk = [&](const auto* p, auto* q) {
        if (!clip) copied(p, q, n);
        else if (ratio >= (double)FLT_MIN) scaled(p, q, n, (float)ratio);
        else scaled(p, q, n, ratio);
    };
    if (first < 0) chunk(static_cast<const uint16_t*>(B.in[t]) + at, static_cast<uint16_t*>(B.out[t]) + at);
    else chunk(static_cast<const float*>(B.in[t]) + at, static_cast<float*>(B.out[t]) + at);
}

// Chunk length: TARGET_CHUNKS workgroups fill the chip several times over; below MIN_CHUNK a workgroup would not have four
// vectors to a thread.  Returns the number of chunks, -1 if the counts make no sense.
int64_t plan(int32_t n, const int64_t* counts, int64_t* chunk) {
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (counts[i] < 0 || counts[i] > INT64_MAX / 16 - total) return -1;
        total += counts[i];
    }
    int64_t c = (total + TARGET_CHUNKS - 1) / TARGET_CHUNKS;
    c = c < MIN_CHUNK ? MIN_CHUNK : (c + 1023) / 1024 * 1024;
    int64_t chunks = 0;
    for (int32_t i = 0; i < n; ++i) chunks += (counts[i] + c - 1) / c;
    *chunk = c;
    return chunks;
}

}  // namespace

extern "C" {

size_t e2f_grad_norm_clip_workspace_bytes(int32_t n, const int64_t* counts) {
    int64_t chunk;
    if (n < 0 || (n > 0 && !counts)) return 0;
    const int64_t chunks = plan(n, counts, &chunk);
    return chunks < 0 ? 0 : (size_t)chunks * sizeof(double);
}

e2f_status e2f_grad_norm_clip(int32_t n, void* const* grads, void* const* out, const int64_t* counts, const int32_t* dtypes,
                              float max_norm, float* norm, void* ws, size_t ws_bytes, void* hip_stream) {
    if (n < 0 || !(max_norm > 0.0f) || !norm || (reinterpret_cast<uintptr_t>(norm) & 3u)) return E2F_ERR_INVALID_ARG;
    if (n > 0 && (!grads || !out || !counts || !dtypes)) return E2F_ERR_INVALID_ARG;
    int64_t chunk;
    const int64_t chunks = plan(n, counts, &chunk);
    if (chunks < 0 || chunks > INT32_MAX) return E2F_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (dtypes[i] != E2F_F32 && dtypes[i] != E2F_BF16) return E2F_ERR_INVALID_ARG;
        const uintptr_t odd = elem_bytes(dtypes[i]) - 1;
        if (counts[i] > 0 && (!grads[i] || !out[i] || (reinterpret_cast<uintptr_t>(grads[i]) & odd) ||
                              (reinterpret_cast<uintptr_t>(out[i]) & odd)))
            return E2F_ERR_INVALID_ARG;
    }
    if (chunks > 0 && (!ws || !aligned_ws(ws))) return E2F_ERR_INVALID_ARG;
    if (ws_bytes < (size_t)chunks * sizeof(double)) return E2F_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    double* partial = static_cast<double*>(ws);
    for (int pass = 0; pass < 2; ++pass) {
        int64_t done = 0;
        int32_t i = 0;
        do {
            Batch B;
            B.n = 0;
            B.chunk = chunk;
            int64_t blocks = 0;
            for (; i < n && B.n < TENSORS; ++i) {
                if (counts[i] == 0) continue;
                B.in[B.n] = grads[i];
                B.out[B.n] = out[i];
                B.count[B.n] = counts[i];
                B.first[B.n] = (int32_t)((uint32_t)blocks | (dtypes[i] == E2F_BF16 ? 0x80000000u : 0u));
                B.n++;
                blocks += (counts[i] + chunk - 1) / chunk;
            }
            B.chunks = (int32_t)blocks;
            if (pass == 0 && blocks) k_clip_squares<<<(unsigned)blocks, THREADS, 0, st>>>(B, partial + done);
            if (pass == 1 && (blocks || !done))
                k_clip_scale<<<(unsigned)(blocks ? blocks : 1), THREADS, 0, st>>>(B, partial, (int)chunks, max_norm,
                                                                                  done ? nullptr : norm);
            E2F_HIP_CHECK(hipGetLastError());
            done += blocks;
        } while (i < n);
    }
    return E2F_OK;
}

}  // extern "C"
