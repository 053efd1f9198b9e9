// What the operators of the all-pair block share: rows of heads on the host and the device, conversions, sums.
#pragma once
#include <math.h>

#include "e2f_internal.h"

namespace e2f {

// ---- host: checks of the rows of heads --------------------------------------------------------------------------

static inline int elem_bytes(int32_t dtype) { return dtype == E2F_BF16 ? 2 : 4; }

// Rows that are read: [N][H][D], 16-byte aligned rows at strides >= 0.
static inline e2f_status check_rows(const e2f_heads* x, int32_t dtype, int64_t N, int32_t H) {
    if (N == 0 || H == 0) return E2F_OK;
    if (!x || !x->ptr || x->token_stride < 0 || x->head_stride < 0) return E2F_ERR_INVALID_ARG;
    const int64_t a = 16 / elem_bytes(dtype);
    if ((reinterpret_cast<uintptr_t>(x->ptr) & 15u) || x->token_stride % a || x->head_stride % a) return E2F_ERR_UNSUPPORTED;
    // the last element's byte offset has to be a 63-bit number
    const int64_t far = INT64_MAX / 8;
    if ((N > 1 && x->token_stride > far / N) || (H > 1 && x->head_stride > far / H)) return E2F_ERR_INVALID_ARG;
    // kernels form offsets of up to 64 rows in 32 bits
    if (N > 1 && x->token_stride * elem_bytes(dtype) >= (1 << 25)) return E2F_ERR_UNSUPPORTED;
    return E2F_OK;
}

// Rows that are written: besides, no two of them may share an element.
static inline e2f_status check_result_rows(const e2f_heads* x, int32_t dtype, int64_t N, int32_t H, int32_t D) {
    const e2f_status rc = check_rows(x, dtype, N, H);
    if (rc != E2F_OK || N == 0 || H == 0) return rc;
    const int64_t t = N > 1 ? x->token_stride : INT64_MAX, h = H > 1 ? x->head_stride : INT64_MAX;
    if (t < D || h < D) return E2F_ERR_INVALID_ARG;
    if (N > 1 && H > 1 && !(t >= (H - 1) * h + D || h >= (N - 1) * t + D)) return E2F_ERR_INVALID_ARG;
    return E2F_OK;
}

// A launch has fewer than 2^32 threads along x.
constexpr int64_t MOST_THREADS = (int64_t)1 << 32;
static inline bool launches(int64_t blocks, int threads) { return blocks * threads < MOST_THREADS; }

// Whether 4-byte elements may lie there (or nothing does).
static inline bool word_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static inline bool aligned_ws(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

// ---- device -------------------------------------------------------------------------------------------------------

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Device form of e2f_heads.
struct Rows {
    char* ptr;
    int64_t token_bytes, head_bytes;
    __device__ __forceinline__ char* row(int64_t t, int64_t h) const { return ptr + t * token_bytes + h * head_bytes; }
};
static inline Rows rows_of(const e2f_heads* x, int32_t dtype) {
    if (!x) return Rows{nullptr, 0, 0};
    const int b = elem_bytes(dtype);
    return Rows{static_cast<char*>(x->ptr), x->token_stride * b, x->head_stride * b};
}

// 16 bytes of features as binary32 and back; V features of the type make 16 bytes.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void unpack(u32x4 x, float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[4]) {
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(f[i]);
        return x;
    }
};
// two binary32 values rounded to nearest even, the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
template <>
struct Vec<uint16_t> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(u32x4 x, float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(x[i] << 16);
            f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
        return x;
    }
};

}  // namespace e2f
