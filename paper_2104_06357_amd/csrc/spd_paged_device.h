// What the kernels over a paged cache share: types of 16 bits, and where a request's tokens lie.
#pragma once
#include "spd_paged.h"

namespace spd {

template <spd_dtype T> struct Half;
template <> struct Half<SPD_BF16> { using type = __bf16; };
template <> struct Half<SPD_F16> { using type = _Float16; };
template <spd_dtype T> using half_t = typename Half<T>::type;
template <spd_dtype T> using half8_t = half_t<T> __attribute__((ext_vector_type(8)));
template <spd_dtype T> using half4_t = half_t<T> __attribute__((ext_vector_type(4)));

// Codes of 8 bits are multiples of the greatest magnitude times this.
constexpr float kPagedCodeStep = 1.0f / 127.0f;

// A request as its kernels see it: lengths that contradict the arrays are cut to them.
struct PagedRequest { int32_t first, count, kv; };
__device__ __forceinline__ PagedRequest paged_request(const PagedRequests &q, int page_shift, int r) {
    PagedRequest p;
    const int32_t end = min(max(q.query_start[r + 1], 0), q.n_tokens);
    p.first = min(max(q.query_start[r], 0), end);
    p.count = end - p.first;
    const int64_t most = (int64_t)q.max_pages << page_shift;
    p.kv = (int32_t)min((int64_t)max(q.kv_lens[r], 0), most);
    return p;
}

// The request of a token: the last one that begins at or before it (-1: none).
__device__ __forceinline__ int paged_request_of(const PagedRequests &q, int token) {
    int lo = 0, hi = q.n_requests;                       // query_start[lo] <= token < query_start[hi], where there are such
    if (q.n_requests == 0 || q.query_start[0] > token || q.query_start[hi] <= token) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q.query_start[mid] <= token) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- matrix products of 16-bit values and their operands -------------------------------------------
// Lane l of a 32x32x16 product holds, of both operands, row l % 32 and the places (l / 32) * 8 .. + 7 of the contraction, and of the result
// column l % 32 and rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15; of a 16x16x32 product row l % 16 and places (l / 16) * 8 .. + 7, and column
// l % 16, rows 4 (l / 16) + i.

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(half8_t<SPD_BF16> a, half8_t<SPD_BF16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(half8_t<SPD_F16> a, half8_t<SPD_F16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(half8_t<SPD_BF16> a, half8_t<SPD_BF16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(half8_t<SPD_F16> a, half8_t<SPD_F16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Of every 16 lanes: lane s names 4 values, the columns 4 (s % 4) .. + 3 of row s / 4, and lane i gets column i of the four rows.
template <spd_dtype T>
__device__ __forceinline__ half4_t<T> read_transposed(const half_t<T> *lds) {
    typedef __attribute__((address_space(3))) i16x4 *Lds;
    return __builtin_bit_cast(half4_t<T>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)(__attribute__((address_space(3))) void *)lds));
}

template <spd_dtype T>
__device__ __forceinline__ half8_t<T> rounded(const float *x) {
    half8_t<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (half_t<T>)x[i];
    return r;
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

}  // namespace spd
