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

}  // namespace spd
