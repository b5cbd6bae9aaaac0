// Attention of a chunk of new tokens over a paged cache, over all of its pages or over selected ones.
#include "spd_paged_device.h"

namespace spd {

namespace {

// A wavefront has one query row: two places (D = 128) or one of it to a lane, key after key, with the running maximum and sum of the
// softmax.
template <spd_dtype T, int D, bool SELECTED>
__global__ void __launch_bounds__(256) spd_paged_attention_kernel(const PagedAttention a) {
    using H = half_t<T>;
    constexpr int E = D / 64;
    const int lane = (int)threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    const int t = (int)(row / a.q.heads), h = (int)(row % a.q.heads), kvh = h / a.q.group;
    if (t >= a.req.n_tokens) return;
    const int r = paged_request_of(a.req, t);
    if (r < 0) return;
    const PagedRequest rq = paged_request(a.req, a.cache.page_shift, r);
    const int position = rq.kv - rq.count + (t - rq.first);
    const int32_t *const table = a.req.block_table + (int64_t)r * a.req.table_stride;
    float q[E], acc[E], top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = (float)((const H *)a.q.ptr)[t * a.q.token_stride + h * a.q.head_stride + lane * E + e] * a.q.scale;
        acc[e] = 0.0f;
    }
    const int pages = SELECTED ? a.n_select : (position >> a.cache.page_shift) + 1;
    for (int i = 0; i < pages; ++i) {
        const int col = SELECTED ? a.selected[((int64_t)t * a.cache.kv_heads + kvh) * a.n_select + i] : i;
        if (col < 0) break;
        const int32_t number = table[col];
        if (number < 0 || number >= a.cache.n_pages) continue;
        const int first = col << a.cache.page_shift, many = min(1 << a.cache.page_shift, position + 1 - first);
        const int64_t at = number * a.cache.page_stride + kvh * a.cache.head_stride + lane * E;
        for (int j = 0; j < many; ++j) {
            const H *const k = (const H *)a.cache.k + at + j * a.cache.token_stride, *const v = (const H *)a.cache.v + at + j * a.cache.token_stride;
            float x = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) x += q[e] * (float)k[e];
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d);
            const float now = fmaxf(top, x), old = exp2f(top - now), p = exp2f(x - now);
            top = now;
            sum = sum * old + p;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = acc[e] * old + p * (float)v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) ((H *)a.out.out)[((int64_t)t * a.q.heads + h) * D + lane * E + e] = (H)(sum > 0.0f ? acc[e] / sum : 0.0f);
    if (lane == 0 && a.out.lse) a.out.lse[(int64_t)t * a.q.heads + h] = sum > 0.0f ? (top + log2f(sum)) * 0.6931471805599453f : -__builtin_inff();
}

template <spd_dtype T, int D>
void start(hipStream_t st, const PagedAttention &a) {
    const dim3 grid((unsigned)(((int64_t)a.req.n_tokens * a.q.heads + 3) / 4));
    if (a.selected) hipLaunchKernelGGL((spd_paged_attention_kernel<T, D, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((spd_paged_attention_kernel<T, D, false>), grid, dim3(256), 0, st, a);
}

}  // namespace

size_t paged_attention_scratch(const PagedAttention &, int) { return 0; }

hipError_t launch_paged_attention(hipStream_t st, const PagedAttention &a, void *, int) {
    if (a.req.n_tokens == 0) return hipSuccess;
    if (a.dtype == SPD_BF16) { if (a.head_dim == 64) start<SPD_BF16, 64>(st, a); else start<SPD_BF16, 128>(st, a); }
    else { if (a.head_dim == 64) start<SPD_F16, 64>(st, a); else start<SPD_F16, 128>(st, a); }
    return hipGetLastError();
}

}  // namespace spd
