// The pages that each token and key head attends to: their scores, and the greatest of them.
#include <algorithm>

#include "spd_paged_device.h"

namespace spd {

namespace {

constexpr int kSelectThreads = 256;

// A workgroup has one token and key head: its queries as 8-bit codes in LDS, then a page to a thread, scores in scratch, and
// the greatest one n_select times.
template <spd_dtype T, int D>
__global__ void __launch_bounds__(kSelectThreads) spd_paged_select_kernel(const PagedAttention a, int32_t *const selected, float *const scores,
                                                                           const int t0) {
    using H = half_t<T>;
    __shared__ __align__(16) int8_t s_code[2][D];                 // u, then w
    __shared__ float s_most[4];
    __shared__ uint64_t s_best[4];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, t = t0 + (int)blockIdx.x, kvh = (int)blockIdx.y, group = a.q.group;
    const int r = paged_request_of(a.req, t);
    if (r < 0) return;
    const PagedRequest rq = paged_request(a.req, a.cache.page_shift, r);
    const int position = rq.kv - rq.count + (t - rq.first);
    int32_t *const out = selected + ((int64_t)t * a.cache.kv_heads + kvh) * a.n_select;
    const int pages = position < 0 ? 0 : (position >> a.cache.page_shift) + 1;
    if (pages <= a.n_select) {
        if (tid < a.n_select) out[tid] = tid < pages ? tid : -1;
        return;
    }
    const H *const q = (const H *)a.q.ptr + t * a.q.token_stride + (int64_t)kvh * group * a.q.head_stride;
    float most = 0.0f;
    for (int i = tid; i < group * D; i += kSelectThreads) most = fmaxf(most, fabsf((float)q[(i / D) * a.q.head_stride + i % D]));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    if (lane == 0) s_most[wave] = most;
    __syncthreads();
    const float step = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3])) * kPagedCodeStep;
    if (tid < D) {
        int up = 0, down = 0;
        for (int g = 0; g < group; ++g) {
            const int c = step > 0.0f ? (int)rintf((float)q[g * a.q.head_stride + tid] / step) : 0;
            up += max(c, 0); down += max(-c, 0);
        }
        const float share = 1.0f / (float)group;
        s_code[0][tid] = (int8_t)rintf((float)up * share);
        s_code[1][tid] = (int8_t)rintf((float)down * share);
    }
    __syncthreads();
    float *const score = scores + ((int64_t)blockIdx.x * a.cache.kv_heads + kvh) * a.req.max_pages;
    const int32_t *const table = a.req.block_table + (int64_t)r * a.req.table_stride;
    for (int p = tid; p < pages; p += kSelectThreads) {
        const int32_t number = table[p];
        float x = -__builtin_inff();
        if (p == 0 || p == pages - 1) x = __builtin_inff();
        else if (number >= 0 && number < a.cache.n_pages) {
            const int64_t at = ((int64_t)number * a.cache.kv_heads + kvh);
            const int8_t *const c = a.cache.codes + at * 2 * D;
            int sum = 0;
            for (int d = 0; d < D; ++d) sum += (int)s_code[0][d] * c[D + d] - (int)s_code[1][d] * c[d];
            x = (float)sum * a.cache.code_scale[at];
        }
        score[p] = x;
    }
    // (one workgroup's own stores: a barrier orders them for it)
    __threadfence_block();
    __syncthreads();
    for (int j = 0; j < a.n_select; ++j) {
        uint64_t best = 0;
        for (int p = tid; p < pages; p += kSelectThreads) {
            const uint32_t b = __float_as_uint(score[p]);
            const uint32_t key = b & 0x80000000u ? ~b : b | 0x80000000u;
            best = max(best, (uint64_t)key << 32 | (uint32_t)~p);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) best = max(best, __shfl_xor(best, d));
        if (lane == 0) s_best[wave] = best;
        __syncthreads();
        best = max(max(s_best[0], s_best[1]), max(s_best[2], s_best[3]));
        const int p = (int)~(uint32_t)best;
        if (tid == 0) { out[j] = p; score[p] = -__builtin_nanf(""); }       // (below every other key)
        __threadfence_block();
        __syncthreads();
    }
    // ascending: every place's rank among the selected
    int mine = 0, rank = 0;
    if (tid < a.n_select) {
        mine = out[tid];
        for (int j = 0; j < a.n_select; ++j) rank += out[j] < mine;
    }
    __syncthreads();
    if (tid < a.n_select) out[rank] = mine;
}

template <spd_dtype T, int D>
void start(hipStream_t st, const PagedAttention &a, int32_t *selected, float *scores, int t0, int count) {
    hipLaunchKernelGGL((spd_paged_select_kernel<T, D>), dim3((unsigned)count, (unsigned)a.cache.kv_heads), dim3(kSelectThreads), 0, st, a,
                       selected, scores, t0);
}

constexpr size_t kScoreBytes = (size_t)256 << 20;                 // tokens whose scores take more are scored in several launches

int tokens_at_once(const PagedAttention &a) {
    const size_t each = std::max<size_t>((size_t)a.cache.kv_heads * (size_t)a.req.max_pages * 4, 1);
    return (int)std::min<size_t>(std::max<size_t>(kScoreBytes / each, 1), (size_t)std::max(a.req.n_tokens, 1));
}

}  // namespace

size_t paged_select_scratch(const PagedAttention &a) {
    return (size_t)tokens_at_once(a) * (size_t)a.cache.kv_heads * (size_t)a.req.max_pages * 4;
}

hipError_t launch_paged_select(hipStream_t st, const PagedAttention &a, int32_t *selected, void *scratch) {
    const int each = tokens_at_once(a);
    for (int t0 = 0; t0 < a.req.n_tokens; t0 += each) {
        const int count = std::min(each, a.req.n_tokens - t0);
        float *const scores = static_cast<float *>(scratch);
        if (a.dtype == SPD_BF16) {
            if (a.head_dim == 64) start<SPD_BF16, 64>(st, a, selected, scores, t0, count);
            else start<SPD_BF16, 128>(st, a, selected, scores, t0, count);
        } else {
            if (a.head_dim == 64) start<SPD_F16, 64>(st, a, selected, scores, t0, count);
            else start<SPD_F16, 128>(st, a, selected, scores, t0, count);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace spd
