// Attention of new tokens over a paged cache, one wave per (token, query head).  64 keys a step: a lane has one key's score, then the
// lanes share the head's elements and walk the keys; running maximum and sum of the softmax, one pass over the keys.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

template <bool BF>
__global__ __launch_bounds__(64) void bcq_attend_kernel(AttendArgs p)
{
    __shared__ float q[BCQ_MAX_HEAD_DIM];
    __shared__ float weight[64];
    __shared__ long long place[64];
    const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x, D = p.cache.head_dim, page = p.cache.page_size;
    int r = 0;
    while (r < p.requests && !(p.q_start[r] <= t && t < p.q_start[r + 1])) ++r;
    if (r == p.requests) return;
    const int start = max(p.q_start[r], 0), n = min(p.q_start[r + 1], p.tokens) - start, i = t - start;
    if (i >= min(n, p.max_new)) return;
    const int len = (int)min((long long)max(p.kv_len[r], 0), (long long)p.max_pages * page), position = len - n + i;
    const int end = p.causal ? min(len, position + 1) : len, begin = p.window ? max(0, position + 1 - p.window) : 0;
    const int kv_head = head / (p.q_heads / p.cache.kv_heads);
    for (int d = lane; d < D; d += 64) q[d] = to_float<BF>(p.q[t * p.ld_q + (long long)head * D + d]);
    float most = -INFINITY, sum = 0.0f, o[BCQ_MAX_HEAD_DIM / 64] = {};
    for (int j0 = begin; j0 < end; j0 += 64) {
        __syncthreads();
        const int j = min(j0 + lane, end - 1);
        const int id = min(max(p.pages[(long long)r * p.max_pages + j / page], 0), p.cache.num_pages - 1);
        const long long at = id * p.cache.page_stride + kv_head * p.cache.head_stride + (j % page) * p.cache.slot_stride;
        float s = 0.0f;
        for (int d = 0; d < D; ++d) s = fmaf(q[d], to_float<BF>(p.k[at + d]), s);
        s = j0 + lane < end ? s * p.scale : -INFINITY;
        float m = s;
        for (int step = 32; step > 0; step >>= 1) m = fmaxf(m, __shfl_xor(m, step));
        m = fmaxf(m, most);
        const float base = m == -INFINITY ? 0.0f : m, shrink = expf(most - base);
        const float e = expf(s - base);
        float es = e;
        for (int step = 32; step > 0; step >>= 1) es += __shfl_xor(es, step);
        sum = sum * shrink + es;
        most = m;
        weight[lane] = e;
        place[lane] = at;
        __syncthreads();
        for (int c = 0; c < BCQ_MAX_HEAD_DIM / 64; ++c) {
            o[c] *= shrink;
            if (lane + 64 * c < D)
                for (int k = 0; k < min(64, end - j0); ++k) o[c] = fmaf(weight[k], to_float<BF>(p.v[place[k] + lane + 64 * c]), o[c]);
        }
    }
    for (int c = 0; c < BCQ_MAX_HEAD_DIM / 64; ++c)
        if (lane + 64 * c < D) p.out[t * p.ld_out + (long long)head * D + lane + 64 * c] = from_float<BF>(begin < end ? o[c] / sum : 0.0f);
}

size_t attend_workspace_bytes(const bcq_cache &, int, int, int, int) { return 0; }

hipError_t launch_attend(const AttendArgs &a, hipStream_t stream)
{
    const dim3 grid(a.tokens, a.q_heads);
    if (a.cache.dtype == BCQ_BF16) bcq_attend_kernel<true><<<grid, 64, 0, stream>>>(a);
    else bcq_attend_kernel<false><<<grid, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace bcq
