// Norm of the q and k heads, rotation by position, append of k and v to the paged cache.  A wave has one head of one token: lane l its
// elements l, l + 64, ..., kept in LDS between the norm and the rotation, whose pairs may be any two lanes apart.
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

template <bool BF>
__global__ __launch_bounds__(64) void bcq_rotate_kernel(RotateArgs p)
{
    __shared__ float x[BCQ_MAX_HEAD_DIM];
    const int D = p.cache.head_dim, lane = threadIdx.x, t = blockIdx.x, head = blockIdx.y;
    const int qh = p.q_heads, kvh = p.cache.kv_heads;
    const uint16_t *src = p.qkv + (long long)t * p.ld_qkv + (long long)head * D;
    const bool is_q = head < qh, is_v = head >= qh + kvh;
    const uint16_t *weight = is_v ? nullptr : is_q ? p.q_weight : p.k_weight;
    float square = 0.0f;
    for (int d = lane; d < D; d += 64) {
        x[d] = to_float<BF>(src[d]);
        square += x[d] * x[d];
    }
    for (int step = 32; step > 0; step >>= 1) square += __shfl_xor(square, step);
    if (weight) {
        const float unit = 1.0f / sqrtf(square / D + p.eps);
        for (int d = lane; d < D; d += 64) x[d] = x[d] * unit * to_float<BF>(weight[d]);
    }
    __syncthreads();
    uint16_t *dst;
    if (is_q) {
        dst = p.q_out + (long long)t * p.ld_q + (long long)head * D;
    } else {
        const int slot = p.slots[t];
        if (slot < 0 || slot >= p.cache.num_pages * p.cache.page_size) return;
        dst = (is_v ? p.v : p.k) + (long long)(slot / p.cache.page_size) * p.cache.page_stride +
              (long long)(slot % p.cache.page_size) * p.cache.slot_stride + (long long)(head - qh - (is_v ? kvh : 0)) * p.cache.head_stride;
    }
    const int rot = is_v ? 0 : p.rot_dim, half = rot / 2;
    const float *turn = p.cos_sin + (long long)min(max(p.positions[t], 0), p.max_position - 1) * rot;
    for (int d = lane; d < D; d += 64) {
        float v = x[d];
        if (d < rot) {
            const int pair = p.interleaved ? d / 2 : d % half;
            const bool second = p.interleaved ? d & 1 : d >= half;
            const float other = x[p.interleaved ? d ^ 1 : second ? d - half : d + half];
            v = second ? v * turn[pair] + other * turn[half + pair] : v * turn[pair] - other * turn[half + pair];
        }
        dst[d] = from_float<BF>(v);
    }
}

hipError_t launch_rotate(const RotateArgs &a, hipStream_t stream)
{
    const dim3 grid(a.tokens, a.q_heads + 2 * a.cache.kv_heads);
    if (a.cache.dtype == BCQ_BF16) bcq_rotate_kernel<true><<<grid, 64, 0, stream>>>(a);
    else bcq_rotate_kernel<false><<<grid, 64, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace bcq
