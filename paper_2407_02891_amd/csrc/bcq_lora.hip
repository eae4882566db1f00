// Low-rank adapters of many requests: v = A x in one launch (a wave per token and rank row), Y = base + scale * B v in a second (a thread
// per token and output row).
#include "bcq_half.h"
#include "bcq_internal.h"

namespace bcq {

namespace {

__device__ __forceinline__ int adapter_rank(const LoraArgs &p, int a) { return p.rank ? min(max(p.rank[a], 0), p.desc.max_rank) : p.desc.max_rank; }

}  // namespace

template <bool BF>
__global__ __launch_bounds__(64) void bcq_lora_shrink_kernel(LoraArgs p)
{
    const int t = blockIdx.x, j = blockIdx.y, a = p.adapter[t];
    if (a < 0 || a >= p.desc.count || j >= adapter_rank(p, a)) return;
    const uint16_t *x = p.X + t * p.ldx, *row = p.A + ((long long)a * p.desc.max_rank + j) * p.desc.N;
    float sum = 0.0f;
    for (int n = threadIdx.x; n < p.desc.N; n += 64) sum = fmaf(to_float<BF>(x[n]), to_float<BF>(row[n]), sum);
    for (int step = 32; step > 0; step >>= 1) sum += __shfl_xor(sum, step);
    if (threadIdx.x == 0) static_cast<float *>(p.workspace)[(long long)t * p.desc.max_rank + j] = sum;
}

template <bool BF>
__global__ __launch_bounds__(256) void bcq_lora_expand_kernel(LoraArgs p)
{
    const int t = blockIdx.x, m = blockIdx.y * 256 + threadIdx.x, a = p.adapter[t];
    if (m >= p.desc.M) return;
    float y = to_float<BF>(p.base[t * p.ld_base + m]);
    if (a >= 0 && a < p.desc.count) {
        const float *v = static_cast<const float *>(p.workspace) + (long long)t * p.desc.max_rank;
        const uint16_t *row = p.B + ((long long)a * p.desc.M + m) * p.desc.max_rank;
        float sum = 0.0f;
        for (int j = 0; j < adapter_rank(p, a); ++j) sum = fmaf(to_float<BF>(row[j]), v[j], sum);
        y = fmaf(p.scale ? p.scale[a] : 1.0f, sum, y);
    }
    p.Y[t * p.ldy + m] = from_float<BF>(y);
}

size_t lora_workspace_bytes(const bcq_adapters &d, int tokens) { return (size_t)tokens * d.max_rank * sizeof(float); }

hipError_t launch_lora(const LoraArgs &a, hipStream_t stream)
{
    const dim3 shrink(a.tokens, a.desc.max_rank), expand(a.tokens, (a.desc.M + 255) / 256);
    if (a.desc.dtype == BCQ_BF16) {
        bcq_lora_shrink_kernel<true><<<shrink, 64, 0, stream>>>(a);
        bcq_lora_expand_kernel<true><<<expand, 256, 0, stream>>>(a);
    } else {
        bcq_lora_shrink_kernel<false><<<shrink, 64, 0, stream>>>(a);
        bcq_lora_expand_kernel<false><<<expand, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace bcq
