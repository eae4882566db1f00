// extern "C" entry points of the serving operators: argument checks (host only, before any launch) and dispatch.
#include <math.h>

#include "bcq_internal.h"

using namespace bcq;

namespace {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A row stride: at least a row, whole 16-byte pieces.
inline bool row_stride_ok(int64_t ld, int64_t cols) { return ld >= cols && ld % 8 == 0; }

bool cache_ok(const bcq_cache *c, bcq_status *why)
{
    *why = BCQ_ERR_INVALID_ARG;
    if (!c || (c->dtype != BCQ_F16 && c->dtype != BCQ_BF16)) return false;
    if (c->kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 || c->num_pages < 1) return false;
    if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0) return false;
    if (c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8) return false;
    if (c->page_size > 1 && c->slot_stride < c->head_dim) return false;
    *why = BCQ_ERR_UNSUPPORTED;
    if (c->head_dim % 8 || c->head_dim > BCQ_MAX_HEAD_DIM) return false;
    if (c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return false;
    if (c->slot_stride > (1 << 30) || c->page_size * c->slot_stride >= (1 << 30)) return false;
    if ((int64_t)c->num_pages * c->page_size > 0x7fffffffLL) return false;  // slots are int32
    *why = BCQ_OK;
    return true;
}

bool adapters_ok(const bcq_adapters *d, bcq_status *why)
{
    *why = BCQ_ERR_INVALID_ARG;
    if (!d || (d->dtype != BCQ_F16 && d->dtype != BCQ_BF16)) return false;
    if (d->count < 1 || d->max_rank < 1 || d->M < 1 || d->N < 1 || d->N % 8 || d->max_rank % 8) return false;
    *why = BCQ_ERR_UNSUPPORTED;
    if (d->max_rank > BCQ_MAX_RANK || d->M > (1 << 23) || d->N > (1 << 23)) return false;
    *why = BCQ_OK;
    return true;
}

// Tokens and requests of one call (int arithmetic over tokens times heads stays in range).
constexpr int32_t kMaxTokens = 1 << 20;

inline const uint16_t *half(const void *p) { return static_cast<const uint16_t *>(p); }
inline uint16_t *half(void *p) { return static_cast<uint16_t *>(p); }

}  // namespace

extern "C" {

bcq_status bcq_rotate(const bcq_cache *cache, int32_t tokens, int32_t q_heads, const void *qkv, int64_t ld_qkv,
                      const int32_t *positions, const float *cos_sin, int32_t max_position, int32_t rot_dim,
                      int32_t interleaved, const void *q_weight, const void *k_weight, float eps, void *q_out, int64_t ld_q,
                      const int32_t *slots, void *k_cache, void *v_cache, void *stream)
{
    bcq_status why;
    if (!cache_ok(cache, &why)) return why;
    const int64_t D = cache->head_dim;
    if (tokens < 0 || q_heads < 1 || rot_dim < 0 || rot_dim % 2 || rot_dim > D || max_position < 1) return BCQ_ERR_INVALID_ARG;
    if ((interleaved != 0 && interleaved != 1) || !(eps >= 0.0f) || isinf(eps)) return BCQ_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || q_heads > 1024 || cache->kv_heads > 1024) return BCQ_ERR_UNSUPPORTED;
    if (!row_stride_ok(ld_qkv, (q_heads + 2 * (int64_t)cache->kv_heads) * D) || !row_stride_ok(ld_q, q_heads * D)) return BCQ_ERR_INVALID_ARG;
    if (tokens == 0) return BCQ_OK;
    if (!qkv || !positions || !q_out || !slots || !k_cache || !v_cache || (rot_dim > 0) != (cos_sin != nullptr)) return BCQ_ERR_INVALID_ARG;
    if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(q_weight, 16) ||
        !aligned(k_weight, 16) || !aligned(cos_sin, 4) || !aligned(positions, 4) || !aligned(slots, 4))
        return BCQ_ERR_INVALID_ARG;
    if (q_out == qkv && tokens > 1 && ld_q != ld_qkv) return BCQ_ERR_INVALID_ARG;  // (a lone row has no next one)
    RotateArgs a{half(qkv), half(q_weight), half(k_weight), positions, slots, cos_sin, half(q_out), half(k_cache), half(v_cache),
                 ld_qkv, ld_q, tokens, q_heads, rot_dim, max_position, eps, interleaved != 0, *cache};
    return launch_rotate(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

static bcq_status attend_shape(const bcq_cache *cache, int32_t tokens, int32_t requests, int32_t q_heads, int32_t max_pages, int32_t max_new)
{
    bcq_status why;
    if (!cache_ok(cache, &why)) return why;
    if (tokens < 0 || requests < 0 || q_heads < 1 || q_heads % cache->kv_heads || max_pages < 1 || max_new < 1) return BCQ_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || requests > kMaxTokens || q_heads > 1024) return BCQ_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * cache->page_size > (1 << 30) || (int64_t)requests * (max_pages * (int64_t)cache->page_size / 32 + 1) > 0x7fffffffLL)
        return BCQ_ERR_UNSUPPORTED;  // keys of a request, and blocks of keys of all requests, are int
    return BCQ_OK;
}

size_t bcq_attend_workspace_bytes(const bcq_cache *cache, int32_t tokens, int32_t requests, int32_t q_heads, int32_t max_pages,
                                  int32_t max_new)
{
    if (attend_shape(cache, tokens, requests, q_heads, max_pages, max_new) != BCQ_OK || tokens == 0 || requests == 0) return 0;
    return attend_workspace_bytes(*cache, tokens, requests, q_heads, max_new, max_pages);
}

bcq_status bcq_attend(const bcq_cache *cache, const void *k_cache, const void *v_cache, int32_t tokens, int32_t requests,
                      int32_t q_heads, const void *q, int64_t ld_q, const int32_t *q_start, const int32_t *kv_len,
                      const int32_t *pages, int32_t max_pages, int32_t max_new, float scale, int32_t causal, int32_t window,
                      void *out, int64_t ld_out, void *workspace, void *stream)
{
    const bcq_status why = attend_shape(cache, tokens, requests, q_heads, max_pages, max_new);
    if (why != BCQ_OK) return why;
    const int64_t cols = (int64_t)q_heads * cache->head_dim;
    if (!row_stride_ok(ld_q, cols) || !row_stride_ok(ld_out, cols) ) return BCQ_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || isinf(scale) || (causal != 0 && causal != 1) || window < 0 || (window > 0 && !causal)) return BCQ_ERR_INVALID_ARG;
    if (tokens == 0 || requests == 0) return BCQ_OK;
    if (!k_cache || !v_cache || !q || !q_start || !kv_len || !pages || !out) return BCQ_ERR_INVALID_ARG;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(q_start, 4) || !aligned(kv_len, 4) ||
        !aligned(pages, 4))
        return BCQ_ERR_INVALID_ARG;
    if (attend_workspace_bytes(*cache, tokens, requests, q_heads, max_new, max_pages) > 0 && (!workspace || !aligned(workspace, 16))) return BCQ_ERR_WORKSPACE;
    AttendArgs a{half(k_cache), half(v_cache), half(q), q_start, kv_len, pages, half(out), ld_q, ld_out, tokens, requests, q_heads, max_pages,
                 max_new, window, scale, causal != 0, workspace, *cache};
    return launch_attend(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

size_t bcq_lora_workspace_bytes(const bcq_adapters *desc, int32_t tokens)
{
    bcq_status why;
    if (!adapters_ok(desc, &why) || tokens < 1 || tokens > kMaxTokens) return 0;
    return lora_workspace_bytes(*desc, tokens);
}

bcq_status bcq_lora(const bcq_adapters *desc, const void *A, const void *B, const int32_t *rank, const float *scale,
                    int32_t tokens, const int32_t *adapter, const void *X, int64_t ldx, const void *base, int64_t ld_base,
                    void *Y, int64_t ldy, void *workspace, void *stream)
{
    bcq_status why;
    if (!adapters_ok(desc, &why)) return why;
    if (tokens < 0 || !row_stride_ok(ldx, desc->N) || ld_base < desc->M || ldy < desc->M) return BCQ_ERR_INVALID_ARG;
    if (tokens > kMaxTokens) return BCQ_ERR_UNSUPPORTED;
    if (tokens == 0) return BCQ_OK;
    if (!A || !B || !adapter || !X || !base || !Y) return BCQ_ERR_INVALID_ARG;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(X, 16) || !aligned(base, 2) || !aligned(Y, 2) || !aligned(rank, 4) || !aligned(scale, 4) ||
        !aligned(adapter, 4))
        return BCQ_ERR_INVALID_ARG;
    if (Y == base && tokens > 1 && ldy != ld_base) return BCQ_ERR_INVALID_ARG;
    if (lora_workspace_bytes(*desc, tokens) > 0 && (!workspace || !aligned(workspace, 16))) return BCQ_ERR_WORKSPACE;
    LoraArgs a{half(A), half(B), half(X), half(base), rank, adapter, scale, half(Y), ldx, ld_base, ldy, tokens, workspace, *desc};
    return launch_lora(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

}  // extern "C"
