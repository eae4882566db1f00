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

// What both attentions check beside the shape.
static bcq_status attend_arguments(const bcq_cache *cache, const void *k_cache, const void *v_cache, int32_t tokens, int32_t requests, int32_t q_heads,
                                   const void *q, int64_t ld_q, const int32_t *q_start, const int32_t *kv_len, const int32_t *pages, int32_t max_new, float scale,
                                   int32_t causal, int32_t window, const void *out, int64_t ld_out)
{
    const int64_t cols = (int64_t)q_heads * cache->head_dim;
    if (!row_stride_ok(ld_q, cols) || !row_stride_ok(ld_out, cols) || max_new < 1) return BCQ_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || isinf(scale) || (causal != 0 && causal != 1) || window < 0 || (window > 0 && !causal)) return BCQ_ERR_INVALID_ARG;
    if (tokens == 0 || requests == 0) return BCQ_OK;
    if (!k_cache || !v_cache || !q || !q_start || !kv_len || !pages || !out) return BCQ_ERR_INVALID_ARG;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(q_start, 4) || !aligned(kv_len, 4) ||
        !aligned(pages, 4))
        return BCQ_ERR_INVALID_ARG;
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
    const bcq_status args = attend_arguments(cache, k_cache, v_cache, tokens, requests, q_heads, q, ld_q, q_start, kv_len, pages, max_new, scale, causal, window,
                                             out, ld_out);
    if (args != BCQ_OK) return args;
    if (tokens == 0 || requests == 0) return BCQ_OK;
    if (attend_workspace_bytes(*cache, tokens, requests, q_heads, max_new, max_pages) > 0 && (!workspace || !aligned(workspace, 16))) return BCQ_ERR_WORKSPACE;
    AttendArgs a{half(k_cache), half(v_cache), half(q), q_start, kv_len, pages, half(out), ld_q, ld_out, tokens, requests, q_heads, max_pages,
                 max_new, window, scale, causal != 0, workspace, *cache};
    return launch_attend(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

static bcq_status attend_shared_shape(const bcq_cache *cache, int32_t tokens, int32_t requests, int32_t groups, int32_t q_heads, int32_t max_pages)
{
    const bcq_status why = attend_shape(cache, tokens, requests, q_heads, max_pages, 1);
    if (why != BCQ_OK) return why;
    if (groups < 0) return BCQ_ERR_INVALID_ARG;
    if (groups > kMaxTokens) return BCQ_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)tokens * (q_heads / cache->kv_heads), row_lanes = cache->head_dim <= 64 ? 16 : cache->head_dim <= 128 ? 32 : 64;
    if ((rows * row_lanes + 256) * cache->kv_heads > 0xffffffffLL) return BCQ_ERR_UNSUPPORTED;  // threads of the join's launch, four elements of a row each
    const int64_t tiles = 2 * rows / 128 + groups + requests + 1;
    return tiles * (max_pages * (int64_t)cache->page_size / 32 + 1) > 0x7fffffffLL ? BCQ_ERR_UNSUPPORTED : BCQ_OK;  // blocks of keys of all tiles are int
}

size_t bcq_attend_shared_workspace_bytes(const bcq_cache *cache, int32_t tokens, int32_t requests, int32_t groups, int32_t q_heads, int32_t max_pages,
                                         int32_t max_new)
{
    if (attend_shared_shape(cache, tokens, requests, groups, q_heads, max_pages) != BCQ_OK || max_new < 1 || tokens == 0 || requests == 0) return 0;
    return attend_shared_workspace_bytes(*cache, tokens, requests, groups, q_heads, max_new);
}

bcq_status bcq_attend_shared(const bcq_cache *cache, const void *k_cache, const void *v_cache, int32_t tokens, int32_t requests, int32_t groups,
                             int32_t q_heads, const void *q, int64_t ld_q, const int32_t *q_start, const int32_t *kv_len, const int32_t *pages,
                             int32_t max_pages, int32_t max_new, const int32_t *group_start, const int32_t *shared_len, int32_t max_shared, float scale,
                             int32_t causal, int32_t window, void *out, int64_t ld_out, void *workspace, void *stream)
{
    bcq_status why = attend_shared_shape(cache, tokens, requests, groups, q_heads, max_pages);
    if (why != BCQ_OK) return why;
    why = attend_arguments(cache, k_cache, v_cache, tokens, requests, q_heads, q, ld_q, q_start, kv_len, pages, max_new, scale, causal, window, out, ld_out);
    if (why != BCQ_OK) return why;
    if (max_shared < 0) return BCQ_ERR_INVALID_ARG;
    if (tokens == 0 || requests == 0) return BCQ_OK;
    if (groups > 0 && (!group_start || !shared_len || !aligned(group_start, 4) || !aligned(shared_len, 4))) return BCQ_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 16)) return BCQ_ERR_WORKSPACE;
    AttendSharedArgs a{{half(k_cache), half(v_cache), half(q), q_start, kv_len, pages, half(out), ld_q, ld_out, tokens, requests, q_heads, max_pages,
                        max_new, window, scale, causal != 0, workspace, *cache},
                       group_start, shared_len, groups, max_shared};
    return launch_attend_shared(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
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

bcq_status bcq_plan(const bcq_page_table *table, int32_t *pages, const int32_t *held, const int32_t *fixed, int32_t *free_pages, const int32_t *free_count,
                    const int32_t *cached, const int32_t *fresh, int32_t tokens, int32_t *q_start, int32_t *kv_len, int32_t *lack, int32_t *held_out,
                    int32_t *free_count_out, int32_t *positions, int32_t *slots, int32_t *owner, void *stream)
{
    if (!table || table->page_size < 1 || table->num_pages < 1 || table->requests < 0 || table->max_pages < 1 || tokens < 0) return BCQ_ERR_INVALID_ARG;
    if (table->page_size > 65536 || (table->page_size & (table->page_size - 1)) || tokens > kMaxTokens || table->requests > kMaxTokens) return BCQ_ERR_UNSUPPORTED;
    if ((int64_t)table->num_pages * table->page_size > 0x7fffffffLL || (int64_t)table->max_pages * table->page_size > (1 << 30) ||
        (int64_t)table->requests * table->max_pages > 0x7fffffffLL)
        return BCQ_ERR_UNSUPPORTED;  // slots, keys of a request, and pages of all requests are int
    if (!free_pages || !free_count || !q_start || !free_count_out) return BCQ_ERR_INVALID_ARG;
    if (table->requests > 0 && (!pages || !held || !cached || !fresh || !kv_len || !lack || !held_out)) return BCQ_ERR_INVALID_ARG;
    if (tokens > 0 && (!positions || !slots || !owner)) return BCQ_ERR_INVALID_ARG;
    const struct { const int32_t *at; int64_t n; } read[] = {{fixed, table->requests}, {cached, table->requests}, {fresh, table->requests}, {held, table->requests}, {free_count, 1}},
        written[] = {{pages, (int64_t)table->requests * table->max_pages}, {free_pages, table->num_pages}, {q_start, (int64_t)table->requests + 1}, {kv_len, table->requests},
                     {lack, table->requests}, {positions, tokens}, {slots, tokens}, {owner, tokens}, {held_out, table->requests}, {free_count_out, 1}};
    constexpr int kRead = sizeof(read) / sizeof(*read), kWritten = sizeof(written) / sizeof(*written);
    const auto meet = [](auto &a, auto &b) { return a.at && b.at && a.n > 0 && b.n > 0 && (uintptr_t)a.at < (uintptr_t)(b.at + b.n) && (uintptr_t)b.at < (uintptr_t)(a.at + a.n); };
    for (int i = 0; i < kRead; ++i)
        if (!aligned(read[i].at, 4)) return BCQ_ERR_INVALID_ARG;
    for (int i = 0; i < kWritten; ++i) {
        if (!aligned(written[i].at, 4)) return BCQ_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (meet(written[i], written[j])) return BCQ_ERR_INVALID_ARG;
        for (int j = 0; j < kRead; ++j)  // (held and free_count may be the counts after the step)
            if (meet(written[i], read[j]) && !(j >= kRead - 2 && i - j == kWritten - kRead && written[i].at == read[j].at)) return BCQ_ERR_INVALID_ARG;
    }
    PlanArgs a{pages, held, fixed, free_pages, free_count, cached, fresh, q_start, kv_len, lack, held_out, free_count_out, positions, slots, owner,
               table->page_size, __builtin_ctz(table->page_size), table->num_pages, table->max_pages, table->requests, tokens};
    return launch_plan(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

bcq_status bcq_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits, int64_t ld, const float *temperature, const int32_t *top_k,
                      const float *top_p, const float *min_p, const float *uniform, int32_t *token, float *probability, void *stream)
{
    if (dtype != BCQ_F16 && dtype != BCQ_BF16) return BCQ_ERR_INVALID_ARG;
    if (rows < 0 || vocab < 1 || ld < vocab) return BCQ_ERR_INVALID_ARG;
    if (rows > kMaxTokens || vocab > BCQ_MAX_VOCAB) return BCQ_ERR_UNSUPPORTED;
    if (rows == 0) return BCQ_OK;
    if (!logits || !temperature || !uniform || !token) return BCQ_ERR_INVALID_ARG;
    if (!aligned(logits, 2) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(uniform, 4) ||
        !aligned(token, 4) || !aligned(probability, 4))
        return BCQ_ERR_INVALID_ARG;
    SampleArgs a{half(logits), ld, temperature, top_p, min_p, uniform, top_k, token, probability, rows, vocab, dtype == BCQ_BF16};
    return launch_sample(a, static_cast<hipStream_t>(stream)) == hipSuccess ? BCQ_OK : BCQ_ERR_HIP;
}

}  // extern "C"
