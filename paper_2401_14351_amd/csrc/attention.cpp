// Entry points of attention: argument checks, then the launchers of attention*.hip.
#include <algorithm>
#include <cmath>

#include "checks.hpp"
#include "common.hpp"
#include "hip_util.hpp"
#include "operators.hpp"

namespace sllm {

namespace {

constexpr uint64_t kMaxRows = 1ull << 30;  // tokens times heads, and a cache's slots
constexpr uint64_t kMaxDim = 128, kMaxHeads = 1ull << 16;
// A workgroup looks through the offsets for its piece; sequences times heads have one at least.
// With these a grid stays below 2^24 workgroups, its threads in 32 bits.
constexpr uint64_t kMaxSequences = 1ull << 16, kMaxListed = 1ull << 22;

// The extent of `t`: from its first element to its last.
int32_t heads_span(const char* name, const sllm_heads* t, Span* out) {
    if (!t) return fail(SLLM_E_INVAL, "%s: NULL", name);
    if (t->dtype != SLLM_DTYPE_F32 && t->dtype != SLLM_DTYPE_F16 && t->dtype != SLLM_DTYPE_BF16)
        return fail(SLLM_E_INVAL, "%s: dtype %u is not f32, f16 or bf16", name, t->dtype);
    if (t->reserved) return fail(SLLM_E_INVAL, "%s: reserved must be 0", name);
    if (t->dim > kMaxDim) return fail(SLLM_E_RANGE, "%s: heads of %llu elements, at most %llu", name, (unsigned long long)t->dim, (unsigned long long)kMaxDim);
    uint64_t rows;
    if (!mul_ok(t->tokens, t->heads, &rows) || rows > kMaxRows || t->heads > kMaxHeads || t->tokens > kMaxRows)
        return fail(SLLM_E_RANGE, "%s: %llu tokens of %llu heads, at most %llu heads and %llu together", name, (unsigned long long)t->tokens,
                    (unsigned long long)t->heads, (unsigned long long)kMaxHeads, (unsigned long long)kMaxRows);
    if (!rows || !t->dim) {
        *out = Span{name, static_cast<const uint8_t*>(t->data), 0};
        return SLLM_OK;
    }
    uint64_t heads_last = 0, tokens_last = 0, last = 0;
    if ((t->heads > 1 && !mul_ok(t->heads - 1, t->head_stride, &heads_last)) ||
        (t->tokens > 1 && !mul_ok(t->tokens - 1, t->token_stride, &tokens_last)) || !add_ok(heads_last, tokens_last, &last) ||
        !add_ok(last, t->dim, &last) || !mul_ok(last, itemsize(t->dtype), &last))
        return fail(SLLM_E_RANGE, "%s: size overflows", name);
    // a token's heads one behind the other and tokens behind those, or the other way round
    const bool tokens_out = (t->heads == 1 || t->head_stride >= t->dim) && (t->tokens == 1 || t->token_stride >= heads_last + t->dim);
    const bool heads_out = (t->tokens == 1 || t->token_stride >= t->dim) && (t->heads == 1 || t->head_stride >= tokens_last + t->dim);
    if (!tokens_out && !heads_out)
        return fail(SLLM_E_INVAL, "%s: rows of %llu elements overlap at strides of %llu and %llu", name, (unsigned long long)t->dim,
                    (unsigned long long)t->token_stride, (unsigned long long)t->head_stride);
    *out = Span{name, static_cast<const uint8_t*>(t->data), last};
    return check_pointer(*out, itemsize(t->dtype));
}

bool aligned(const sllm_heads& t) {
    const uint64_t size = itemsize(t.dtype);
    return reinterpret_cast<uintptr_t>(t.data) % 16 == 0 && t.dim * size % 16 == 0 && (t.tokens == 1 || t.token_stride * size % 16 == 0) &&
           (t.heads == 1 || t.head_stride * size % 16 == 0);
}

int32_t same_shape(const char* name, const sllm_heads& t, const sllm_heads& like, uint64_t heads) {
    if (t.tokens != like.tokens || t.heads != heads || t.dim != like.dim || t.dtype != like.dtype)
        return fail(SLLM_E_INVAL, "%s: %llu x %llu x %llu of dtype %u, not %llu x %llu x %llu of dtype %u", name, (unsigned long long)t.tokens,
                    (unsigned long long)t.heads, (unsigned long long)t.dim, t.dtype, (unsigned long long)like.tokens, (unsigned long long)heads,
                    (unsigned long long)like.dim, like.dtype);
    return SLLM_OK;
}

// What all calls have: q, k, v and the scale; their spans, from s on.
int32_t common_args(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, float scale, AttentionArgs* a, Span* s, int* n) {
    SLLM_TRY(heads_span("q", q, &s[(*n)++]));
    SLLM_TRY(heads_span("k", k, &s[(*n)++]));
    SLLM_TRY(heads_span("v", v, &s[(*n)++]));
    SLLM_TRY(same_shape("k", *k, *q, k->heads));
    SLLM_TRY(same_shape("v", *v, *q, k->heads));
    if (q->heads && (!k->heads || q->heads % k->heads))
        return fail(SLLM_E_INVAL, "%llu heads do not share %llu heads of keys", (unsigned long long)q->heads, (unsigned long long)k->heads);
    if (!q->heads && k->heads) return fail(SLLM_E_INVAL, "no heads for %llu heads of keys", (unsigned long long)k->heads);
    // (weights are powers of two: the kernels take it times log2 e, in 32 bits)
    if (!(scale > 0) || !std::isfinite(scale * 1.4426950408889634f))
        return fail(SLLM_E_INVAL, "scale %g is not a positive number up to 2.3e38", scale);
    a->q = q->data, a->q_token = q->token_stride, a->q_head = q->head_stride;
    a->k = k->data, a->k_token = k->token_stride, a->k_head = k->head_stride;
    a->v = v->data, a->v_token = v->token_stride, a->v_head = v->head_stride;
    a->tokens = (uint32_t)q->tokens, a->heads = (uint32_t)q->heads, a->kv_heads = (uint32_t)k->heads;
    a->group = k->heads ? (uint32_t)(q->heads / k->heads) : 0;
    a->dim = (uint32_t)q->dim, a->dtype = q->dtype;
    a->scale = scale;
    a->vec = aligned(*q) && aligned(*k) && aligned(*v);
    return SLLM_OK;
}

int32_t offsets_args(const sllm_ids* offsets, AttentionArgs* a, Span* s) {
    *s = Span{"offsets", nullptr, 0};
    a->sequences = 1;
    if (!offsets) return SLLM_OK;
    SLLM_TRY(ids_span(offsets, s));
    s->name = "offsets";
    if (!offsets->n) return fail(SLLM_E_INVAL, "offsets: none");
    if (offsets->n - 1 > kMaxSequences || (offsets->n - 1) * a->heads > kMaxListed)
        return fail(SLLM_E_RANGE, "%llu sequences of %u heads, at most %llu sequences and %llu together", (unsigned long long)(offsets->n - 1),
                    a->heads, (unsigned long long)kMaxSequences, (unsigned long long)kMaxListed);
    a->offsets = offsets->data, a->wide_offsets = offsets->bits == 64;
    a->sequences = (uint32_t)(offsets->n - 1);
    return SLLM_OK;
}

void window_args(uint64_t window, uint64_t sinks, AttentionArgs* a) {
    // no window, and one or sinks that reach behind every token, are the same as all tokens
    a->window = (int32_t)(window && window < kMaxRows ? window : kMaxRows);
    a->sinks = (int32_t)std::min<uint64_t>(sinks, a->tokens);
}

int32_t out_args(const char* name, const sllm_heads* out, const sllm_heads& q, AttentionArgs* a, Span* s) {
    SLLM_TRY(heads_span(name, out, s));
    SLLM_TRY(same_shape(name, *out, q, q.heads));
    a->out = out->data, a->out_token = out->token_stride, a->out_head = out->head_stride;
    a->vec = a->vec && aligned(*out);
    return SLLM_OK;
}

int32_t lse_span(const char* name, const float* lse, const AttentionArgs& a, Span* s) {
    *s = Span{name, reinterpret_cast<const uint8_t*>(lse), lse ? (uint64_t)a.tokens * a.heads * 4 : 0};
    return check_pointer(*s, 4);
}

int32_t cached_args(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, const sllm_kv_cache* cache, const sllm_ids* lengths,
                    const sllm_ids* offsets, float scale, AttentionArgs* a, Span* s, int* n) {
    SLLM_TRY(common_args(q, k, v, scale, a, s, n));
    SLLM_TRY(offsets_args(offsets, a, &s[*n]));
    ++*n;
    SLLM_TRY(ids_span(lengths, &s[*n]));
    s[(*n)++].name = "lengths";
    if (!cache) return fail(SLLM_E_INVAL, "cache: NULL");
    if (cache->reserved) return fail(SLLM_E_INVAL, "cache: reserved must be 0");
    if (cache->dtype != q->dtype || cache->heads != k->heads || cache->dim != k->dim)
        return fail(SLLM_E_INVAL, "cache: %llu heads of %llu elements of dtype %u, not %llu of %llu of dtype %u", (unsigned long long)cache->heads,
                    (unsigned long long)cache->dim, cache->dtype, (unsigned long long)k->heads, (unsigned long long)k->dim, q->dtype);
    if (!cache->window) return fail(SLLM_E_INVAL, "cache: a window of no tokens");
    if (cache->window > kMaxRows || cache->sinks > kMaxRows || cache->window + cache->sinks > kMaxRows)
        return fail(SLLM_E_RANGE, "cache: %llu sinks and a window of %llu, at most %llu together", (unsigned long long)cache->sinks,
                    (unsigned long long)cache->window, (unsigned long long)kMaxRows);
    if (lengths->n != cache->sequences)
        return fail(SLLM_E_INVAL, "%llu lengths for a cache of %llu sequences", (unsigned long long)lengths->n, (unsigned long long)cache->sequences);
    if (offsets ? offsets->n - 1 != cache->sequences : q->tokens != cache->sequences)
        return fail(SLLM_E_INVAL, "%llu %s for a cache of %llu sequences", (unsigned long long)(offsets ? offsets->n : q->tokens),
                    offsets ? "offsets" : "tokens, one each,", (unsigned long long)cache->sequences);
    if (!offsets && q->tokens * q->heads > kMaxListed)
        return fail(SLLM_E_RANGE, "%llu sequences of %llu heads, at most %llu together", (unsigned long long)q->tokens, (unsigned long long)q->heads,
                    (unsigned long long)kMaxListed);
    a->sequences = (uint32_t)cache->sequences;
    a->slots = cache->window + cache->sinks;
    uint64_t bytes = 0;
    if (!mul_ok(cache->sequences, cache->heads, &bytes) || !mul_ok(bytes, a->slots, &bytes) || !mul_ok(bytes, cache->dim * itemsize(cache->dtype), &bytes))
        return fail(SLLM_E_RANGE, "cache: size overflows");
    a->window = (int32_t)cache->window, a->sinks = (int32_t)cache->sinks;
    a->lengths = lengths->data, a->wide_lengths = lengths->bits == 64;
    a->cache_k = cache->k, a->cache_v = cache->v;
    s[*n] = Span{"cached keys", static_cast<const uint8_t*>(cache->k), bytes};
    SLLM_TRY(check_pointer(s[(*n)++], itemsize(cache->dtype)));
    s[*n] = Span{"cached values", static_cast<const uint8_t*>(cache->v), bytes};
    SLLM_TRY(check_pointer(s[(*n)++], itemsize(cache->dtype)));
    a->vec = a->vec && reinterpret_cast<uintptr_t>(cache->k) % 16 == 0 && reinterpret_cast<uintptr_t>(cache->v) % 16 == 0;
    return SLLM_OK;
}

}  // namespace

}  // namespace sllm

using namespace sllm;

extern "C" int32_t sllm_attention(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, const sllm_ids* offsets, uint64_t window,
                                  uint64_t sinks, float scale, const sllm_heads* out, float* lse, int32_t device, void* stream) try {
    clear_error();
    AttentionArgs a;
    Span s[6];
    int n = 2;
    SLLM_TRY(common_args(q, k, v, scale, &a, s, &n));
    SLLM_TRY(out_args("out", out, *q, &a, &s[0]));
    SLLM_TRY(lse_span("lse", lse, a, &s[1]));
    a.lse = lse;
    SLLM_TRY(offsets_args(offsets, &a, &s[n++]));
    window_args(window, sinks, &a);
    SLLM_TRY(check_overlaps(s, n, 2));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, 2, device));
    if (!a.tokens || !a.heads || !a.dim) return SLLM_OK;
    return launch_attention(a, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_attention_cached(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, const sllm_kv_cache* cache,
                                         const sllm_ids* lengths, const sllm_ids* offsets, float scale, const sllm_heads* out,
                                         void* workspace, uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    AttentionArgs a;
    Span s[9], parts[7];
    int n = 0;
    SLLM_TRY(cached_args(q, k, v, cache, lengths, offsets, scale, &a, parts, &n));
    SLLM_TRY(out_args("out", out, *q, &a, &s[0]));
    SLLM_TRY(workspace_span(workspace, workspace_bytes, a.offsets ? 0 : attention_step_workspace(a), &s[1]));
    // written: the output, the workspace and the cache, the last two of the parts
    s[2] = parts[5], s[3] = parts[6];
    for (int i = 0; i < 5; ++i) s[4 + i] = parts[i];
    SLLM_TRY(check_overlaps(s, 9, 4));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, 9, 4, device));
    if (!a.tokens || !a.heads || !a.dim) return SLLM_OK;
    if (a.offsets) return launch_attention(a, static_cast<hipStream_t>(stream));
    return launch_attention_step(a, workspace, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_attention_cached_workspace(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, const sllm_kv_cache* cache,
                                                   const sllm_ids* lengths, const sllm_ids* offsets, uint64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(SLLM_E_INVAL, "bytes: NULL");
    AttentionArgs a;
    Span s[7];
    int n = 0;
    SLLM_TRY(cached_args(q, k, v, cache, lengths, offsets, 1.0f, &a, s, &n));
    *bytes = a.offsets || !a.tokens ? 0 : attention_step_workspace(a);
    return SLLM_OK;
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_attention_grad(const sllm_heads* dout, const sllm_heads* q, const sllm_heads* k, const sllm_heads* v,
                                       const sllm_heads* out, const float* lse, const sllm_ids* offsets, uint64_t window, uint64_t sinks,
                                       float scale, const sllm_heads* dq, const sllm_heads* dk, const sllm_heads* dv, void* workspace,
                                       uint64_t workspace_bytes, int32_t device, void* stream) try {
    clear_error();
    AttentionGradArgs a;
    Span s[11];
    int n = 4;
    SLLM_TRY(common_args(q, k, v, scale, &a, s, &n));
    SLLM_TRY(out_args("out", out, *q, &a, &s[n++]));
    SLLM_TRY(heads_span("dout", dout, &s[n++]));
    SLLM_TRY(same_shape("dout", *dout, *q, q->heads));
    SLLM_TRY(heads_span("dq", dq, &s[0]));
    SLLM_TRY(same_shape("dq", *dq, *q, q->heads));
    SLLM_TRY(heads_span("dk", dk, &s[1]));
    SLLM_TRY(same_shape("dk", *dk, *k, k->heads));
    SLLM_TRY(heads_span("dv", dv, &s[2]));
    SLLM_TRY(same_shape("dv", *dv, *v, k->heads));
    if (!lse && a.tokens && a.heads) return fail(SLLM_E_INVAL, "lse: NULL");
    SLLM_TRY(lse_span("lse", lse, a, &s[n++]));
    SLLM_TRY(offsets_args(offsets, &a, &s[n++]));
    window_args(window, sinks, &a);
    SLLM_TRY(workspace_span(workspace, workspace_bytes, attention_grad_workspace(a), &s[3]));
    a.lse = const_cast<float*>(lse);
    a.dout = dout->data, a.dout_token = dout->token_stride, a.dout_head = dout->head_stride;
    a.dq = dq->data, a.dq_token = dq->token_stride, a.dq_head = dq->head_stride;
    a.dk = dk->data, a.dk_token = dk->token_stride, a.dk_head = dk->head_stride;
    a.dv = dv->data, a.dv_token = dv->token_stride, a.dv_head = dv->head_stride;
    a.vec = a.vec && aligned(*dout) && aligned(*dq) && aligned(*dk) && aligned(*dv);
    SLLM_TRY(check_overlaps(s, n, 4));
    DeviceGuard guard(device);
    if (!guard.ok()) return fail(SLLM_E_HIP, "cannot make device %d current", device);
    SLLM_TRY(check_spans(s, n, 4, device));
    if (!a.tokens || !a.heads || !a.dim) return SLLM_OK;
    return launch_attention_grad(a, workspace, static_cast<hipStream_t>(stream));
}
SLLM_CATCH_ALL

extern "C" int32_t sllm_attention_grad_workspace(const sllm_heads* q, const sllm_heads* k, const sllm_ids* offsets, uint64_t window,
                                                 uint64_t sinks, uint64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(SLLM_E_INVAL, "bytes: NULL");
    AttentionGradArgs a;
    Span s[4];
    int n = 0;
    SLLM_TRY(common_args(q, k, k, 1.0f, &a, s, &n));
    SLLM_TRY(offsets_args(offsets, &a, &s[n]));
    window_args(window, sinks, &a);
    *bytes = attention_grad_workspace(a);
    return SLLM_OK;
}
SLLM_CATCH_ALL
