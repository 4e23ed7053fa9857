// C ABI of the generator's operators: argument checks (on the host, before any launch) and launches.  See include/ralm.h.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/ralm.h"
#include "ralm_common.h"
#include "ralm_kernels.h"
#include "kv_kernels.h"

using namespace ralm;

namespace {

constexpr int64_t MAX_TOKENS = 1 << 22;      // new tokens or queries of a call: keeps every launch below 2^32 work-items
constexpr int64_t MAX_KV_REQUESTS = 1 << 16;
constexpr int64_t MAX_PAGES = 1 << 22;

#define KV_CHECK(call)                            \
    do {                                          \
        const ralm_status st_ = (call);           \
        if (st_ != RALM_OK) return st_;           \
    } while (0)
ralm_status launched(hipError_t e)
{
    return e == hipSuccess ? RALM_OK : set_error(RALM_ERR_DEVICE, "launch failed: %s", hipGetErrorString(e));
}
bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int elem_bytes(int dt) { return dt == RALM_F32 ? 4 : 2; }

bool shape_ok(int32_t n_layers, int32_t n_heads, int32_t d, int32_t page_tokens)
{
    return n_layers >= 1 && n_layers <= 1024 && n_heads >= 1 && n_heads <= 1024 && (d == 64 || d == 128 || d == 256) && page_tokens >= 16 &&
           page_tokens <= 256 && (page_tokens & (page_tokens - 1)) == 0;
}

ralm_status check_cache(const ralm_kv_t *kv, bool refs)
{
    if (!kv) return set_error(RALM_ERR_NULL, "cache descriptor is NULL");
    if (!kv->pages || !kv->table || !kv->lens || (refs && !kv->refs)) return set_error(RALM_ERR_NULL, "cache.pages/table/lens%s is NULL", refs ? "/refs" : "");
    if (!shape_ok(kv->n_layers, kv->n_heads, kv->d, kv->page_tokens))
        return set_error(RALM_ERR_SHAPE, "cache: n_layers and n_heads in [1, 1024], d 64, 128 or 256, page_tokens a power of two in [16, 256]");
    if (kv->n_pages < 1 || kv->n_pages > MAX_PAGES) return set_error(RALM_ERR_SHAPE, "n_pages=%lld out of [1, 2^22]", (long long)kv->n_pages);
    if (kv->R < 1 || kv->R > MAX_KV_REQUESTS || kv->max_pages < 1 || (int64_t)kv->max_pages * kv->page_tokens > (1 << 30) ||
        kv->R * kv->max_pages > 0x7fffffffLL)
        return set_error(RALM_ERR_SHAPE, "R=%lld, max_pages=%d: at most 2^16 requests, 2^30 tokens each and 2^31 - 1 places of the table",
                         (long long)kv->R, kv->max_pages);
    if (!aligned(kv->pages, 16)) return set_error(RALM_ERR_ALIGN, "cache.pages must be 16-byte aligned");
    return RALM_OK;
}

KvView view_of(const ralm_kv_t *kv, int32_t layer)
{
    KvView v;
    v.pages = static_cast<uint8_t *>(kv->pages);
    v.head_bytes = (int64_t)kv->page_tokens / KV_TILE * kv_tile_bytes(kv->d);
    v.layer_bytes = v.head_bytes * kv->n_heads * layer;
    v.page_bytes = v.head_bytes * kv->n_heads * kv->n_layers;
    v.n_pages = (int32_t)kv->n_pages;
    v.n_heads = kv->n_heads;
    v.d = kv->d;
    v.tile_shift = __builtin_ctz(kv->page_tokens / KV_TILE);
    v.table = kv->table;
    v.lens = kv->lens;
    v.R = (int32_t)kv->R;
    v.max_pages = kv->max_pages;
    return v;
}
KvPages pages_of(const ralm_kv_t *kv)
{
    KvPages p;
    p.pages = static_cast<uint8_t *>(kv->pages);
    p.page_bytes = (int64_t)ralm_kv_page_bytes(kv->n_layers, kv->n_heads, kv->d, kv->page_tokens);
    p.n_pages = (int32_t)kv->n_pages;
    p.page_tokens = kv->page_tokens;
    p.max_pages = kv->max_pages;
    p.R = (int32_t)kv->R;
    p.table = kv->table;
    p.lens = kv->lens;
    p.refs = kv->refs;
    return p;
}

ralm_status check_rows(const ralm_kv_t *kv, int32_t layer, const void *k, const void *v, int32_t dtype, int64_t strides[4], const int64_t *offsets,
                       int64_t n)
{
    KV_CHECK(check_cache(kv, false));
    if (layer < 0 || layer >= kv->n_layers) return set_error(RALM_ERR_RANGE, "layer=%d out of [0, %d)", layer, kv->n_layers);
    if (n < 0 || n > MAX_TOKENS) return set_error(RALM_ERR_RANGE, "n=%lld out of [0, 2^22]", (long long)n);
    if (dtype != RALM_F32 && dtype != RALM_BF16 && dtype != RALM_F16) return set_error(RALM_ERR_DTYPE, "dtype unknown");
    if (n == 0) return RALM_OK;
    if (!k || !v || !offsets) return set_error(RALM_ERR_NULL, "k/v/offsets is NULL");
    if (!aligned(k, 16) || !aligned(v, 16)) return set_error(RALM_ERR_ALIGN, "k and v must be 16-byte aligned");
    for (int i = 0; i < 4; i += 2) {
        if (strides[i + 1] == 0) strides[i + 1] = kv->d;
        if (strides[i] == 0) strides[i] = strides[i + 1] * kv->n_heads;
    }
    for (int i = 0; i < 4; ++i)
        if (strides[i] < kv->d || strides[i] * elem_bytes(dtype) % 16) return set_error(RALM_ERR_ALIGN, "strides of k and v must be at least d and multiples of 16 bytes");
    return RALM_OK;
}

ralm_status rows(bool append, const ralm_kv_t *kv, int32_t layer, const void *k, const void *v, int32_t dtype, int64_t k_token, int64_t k_head,
                 int64_t v_token, int64_t v_head, const int64_t *offsets, int64_t n, const int32_t *start, void *stream)
{
    int64_t st[4] = {k_token, k_head, v_token, v_head};
    KV_CHECK(check_rows(kv, layer, k, v, dtype, st, offsets, n));
    if (n == 0) return RALM_OK;
    KvRows r;
    r.k = const_cast<void *>(k);
    r.v = const_cast<void *>(v);
    r.dtype = dtype;
    r.k_token = st[0], r.k_head = st[1], r.v_token = st[2], r.v_head = st[3];
    r.offsets = offsets;
    r.n = n;
    r.start = start;
    const KvView view = view_of(kv, layer);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(append ? launch_kv_append(view, r, s) : launch_kv_read(view, r, s));
}

// plan and workspace of an attention call
ralm_status plan_of(const ralm_kv_t *kv, int32_t n_q_heads, int64_t Qt, int64_t max_q, int64_t max_len, int32_t window, int32_t sinks,
                    KvAttentionPlan &plan, size_t &out_bytes, size_t &bytes)
{
    KV_CHECK(check_cache(kv, false));
    if (n_q_heads < kv->n_heads || n_q_heads % kv->n_heads || n_q_heads > 4096)
        return set_error(RALM_ERR_SHAPE, "n_q_heads=%d must be a multiple of n_heads=%d of at most 4096", n_q_heads, kv->n_heads);
    if (Qt < 0 || Qt > MAX_TOKENS) return set_error(RALM_ERR_RANGE, "Qt=%lld out of [0, 2^22]", (long long)Qt);
    if (Qt * n_q_heads > (1 << 30)) return set_error(RALM_ERR_SHAPE, "Qt x n_q_heads beyond 2^30; split the batch");
    if (max_q < 0 || max_len < 0 || window < 0 || sinks < 0) return set_error(RALM_ERR_RANGE, "max_q, max_len, window and sinks must not be negative");
    const int64_t room = (int64_t)kv->max_pages * kv->page_tokens;
    if (max_q > Qt) max_q = 0;   // says nothing
    if (max_len == 0 || max_len > room) max_len = room;
    if (window > room) window = 0;
    if (kv->R * kv->n_heads > KV_MAX_PAIRS) return set_error(RALM_ERR_SHAPE, "R x n_heads beyond %lld; split the batch", (long long)KV_MAX_PAIRS);
    plan = kv_attention_plan(kv->R, kv->n_heads, n_q_heads / kv->n_heads, kv->d, Qt, max_q, max_len, window, sinks);
    out_bytes = plan.parts > 1 ? (size_t)plan.parts * Qt * n_q_heads * kv->d * 4 : 0;
    bytes = plan.parts > 1 ? out_bytes + (size_t)plan.parts * Qt * n_q_heads * 8 : 256;
    return RALM_OK;
}

ralm_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (!ws || !aligned(ws, 16)) return set_error(RALM_ERR_WORKSPACE, "workspace is NULL or not 16-byte aligned");
    if (have < need) return set_error(RALM_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", have, need);
    return RALM_OK;
}

}  // namespace

extern "C" {

size_t ralm_kv_page_bytes(int32_t n_layers, int32_t n_heads, int32_t d, int32_t page_tokens)
{
    if (!shape_ok(n_layers, n_heads, d, page_tokens)) return 0;
    return (size_t)n_layers * n_heads * (page_tokens / KV_TILE) * kv_tile_bytes(d);
}

ralm_status ralm_kv_append(const ralm_kv_t *kv, int32_t layer, const void *k, const void *v, int32_t dtype, int64_t k_token_stride,
                           int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, const int64_t *offsets, int64_t n, void *stream)
{
    return rows(true, kv, layer, k, v, dtype, k_token_stride, k_head_stride, v_token_stride, v_head_stride, offsets, n, nullptr, stream);
}

ralm_status ralm_kv_read(const ralm_kv_t *kv, int32_t layer, const int64_t *offsets, int64_t n, const int32_t *start, void *k, void *v, int32_t dtype,
                         int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride, void *stream)
{
    return rows(false, kv, layer, k, v, dtype, k_token_stride, k_head_stride, v_token_stride, v_head_stride, offsets, n, start, stream);
}

size_t ralm_kv_attention_workspace_bytes(const ralm_kv_t *kv, int32_t n_q_heads, int64_t Qt, int64_t max_q, int64_t max_len, int32_t window,
                                         int32_t sinks)
{
    KvAttentionPlan plan;
    size_t out_bytes, bytes;
    return plan_of(kv, n_q_heads, Qt, max_q, max_len, window, sinks, plan, out_bytes, bytes) == RALM_OK ? bytes : 0;
}

ralm_status ralm_kv_attention(const ralm_kv_t *kv, int32_t layer, const void *q, int32_t dtype, int64_t q_token_stride, int64_t q_head_stride,
                              int32_t n_q_heads, const int64_t *offsets, int64_t Qt, int64_t max_q, int64_t max_len, float scale, int32_t window,
                              int32_t sinks, void *out, int64_t out_token_stride, int64_t out_head_stride, float *lse, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    KvAttentionPlan plan;
    size_t out_bytes, bytes;
    KV_CHECK(plan_of(kv, n_q_heads, Qt, max_q, max_len, window, sinks, plan, out_bytes, bytes));
    if (layer < 0 || layer >= kv->n_layers) return set_error(RALM_ERR_RANGE, "layer=%d out of [0, %d)", layer, kv->n_layers);
    if (dtype != RALM_BF16 && dtype != RALM_F16) return set_error(RALM_ERR_DTYPE, "dtype must be RALM_BF16 or RALM_F16");
    if (!(scale > 0.0f) || !isfinite(scale)) return set_error(RALM_ERR_RANGE, "scale must be positive and finite");
    if (Qt == 0) return RALM_OK;
    if (!q || !out || !offsets) return set_error(RALM_ERR_NULL, "q/out/offsets is NULL");
    int64_t st[4] = {q_token_stride, q_head_stride, out_token_stride, out_head_stride};
    for (int i = 0; i < 4; i += 2) {
        if (st[i + 1] == 0) st[i + 1] = kv->d;
        if (st[i] == 0) st[i] = st[i + 1] * n_q_heads;
    }
    for (int i = 0; i < 4; ++i)
        if (st[i] < kv->d || st[i] % 8) return set_error(RALM_ERR_ALIGN, "strides of q and out must be at least d and multiples of 8 elements");
    if (!aligned(q, 16) || !aligned(out, 16)) return set_error(RALM_ERR_ALIGN, "q and out must be 16-byte aligned");
    if (plan.parts > 1) KV_CHECK(check_workspace(workspace, workspace_bytes, bytes));
    KvAttention a;
    a.q = q;
    a.dtype = dtype;
    a.q_token = st[0], a.q_head = st[1];
    a.out = out;
    a.out_token = st[2], a.out_head = st[3];
    a.lse = lse;
    a.offsets = offsets;
    a.Qt = Qt;
    a.group = n_q_heads / kv->n_heads;
    a.scale = scale * 1.4426950408889634f;
    // a window that reaches beyond every place of the table hides nothing
    a.window = (int64_t)window > (int64_t)kv->max_pages * kv->page_tokens ? 0 : window;
    a.sinks = sinks > (1 << 30) ? 1 << 30 : sinks;
    a.row_tiles = plan.row_tiles;
    a.parts = plan.parts;
    a.part_tiles = plan.part_tiles;
    a.max_rows = plan.max_rows;
    a.by_length = plan.by_length;
    a.part_out = static_cast<float *>(workspace);
    a.part_stat = plan.parts > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + out_bytes) : nullptr;
    return launched(launch_kv_attention(view_of(kv, layer), a, plan, static_cast<hipStream_t>(stream)));
}

size_t ralm_kv_pages_workspace_bytes(const ralm_kv_t *kv)
{
    if (check_cache(kv, false) != RALM_OK) return 0;
    return kv_pages_scratch_words(kv->n_pages, kv->R) * 4;
}

ralm_status ralm_kv_reserve(const ralm_kv_t *kv, const int32_t *grow, int32_t *granted, void *workspace, size_t workspace_bytes, void *stream)
{
    KV_CHECK(check_cache(kv, true));
    if (!grow) return set_error(RALM_ERR_NULL, "grow is NULL");
    KV_CHECK(check_workspace(workspace, workspace_bytes, ralm_kv_pages_workspace_bytes(kv)));
    return launched(launch_kv_reserve(pages_of(kv), grow, granted, static_cast<int32_t *>(workspace), static_cast<hipStream_t>(stream)));
}

ralm_status ralm_kv_fork(const ralm_kv_t *kv, const int32_t *src, const int32_t *dst, const int32_t *keep, int64_t n, void *stream)
{
    KV_CHECK(check_cache(kv, true));
    if (n < 0 || n > MAX_TOKENS) return set_error(RALM_ERR_RANGE, "n=%lld out of [0, 2^22]", (long long)n);
    if (n == 0) return RALM_OK;
    if (!src || !dst) return set_error(RALM_ERR_NULL, "src/dst is NULL");
    return launched(launch_kv_fork(pages_of(kv), src, dst, keep, n, static_cast<hipStream_t>(stream)));
}

ralm_status ralm_kv_truncate(const ralm_kv_t *kv, const int32_t *new_lens, void *stream)
{
    KV_CHECK(check_cache(kv, true));
    if (!new_lens) return set_error(RALM_ERR_NULL, "new_lens is NULL");
    return launched(launch_kv_truncate(pages_of(kv), new_lens, static_cast<hipStream_t>(stream)));
}

ralm_status ralm_kv_copy_pages(const ralm_kv_t *kv, const int32_t *src, const int32_t *dst, int64_t n, void *stream)
{
    KV_CHECK(check_cache(kv, false));
    if (n < 0 || n > MAX_PAGES) return set_error(RALM_ERR_RANGE, "n=%lld out of [0, 2^22]", (long long)n);
    if (n == 0) return RALM_OK;
    if (!src || !dst) return set_error(RALM_ERR_NULL, "src/dst is NULL");
    return launched(launch_kv_copy_pages(pages_of(kv), src, dst, n, static_cast<hipStream_t>(stream)));
}

ralm_status ralm_kv_compact(const ralm_kv_t *kv, int32_t *table_out, int32_t *refs_out, int32_t *used, void *workspace, size_t workspace_bytes,
                            void *stream)
{
    KV_CHECK(check_cache(kv, true));
    if (!table_out || !refs_out || !used) return set_error(RALM_ERR_NULL, "table_out/refs_out/used is NULL");
    KV_CHECK(check_workspace(workspace, workspace_bytes, ralm_kv_pages_workspace_bytes(kv)));
    return launched(launch_kv_compact(pages_of(kv), table_out, refs_out, used, static_cast<int32_t *>(workspace), static_cast<hipStream_t>(stream)));
}

size_t ralm_verify_draft_workspace_bytes(int64_t R, int32_t V)
{
    if (R < 1 || R > MAX_KV_REQUESTS || V < 1 || V > RALM_MAX_VOCABULARY) return 0;
    return (size_t)R * draft_chunks(V) * 8;
}

ralm_status ralm_verify_draft(const int32_t *draft_ids, const void *draft_probs, int64_t draft_stride, const void *target_probs, int64_t target_stride,
                              int32_t dtype, int32_t V, const float *u, const float *u_next, int64_t Qt, const int64_t *q_offsets, int64_t R,
                              int32_t *accepted, int32_t *next_token, void *workspace, size_t workspace_bytes, void *stream)
{
    if (R < 1 || R > MAX_KV_REQUESTS) return set_error(RALM_ERR_SHAPE, "R=%lld out of [1, 2^16]", (long long)R);
    if (V < 1 || V > RALM_MAX_VOCABULARY) return set_error(RALM_ERR_SHAPE, "V=%d out of [1, %d]", V, RALM_MAX_VOCABULARY);
    if (Qt < 0 || Qt > MAX_TOKENS) return set_error(RALM_ERR_RANGE, "Qt=%lld out of [0, 2^22]", (long long)Qt);
    if (dtype != RALM_F32 && dtype != RALM_BF16 && dtype != RALM_F16) return set_error(RALM_ERR_DTYPE, "dtype unknown");
    if (!target_probs || !u_next || !q_offsets || !accepted || !next_token || (Qt > 0 && (!draft_ids || !u)))
        return set_error(RALM_ERR_NULL, "a pointer is NULL");
    if (target_stride == 0) target_stride = V;
    if (draft_stride == 0) draft_stride = V;
    if (target_stride < V || draft_stride < V) return set_error(RALM_ERR_SHAPE, "target_stride or draft_stride < V");
    const size_t es = elem_bytes(dtype);
    if (!aligned(target_probs, es) || !aligned(draft_probs, es)) return set_error(RALM_ERR_ALIGN, "probabilities must be aligned to their type");
    KV_CHECK(check_workspace(workspace, workspace_bytes, ralm_verify_draft_workspace_bytes(R, V)));
    DraftParams p;
    p.draft_ids = draft_ids;
    p.draft_probs = draft_probs;
    p.target_probs = target_probs;
    p.draft_stride = draft_stride, p.target_stride = target_stride;
    p.dtype = dtype;
    p.V = V;
    p.u = u, p.u_next = u_next;
    p.offsets = q_offsets;
    p.Qt = Qt, p.R = R;
    p.accepted = accepted, p.next = next_token;
    p.sums = static_cast<u64 *>(workspace);
    p.chunks = draft_chunks(V);
    return launched(launch_verify_draft(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
