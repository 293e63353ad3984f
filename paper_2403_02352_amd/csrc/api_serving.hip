// C ABI of the serving path: argument checks and launches.  Nothing here allocates or synchronises.
#include "api_common.h"
#include "serving.h"

using namespace atp;

namespace {

constexpr int64_t MAX_SEQ = 65536;   // (every workgroup counts the sequences up)

// what the checks of a cache and a batch leave in the arguments of a kernel
atp_status take_cache(const atp_cache* c, const atp_batch* b, const atp_dtype& t, ServeArgs& a, bool pointers) {
    if (!c || !b || bad_dtype(t)) return ATP_ERR_INVALID_ARG;
    const int type = raw_enum(c->type);
    if (type != ATP_CACHE_SAME && type != ATP_CACHE_E4M3) return ATP_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->n_pages > 0x7fffffff || c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) || c->kv_heads < 1 || c->d_h < 1)
        return ATP_ERR_INVALID_ARG;
    if (b->n_seq < 1 || b->n_seq > MAX_SEQ || b->max_pages < 1 || b->tokens < 0 || b->tokens > 0x7fffffff) return ATP_ERR_INVALID_ARG;
    if (c->d_h % 8 || c->d_h > 256 || c->kv_heads > 65535) return ATP_ERR_UNSUPPORTED;
    if (b->max_pages > (1 << 30) / c->page_size || b->tokens > 0x7fffffff / c->kv_heads) return ATP_ERR_UNSUPPORTED;
    if (pointers) {
        if (!c->K || !c->V || !b->table || !b->length || !b->offsets) return ATP_ERR_INVALID_ARG;
        if ((type == ATP_CACHE_E4M3) != (c->K_scale != nullptr) || (type == ATP_CACHE_E4M3) != (c->V_scale != nullptr)) return ATP_ERR_INVALID_ARG;
        if (!aligned16(c->K) || !aligned16(c->V) || !aligned16(c->K_scale) || !aligned16(c->V_scale)) return ATP_ERR_INVALID_ARG;
        if (((uintptr_t)b->table & 3) || ((uintptr_t)b->length & 3) || ((uintptr_t)b->offsets & 3)) return ATP_ERR_INVALID_ARG;
    }
    a.offsets = b->offsets; a.length = b->length; a.table = b->table;
    a.n_seq = (int)b->n_seq; a.tokens = (int)b->tokens;
    a.max_pages = b->max_pages; a.n_pages = c->n_pages;
    a.page_shift = __builtin_ctz((unsigned)c->page_size);
    a.max_kv = (int)(b->max_pages * c->page_size);
    a.kv_heads = c->kv_heads; a.dh = c->d_h;
    a.K = c->K; a.V = c->V; a.Ks = c->K_scale; a.Vs = c->V_scale;
    return ATP_OK;
}

// a packed tensor: rows of `row` elements, `ld` apart
bool bad_rows(const void* p, int64_t ld, int64_t row, atp_dtype t) {
    return !p || !aligned16(p) || ld < row || ld > (1 << 24) || (ld * (int64_t)esize(t)) % 16;
}

KvSource source_of(const atp_cache* c) { return raw_enum(c->type) == ATP_CACHE_E4M3 ? KV_PAGED_E4M3 : KV_PAGED; }

// keys and values of the new tokens, as the cache holds them and as the packed tensors do
double moved_bytes(const atp_cache* c, const atp_batch* b, atp_dtype t) {
    const double cached = raw_enum(c->type) == ATP_CACHE_E4M3 ? c->d_h + 1.0 : (double)c->d_h * esize(t);
    return 2.0 * b->tokens * c->kv_heads * (cached + (double)c->d_h * esize(t));
}

atp_status packed_shape(int64_t n_seq, int64_t tokens, int heads, int kv_heads, int d_h, const atp_dtype& t, ServeArgs& a) {
    if (bad_dtype(t) || n_seq < 1 || n_seq > MAX_SEQ || tokens < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || d_h < 1) return ATP_ERR_INVALID_ARG;
    if (d_h % 8 || d_h > 256 || kv_heads > 65535 || tokens > 0x7fffffff / heads) return ATP_ERR_UNSUPPORTED;
    a.n_seq = (int)n_seq; a.tokens = (int)tokens; a.heads = heads; a.kv_heads = kv_heads; a.dh = d_h;
    a.max_kv = (int)tokens;
    return ATP_OK;
}

}  // namespace

extern "C" {

atp_status atp_cache_write(const atp_cache* cache, const atp_batch* batch, const void* K, const void* V, int64_t ldk, int64_t ldv,
                           atp_dtype t, void* hip_stream) {
    ServeArgs a;
    const atp_status s = take_cache(cache, batch, t, a, true);
    if (s != ATP_OK) return s;
    if (!a.tokens) return ATP_OK;
    const int64_t row = (int64_t)a.kv_heads * a.dh;
    if (bad_rows(K, ldk, row, t) || bad_rows(V, ldv, row, t)) return ATP_ERR_INVALID_ARG;
    a.Kn = K; a.Vn = V; a.ldk = ldk; a.ldv = ldv;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    ProfScope ps(st, ATP_K_STREAM, 0.0, moved_bytes(cache, batch, t));
    ATP_HIP(cache_write_rows(st, a, (int)esize(t), source_of(cache) == KV_PAGED_E4M3));
    return ATP_OK;
}

atp_status atp_cache_read(const atp_cache* cache, const atp_batch* batch, void* K, void* V, int64_t ldk, int64_t ldv, atp_dtype t,
                          void* hip_stream) {
    ServeArgs a;
    const atp_status s = take_cache(cache, batch, t, a, true);
    if (s != ATP_OK) return s;
    if (!a.tokens) return ATP_OK;
    const int64_t row = (int64_t)a.kv_heads * a.dh;
    if (bad_rows(K, ldk, row, t) || bad_rows(V, ldv, row, t)) return ATP_ERR_INVALID_ARG;
    a.Ko = K; a.Vo = V; a.ldk = ldk; a.ldv = ldv;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    ProfScope ps(st, ATP_K_STREAM, 0.0, moved_bytes(cache, batch, t));
    ATP_HIP(cache_read_rows(st, a, (int)esize(t), source_of(cache) == KV_PAGED_E4M3));
    return ATP_OK;
}

size_t atp_attention_packed_workspace(int64_t n_seq, int64_t tokens, int heads, int kv_heads, int d_h, atp_dtype t) {
    ServeArgs a;
    if (packed_shape(n_seq, tokens, heads, kv_heads, d_h, t, a) != ATP_OK || !tokens) return 0;
    return serve_attention_workspace(a, KV_PACKED, (int)esize(t), 0);
}

atp_status atp_attention_packed(const void* Q, const void* K, const void* V, void* O, int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldo,
                                const int32_t* offsets, int64_t n_seq, int64_t tokens, int heads, int kv_heads, int d_h, int causal,
                                float scale, void* workspace, size_t workspace_bytes, atp_dtype t, void* hip_stream) {
    ServeArgs a;
    const atp_status s = packed_shape(n_seq, tokens, heads, kv_heads, d_h, t, a);
    if (s != ATP_OK) return s;
    if (!tokens) return ATP_OK;
    if (!offsets || ((uintptr_t)offsets & 3) || !aligned16(workspace)) return ATP_ERR_INVALID_ARG;
    const int64_t qrow = (int64_t)heads * d_h, krow = (int64_t)kv_heads * d_h;
    if (bad_rows(Q, ldq, qrow, t) || bad_rows(O, ldo, qrow, t) || bad_rows(K, ldk, krow, t) || bad_rows(V, ldv, krow, t)) return ATP_ERR_INVALID_ARG;
    const size_t need = serve_attention_workspace(a, KV_PACKED, (int)esize(t), 0);
    if (need && (!workspace || workspace_bytes < need)) return ATP_ERR_WORKSPACE;
    a.offsets = offsets;
    a.Q = Q; a.O = O; a.K = const_cast<void*>(K); a.V = const_cast<void*>(V);   // (read only)
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
    a.causal = causal != 0;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)d_h);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    // (the lengths are not known here: counted as if they were equal)
    const double len = (double)tokens / n_seq;
    ProfScope ps(st, ATP_K_ATTENTION, 4.0 * d_h * heads * tokens * (causal ? (len + 1) / 2 : len), 2.0 * tokens * (qrow + krow) * esize(t));
    ATP_HIP(serve_attention(st, a, KV_PACKED, (int)esize(t), 0, workspace));
    return ATP_OK;
}

size_t atp_attention_paged_workspace(const atp_cache* cache, const atp_batch* batch, int heads, int64_t max_new, atp_dtype t) {
    ServeArgs a;
    if (take_cache(cache, batch, t, a, false) != ATP_OK || !a.tokens) return 0;
    if (heads < 1 || heads % a.kv_heads || batch->tokens > 0x7fffffff / heads || max_new < 0) return 0;
    a.heads = heads;
    return serve_attention_workspace(a, source_of(cache), (int)esize(t), max_new);
}

atp_status atp_attention_paged(const void* Q, const atp_cache* cache, const atp_batch* batch, void* O, int64_t ldq, int64_t ldo, int heads,
                               int causal, float scale, int64_t max_new, void* workspace, size_t workspace_bytes, atp_dtype t,
                               void* hip_stream) {
    ServeArgs a;
    const atp_status s = take_cache(cache, batch, t, a, true);
    if (s != ATP_OK) return s;
    if (heads < 1 || heads % a.kv_heads || max_new < 0 || !aligned16(workspace)) return ATP_ERR_INVALID_ARG;
    if (batch->tokens > 0x7fffffff / heads) return ATP_ERR_UNSUPPORTED;
    if (!a.tokens) return ATP_OK;
    a.heads = heads;
    const int64_t qrow = (int64_t)heads * a.dh;
    if (bad_rows(Q, ldq, qrow, t) || bad_rows(O, ldo, qrow, t)) return ATP_ERR_INVALID_ARG;
    const KvSource src = source_of(cache);
    const size_t need = serve_attention_workspace(a, src, (int)esize(t), max_new);
    if (need && (!workspace || workspace_bytes < need)) return ATP_ERR_WORKSPACE;
    a.Q = Q; a.O = O; a.ldq = ldq; a.ldo = ldo;
    a.causal = causal != 0;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)a.dh);
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    // (the lengths are not known here: the queries' own bytes are counted)
    ProfScope ps(st, ATP_K_ATTENTION, 0.0, 2.0 * a.tokens * qrow * esize(t));
    ATP_HIP(serve_attention(st, a, src, (int)esize(t), max_new, workspace));
    return ATP_OK;
}

}  // extern "C"
