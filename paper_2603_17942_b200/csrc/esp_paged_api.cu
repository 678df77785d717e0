// C entry points of the operators over a paged key/value cache (declared in include/esp.h): checks of arguments and launches.
#include <math.h>
#include <string.h>

#include "esp_paged.cuh"

using namespace esp;

namespace {

int cuda_ok(cudaError_t e) { return e == cudaSuccess ? ESP_OK : ESP_E_CUDA; }
size_t elem_size(int32_t dtype) { return dtype == 0 ? 4 : 2; }
bool off(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }      // (NULL is on every boundary)

constexpr int32_t MAX_HEADS = 1 << 20, MAX_BATCH = 1 << 30;
// A token-major tensor of n_tokens tokens: 0 or an error.  written: its rows must not share elements.
int check_heads(const esp_heads* x, int32_t dtype, int32_t n_tokens, int32_t head_dim, bool written) {
    if ((!x->data && n_tokens > 0) || x->n_heads < 1 || x->n_heads > MAX_HEADS || x->token_stride < 0 || x->head_stride < 0) return ESP_E_ARG;
    if (off(x->data, elem_size(dtype))) return ESP_E_ARG;
    if (x->token_stride > ((int64_t)1 << 40) || x->head_stride > ((int64_t)1 << 40)) return ESP_E_ARG;
    if (written) {
        if (x->n_heads > 1 && x->head_stride < head_dim) return ESP_E_ARG;
        if (n_tokens > 1 && x->token_stride < head_dim) return ESP_E_ARG;
        // either the heads of a token lie inside its stride or the tokens of a head inside the head's
        const bool by_token = x->token_stride >= (__int128)(x->n_heads - 1) * x->head_stride + head_dim;
        const bool by_head = x->head_stride >= (__int128)(n_tokens - 1) * x->token_stride + head_dim;
        if (x->n_heads > 1 && n_tokens > 1 && !by_token && !by_head) return ESP_E_ARG;
    }
    return ESP_OK;
}
// (a stride that nothing is reached by is 0, so that it has no say in what the strides allow)
HeadsView view_of(const esp_heads* x, int32_t n_tokens) {
    HeadsView v;
    v.p = x ? x->data : nullptr;
    v.tok = x && n_tokens > 1 ? x->token_stride : 0;
    v.head = x && x->n_heads > 1 ? x->head_stride : 0;
    v.n = x ? x->n_heads : 0;
    return v;
}

int check_cache(const esp_paged_cache* c) {
    if (!c->k || !c->v || c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1) return ESP_E_ARG;
    if (c->dtype != 0 && c->dtype != 1) return ESP_E_BADCFG;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return ESP_E_BADCFG;
    if (off(c->k, elem_size(c->dtype)) || off(c->v, elem_size(c->dtype))) return ESP_E_ARG;
    if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return ESP_E_ARG;
    if (c->page_stride > ((int64_t)1 << 40) || c->token_stride > ((int64_t)1 << 40) || c->head_stride > ((int64_t)1 << 40)) return ESP_E_ARG;
    // no two pages, tokens or heads share elements (the pages of k may lie between those of v)
    if ((c->n_pages > 1 && c->page_stride < c->head_dim) || (c->page_size > 1 && c->token_stride < c->head_dim) ||
        (c->n_kv_heads > 1 && c->head_stride < c->head_dim)) return ESP_E_ARG;
    return ESP_OK;
}
// Slots that are written: no two of them share elements, whichever of pages, tokens and heads lie inside which.
int check_slots(const esp_paged_cache* c) {
    struct { int64_t stride, count; } dim[3] = {{c->page_stride, c->n_pages}, {c->token_stride, c->page_size}, {c->head_stride, c->n_kv_heads}};
    __int128 span = c->head_dim;
    for (int done = 0; done < 3; ++done) {                  // the smallest stride of those left: it has to span what lies inside
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (dim[i].count > 0 && (at < 0 || dim[i].stride < dim[at].stride)) at = i;
        if (dim[at].count > 1) {
            if (dim[at].stride < span) return ESP_E_ARG;
            span += (__int128)(dim[at].count - 1) * dim[at].stride;
        }
        dim[at].count = 0;
    }
    return ESP_OK;
}
int check_batch(const esp_paged_batch* b) {
    if (b->batch < 0 || b->batch > MAX_BATCH || b->max_new < 0) return ESP_E_ARG;
    if (b->batch > 0 && (!b->q_start || !b->kv_len || !b->page_table || b->table_pages < 1)) return ESP_E_ARG;
    if (b->batch > 1 && b->table_stride < b->table_pages) return ESP_E_ARG;
    if (off(b->q_start, 4) || off(b->kv_len, 4) || off(b->page_table, 4) || off(b->status, 4)) return ESP_E_ARG;
    return ESP_OK;
}
PagesView pages_of(const esp_paged_cache* c) {
    PagesView p;
    p.k = c->k; p.v = c->v;
    p.page = c->n_pages > 1 ? c->page_stride : 0;
    p.tok = c->page_size > 1 ? c->token_stride : 0;
    p.head = c->n_kv_heads > 1 ? c->head_stride : 0;
    p.n_pages = c->n_pages; p.page_size = c->page_size; p.page_shift = c->page_size <= (1 << 30) ? shift_of(c->page_size) : -1;
    return p;
}
SeqTable seqs_of(const esp_paged_batch* b, const esp_paged_cache* c, int32_t n_tokens) {
    SeqTable t;
    t.q_start = b->q_start; t.kv_len = b->kv_len; t.table = b->page_table;
    t.batch = b->batch; t.table_stride = b->table_stride; t.max_new = b->max_new; t.n_tokens = n_tokens;
    const int64_t cap = (int64_t)b->table_pages * c->page_size;
    t.kv_cap = cap < paged::KV_LIMIT ? (int32_t)cap : paged::KV_LIMIT;
    t.status = b->status;
    return t;
}

int check_rope(const esp_rope_cfg* r) {
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > ESP_ROPE_MAX_DIM) return ESP_E_BADCFG;
    if (r->interleaved != 0 && r->interleaved != 1) return ESP_E_BADCFG;
    if (r->scaling < ESP_ROPE_PLAIN || r->scaling > ESP_ROPE_INDEX) return ESP_E_BADCFG;
    if (!(r->base > 0.f) || !isfinite(r->base) || !isfinite(r->amplitude)) return ESP_E_BADCFG;
    if (r->scaling != ESP_ROPE_PLAIN && (!(r->factor > 0.f) || !isfinite(r->factor))) return ESP_E_BADCFG;
    if (r->scaling == ESP_ROPE_BASE && r->rotary_dim < 4) return ESP_E_BADCFG;
    if (r->scaling == ESP_ROPE_ROTATIONS || r->scaling == ESP_ROPE_INDEX) {
        if (r->original_len < 1 || !(r->low > 0.f) || !(r->high > r->low) || !isfinite(r->high)) return ESP_E_BADCFG;
        if (r->scaling == ESP_ROPE_INDEX && !(r->base > 1.f)) return ESP_E_BADCFG;
    }
    return ESP_OK;
}
// radians per position of every pair, in extended precision (as their formulas in esp.h)
void frequencies(const esp_rope_cfg* r, long double* f) {
    const long double two_pi = 6.283185307179586476925286766559L;
    const long double rd = r->rotary_dim, len = r->original_len, factor = r->factor;
    long double base = r->base;
    if (r->scaling == ESP_ROPE_BASE) base *= powl(factor, rd / (rd - 2.0L));
    long double lo = 0.0L, hi = 0.0L;
    if (r->scaling == ESP_ROPE_INDEX) {
        // index of the pair that turns n times in the original length: len * base^(-2i/rd) = 2 pi n
        lo = floorl(rd * logl(len / (r->high * two_pi)) / (2.0L * logl(base)));
        hi = ceill(rd * logl(len / (r->low * two_pi)) / (2.0L * logl(base)));
        lo = lo < 0.0L ? 0.0L : lo;
        hi = hi > rd - 1.0L ? rd - 1.0L : hi;
        if (hi - lo < 0.001L) hi = lo + 0.001L;
    }
    for (int i = 0; i < r->rotary_dim / 2; ++i) {
        long double x = powl(base, -2.0L * i / rd), w = 1.0L;
        if (r->scaling == ESP_ROPE_LINEAR) w = 0.0L;
        else if (r->scaling == ESP_ROPE_ROTATIONS) w = (len * x / two_pi - r->low) / ((long double)r->high - r->low);
        else if (r->scaling == ESP_ROPE_INDEX) w = 1.0L - (i - lo) / (hi - lo);
        w = w < 0.0L ? 0.0L : (w > 1.0L ? 1.0L : w);
        f[i] = w == 1.0L ? x : x * (w + (1.0L - w) / factor);
    }
}

// What esp_qk_norm_rope and esp_paged_append share of their rotation's arguments.
int set_rope(NormRopeArgs& a, const esp_rope_cfg* rope, const void* table, int32_t head_dim) {
    if (!rope) return ESP_OK;
    if (const int rc = check_rope(rope)) return rc;
    if (rope->rotary_dim > head_dim) return ESP_E_BADCFG;
    if (!table || off(table, 16)) return ESP_E_ARG;
    a.freq = reinterpret_cast<const uint64_t*>(table);
    a.pairs = rope->rotary_dim / 2;
    a.interleaved = rope->interleaved;
    a.amplitude = rope->amplitude;
    return ESP_OK;
}

}  // namespace

extern "C" {

int esp_rope_frequencies(const esp_rope_cfg* rope, double* out) {
    if (!rope || !out) return ESP_E_ARG;
    if (const int rc = check_rope(rope)) return rc;
    long double f[ESP_ROPE_MAX_DIM / 2];
    frequencies(rope, f);
    for (int i = 0; i < rope->rotary_dim / 2; ++i) out[i] = (double)f[i];
    return ESP_OK;
}

int esp_rope_table_bytes(const esp_rope_cfg* rope, size_t* bytes_out) {
    if (!rope || !bytes_out) return ESP_E_ARG;
    if (const int rc = check_rope(rope)) return rc;
    *bytes_out = sizeof(uint64_t) * ((size_t)rope->rotary_dim / 2 + 1) / 2 * 2;
    return ESP_OK;
}

int esp_rope_table(const esp_rope_cfg* rope, void* table, size_t table_bytes, void* cuda_stream) {
    size_t need = 0;
    if (const int rc = esp_rope_table_bytes(rope, &need)) return rc;
    if (!table || off(table, 16)) return ESP_E_ARG;
    if (table_bytes < need) return ESP_E_WORKSPACE;
    long double f[ESP_ROPE_MAX_DIM / 2];
    uint64_t turns[ESP_ROPE_MAX_DIM / 2];
    frequencies(rope, f);
    for (int i = 0; i < rope->rotary_dim / 2; ++i) {
        const long double t = fmodl(f[i] / 6.283185307179586476925286766559L, 1.0L) * 18446744073709551616.0L;
        turns[i] = t >= 18446744073709551615.0L ? ~0ull : (uint64_t)(t + 0.5L);
    }
    launch_rope_table(turns, rope->rotary_dim / 2, reinterpret_cast<uint64_t*>(table), reinterpret_cast<cudaStream_t>(cuda_stream));
    return cuda_ok(cudaGetLastError());
}

int esp_qk_norm_rope(int32_t dtype, int32_t n_tokens, int32_t head_dim, const esp_heads* q, const esp_heads* k, const void* q_gain, const void* k_gain,
                     float eps, const esp_rope_cfg* rope, const void* rope_table, const int32_t* positions, const esp_heads* q_out,
                     const esp_heads* k_out, void* cuda_stream) {
    if (dtype != 0 && dtype != 1) return ESP_E_BADCFG;
    if (head_dim < 1 || head_dim > ESP_ROPE_MAX_DIM) return ESP_E_BADCFG;
    if (n_tokens < 0 || n_tokens > paged::KV_LIMIT || (!q && !k) || !q != !q_out || !k != !k_out || !(eps >= 0.f)) return ESP_E_ARG;
    if ((q_gain && !q) || (k_gain && !k) || (rope && !positions && n_tokens > 0)) return ESP_E_ARG;
    if (off(q_gain, elem_size(dtype)) || off(k_gain, elem_size(dtype)) || off(positions, 4)) return ESP_E_ARG;
    for (int i = 0; i < 2; ++i) {
        const esp_heads *x = i ? k : q, *y = i ? k_out : q_out;
        if (!x) continue;
        if (const int rc = check_heads(x, dtype, n_tokens, head_dim, false)) return rc;
        if (const int rc = check_heads(y, dtype, n_tokens, head_dim, true)) return rc;
        if (x->n_heads != y->n_heads) return ESP_E_ARG;
        if (x->data == y->data && ((n_tokens > 1 && x->token_stride != y->token_stride) || (x->n_heads > 1 && x->head_stride != y->head_stride))) return ESP_E_ARG;
    }
    NormRopeArgs a;
    memset(&a, 0, sizeof(a));
    if (const int rc = set_rope(a, rope, rope_table, head_dim)) return rc;
    if (n_tokens == 0) return ESP_OK;
    a.in[0] = view_of(q, n_tokens); a.in[1] = view_of(k, n_tokens); a.in[2] = view_of(nullptr, n_tokens);
    a.out[0] = view_of(q_out, n_tokens); a.out[1] = view_of(k_out, n_tokens);
    a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps;
    a.positions = positions;
    a.n_tokens = n_tokens; a.D = head_dim;
    if (launch_norm_rope(dtype, a, reinterpret_cast<cudaStream_t>(cuda_stream))) return ESP_E_BADCFG;
    return cuda_ok(cudaGetLastError());
}

int esp_paged_append(int32_t n_tokens, const esp_paged_cache* cache, const esp_paged_batch* batch, const esp_heads* k, const esp_heads* v,
                     const esp_heads* q, const void* q_gain, const void* k_gain, float eps, const esp_rope_cfg* rope, const void* rope_table,
                     const int32_t* positions, const esp_heads* q_out, void* cuda_stream) {
    if (!cache || !batch || !k || !v || n_tokens < 0 || n_tokens > paged::KV_LIMIT || !q != !q_out || (q_gain && !q) || !(eps >= 0.f)) return ESP_E_ARG;
    if (const int rc = check_cache(cache)) return rc;
    if (const int rc = check_slots(cache)) return rc;
    if (const int rc = check_batch(batch)) return rc;
    if (off(q_gain, elem_size(cache->dtype)) || off(k_gain, elem_size(cache->dtype)) || off(positions, 4)) return ESP_E_ARG;
    const esp_heads* ins[3] = {k, v, q};
    for (int i = 0; i < 3; ++i) {
        if (!ins[i]) continue;
        if (const int rc = check_heads(ins[i], cache->dtype, n_tokens, cache->head_dim, false)) return rc;
        if (i < 2 && ins[i]->n_heads != cache->n_kv_heads) return ESP_E_ARG;
    }
    if (q) {
        if (const int rc = check_heads(q_out, cache->dtype, n_tokens, cache->head_dim, true)) return rc;
        if (q->n_heads != q_out->n_heads) return ESP_E_ARG;
        if (q->data == q_out->data && ((n_tokens > 1 && q->token_stride != q_out->token_stride) || (q->n_heads > 1 && q->head_stride != q_out->head_stride))) return ESP_E_ARG;
    }
    NormRopeArgs a;
    memset(&a, 0, sizeof(a));
    if (const int rc = set_rope(a, rope, rope_table, cache->head_dim)) return rc;
    if (n_tokens == 0 || batch->batch == 0 || batch->max_new == 0) return ESP_OK;
    a.in[0] = view_of(q, n_tokens); a.in[1] = view_of(k, n_tokens); a.in[2] = view_of(v, n_tokens);
    a.out[0] = view_of(q_out, n_tokens); a.out[1] = view_of(nullptr, n_tokens);
    a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps;
    a.positions = positions;
    a.n_tokens = n_tokens; a.D = cache->head_dim;
    a.pages = pages_of(cache);
    a.seq = seqs_of(batch, cache, n_tokens);
    a.append = 1;
    if (launch_norm_rope(cache->dtype, a, reinterpret_cast<cudaStream_t>(cuda_stream))) return ESP_E_BADCFG;
    return cuda_ok(cudaGetLastError());
}

// scratch layout: [split tiles][split partials: weighted values][split partials: (maximum, sum)]
int esp_paged_attention_scratch_bytes(int32_t n_q_heads, int32_t head_dim, size_t* bytes_out) {
    if (!bytes_out || n_q_heads < 1) return ESP_E_ARG;
    if (head_dim != 32 && head_dim != 64 && head_dim != 128) return ESP_E_BADCFG;
    const size_t rows = (size_t)PAGED_MAX_SMS * 2 * PAGED_MAX_PAIRS;
    *bytes_out = 2 * sizeof(MergeDesc) * PAGED_MAX_CTAS + rows * head_dim * sizeof(float) + rows * sizeof(float2);
    return ESP_OK;
}

int esp_paged_attention(int32_t n_tokens, const esp_paged_cache* cache, const esp_paged_batch* batch, const esp_heads* q, const uint64_t* anc,
                        int32_t window, float scale, const esp_heads* out, float* lse, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    if (!cache || !batch || !q || !out || !scratch || n_tokens < 0 || n_tokens > paged::KV_LIMIT || window < 0 || !(scale >= 0.f) || !isfinite(scale)) return ESP_E_ARG;
    if (const int rc = check_cache(cache)) return rc;
    if (const int rc = check_batch(batch)) return rc;
    if (const int rc = check_heads(q, cache->dtype, n_tokens, cache->head_dim, false)) return rc;
    if (const int rc = check_heads(out, cache->dtype, n_tokens, cache->head_dim, true)) return rc;
    if (q->n_heads != out->n_heads || (n_tokens > 0 && q->data == out->data)) return ESP_E_ARG;
    if (q->n_heads % cache->n_kv_heads || q->n_heads / cache->n_kv_heads > 64) return ESP_E_BADCFG;
    if (anc && (batch->max_new > RT || window)) return ESP_E_ARG;
    if (off(anc, 8) || off(lse, 4)) return ESP_E_ARG;
    size_t need = 0;
    if (const int rc = esp_paged_attention_scratch_bytes(q->n_heads, cache->head_dim, &need)) return rc;
    if (scratch_bytes < need || off(scratch, 256)) return ESP_E_WORKSPACE;
    if (n_tokens == 0 || batch->batch == 0 || batch->max_new == 0) return ESP_OK;
    int n_sm = current_sm_count();
    if (n_sm < 1) return ESP_E_CUDA;
    if (n_sm > PAGED_MAX_SMS) n_sm = PAGED_MAX_SMS;
    PagedAttnArgs a;
    memset(&a, 0, sizeof(a));
    a.q = view_of(q, n_tokens); a.out = view_of(out, n_tokens); a.lse = lse;
    a.pages = pages_of(cache);
    a.seq = seqs_of(batch, cache, n_tokens);
    a.anc = reinterpret_cast<const unsigned long long*>(anc);
    a.Hq = q->n_heads; a.Hkv = cache->n_kv_heads; a.group = a.Hq / a.Hkv; a.D = cache->head_dim;
    a.window = window > paged::KV_LIMIT ? 0 : window;      // no position is that far back
    a.scale_log2 = (float)(1.4426950408889634 * (scale != 0.f ? (double)scale : 1.0 / sqrt((double)a.D)));
    const size_t rows = (size_t)PAGED_MAX_SMS * 2 * PAGED_MAX_PAIRS;
    a.min_units = 1;
    a.desc = reinterpret_cast<MergeDesc*>(scratch);
    a.part_o = reinterpret_cast<float4*>(a.desc + 2 * PAGED_MAX_CTAS);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + rows * (a.D / 4));
    const size_t es = elem_size(cache->dtype), quad = 4 * es;
    auto by4 = [&](const void* p, int64_t s0, int64_t s1, int64_t s2) {
        return reinterpret_cast<uintptr_t>(p) % quad == 0 && s0 % 4 == 0 && s1 % 4 == 0 && s2 % 4 == 0;
    };
    a.out_vec = by4(a.out.p, a.out.tok, a.out.head, 0);
    a.vec = by4(a.q.p, a.q.tok, a.q.head, 0) && by4(a.pages.k, a.pages.page, a.pages.tok, a.pages.head) && by4(a.pages.v, 0, 0, 0);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    const int rc = paged_few_supported(cache->dtype, a)  ? launch_paged_few(a, n_sm, s)
                   : paged_tc_supported(cache->dtype, a) ? launch_paged_tc(a, n_sm, s)
                                                         : launch_paged_simt(cache->dtype, a, n_sm, s);
    const cudaError_t e = cudaGetLastError();       // taken in either case: the next call's error is its own
    return rc ? ESP_E_CUDA : cuda_ok(e);
}

int esp_paged_status(const int32_t* status, void* cuda_stream, int32_t* device_status_out) {
    if (!status || off(status, 4)) return ESP_E_ARG;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    int32_t e = 0;
    if (cudaMemcpyAsync(&e, status, sizeof(e), cudaMemcpyDeviceToHost, s) != cudaSuccess) return ESP_E_CUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return ESP_E_CUDA;
    if (device_status_out) *device_status_out = e;
    return e ? ESP_E_DEVICE : ESP_OK;
}

}  // extern "C"
