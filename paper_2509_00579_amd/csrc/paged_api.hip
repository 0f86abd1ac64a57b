// The C entry points of the paged cache of 8-bit codes: checks of what the host can see, and the launches.
#include <stdio.h>

#include "api_error.h"
#include "paged.cuh"

using namespace kvc;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int kMaxGroup = 32, kMaxPagesPerSeq = 1 << 20;

kvcomp_status check_config(const kvcomp_paged_config *c) {
    if (!c) return fail(KVCOMP_ERR_INVALID_ARG, "NULL argument");
    if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > kMaxGroup)
        return fail(KVCOMP_ERR_INVALID_ARG, "n_q_heads must be 1 to %d times n_kv_heads", kMaxGroup);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(KVCOMP_ERR_INVALID_ARG, "head_dim must be 64 or 128");
    if (c->data_type != KVCOMP_FP16 && c->data_type != KVCOMP_BF16) return fail(KVCOMP_ERR_INVALID_ARG, "unknown data_type");
    if (c->code_type != KVCOMP_INT8 && c->code_type != KVCOMP_E4M3) return fail(KVCOMP_ERR_INVALID_ARG, "unknown code_type");
    if (c->n_pages < 1 || c->n_tails < 1) return fail(KVCOMP_ERR_INVALID_ARG, "n_pages and n_tails must be positive");
    if (c->max_pages < 1 || c->max_pages > kMaxPagesPerSeq)
        return fail(KVCOMP_ERR_INVALID_ARG, "max_pages must be 1 to %d", kMaxPagesPerSeq);
    return KVCOMP_OK;
}

kvcomp_status check_all(const kvcomp_paged_config *c, const kvcomp_paged_cache *m, const kvcomp_paged_batch *b, PagedGeo *g) {
    kvcomp_status st = check_config(c);
    if (st) return st;
    if (!m || !b || !m->d_k_codes || !m->d_v_codes || !m->d_scales || !m->d_k_tail || !m->d_v_tail || !m->d_fault)
        return fail(KVCOMP_ERR_INVALID_ARG, "NULL argument");
    if (!aligned16(m->d_k_codes) || !aligned16(m->d_v_codes) || !aligned16(m->d_scales) || !aligned16(m->d_k_tail) ||
        !aligned16(m->d_v_tail) || (reinterpret_cast<uintptr_t>(m->d_fault) & 3u))
        return fail(KVCOMP_ERR_INVALID_ARG, "the cache's tensors must be 16-byte aligned");
    if (b->batch < 0 || (b->batch && (!b->d_lens || !b->d_table || !b->d_tails))) return fail(KVCOMP_ERR_INVALID_ARG, "bad batch");
    if ((long long)b->batch * c->n_q_heads > (1ll << 24)) return fail(KVCOMP_ERR_INVALID_ARG, "more than 2^24 sequences times query heads");
    g->H = c->n_kv_heads;
    g->G = c->n_q_heads / c->n_kv_heads;
    g->n_pages = c->n_pages;
    g->n_tails = c->n_tails;
    g->max_pages = c->max_pages;
    g->batch = b->batch;
    g->k_codes = static_cast<uint8_t *>(m->d_k_codes);
    g->v_codes = static_cast<uint8_t *>(m->d_v_codes);
    g->scales = m->d_scales;
    g->k_tail = static_cast<uint16_t *>(m->d_k_tail);
    g->v_tail = static_cast<uint16_t *>(m->d_v_tail);
    g->fault = m->d_fault;
    g->lens = b->d_lens;
    g->table = b->d_table;
    g->tails = b->d_tails;
    return KVCOMP_OK;
}

// a tensor of rows [n][heads][head_dim] with `stride` elements from row to row
kvcomp_status check_rows(const char *name, const void *p, size_t stride, int heads, int head_dim) {
    if (!p) return fail(KVCOMP_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned16(p) || stride % 8) return fail(KVCOMP_ERR_INVALID_ARG, "rows of %s must start at multiples of 16 bytes", name);
    if (stride < (size_t)heads * head_dim) return fail(KVCOMP_ERR_INVALID_ARG, "rows of %s overlap", name);
    return KVCOMP_OK;
}

// Whether two tensors of `rows` rows have 16-bit elements in common; slices of one buffer's rows do not.
bool overlap(const void *a, size_t a_stride, size_t a_width, const void *b, size_t b_stride, size_t b_width, long long rows) {
    if (reinterpret_cast<uintptr_t>(a) > reinterpret_cast<uintptr_t>(b)) return overlap(b, b_stride, b_width, a, a_stride, a_width, rows);
    const size_t off = (reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a)) / 2;
    if (off >= (size_t)(rows - 1) * a_stride + a_width) return false;
    if (rows == 1 || a_stride != b_stride) return true;
    return off % a_stride < a_width || off % a_stride + b_width > a_stride;
}

__global__ void paged_clear_kernel(uint32_t *word, uint32_t bits) {
    __hip_atomic_fetch_and(word, ~bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace

extern "C" {

kvcomp_status kvcomp_paged_append(const kvcomp_paged_config *cfg, const kvcomp_paged_cache *cache,
                                  const kvcomp_paged_batch *seqs, const kvcomp_paged_new *fresh, void *stream) {
    PagedGeo g;
    kvcomp_status st = check_all(cfg, cache, seqs, &g);
    if (st) return st;
    if (!fresh) return fail(KVCOMP_ERR_INVALID_ARG, "NULL argument");
    const kvcomp_paged_new &f = *fresh;
    if (f.n_tokens < 0) return fail(KVCOMP_ERR_INVALID_ARG, "n_tokens is negative");
    if (!f.d_starts && f.n_tokens != g.batch) return fail(KVCOMP_ERR_INVALID_ARG, "without d_starts there is one token per sequence");
    if ((long long)f.n_tokens * cfg->n_q_heads > (1ll << 30)) return fail(KVCOMP_ERR_INVALID_ARG, "more than 2^30 tokens times query heads");
    PagedNew n = {};
    n.rot_dim = 0;
    if (f.d_cos_sin) {
        if (f.rot_dim < 16 || f.rot_dim % 16 || f.rot_dim > cfg->head_dim)
            return fail(KVCOMP_ERR_INVALID_ARG, "rot_dim must be a multiple of 16, at most head_dim");
        if (!aligned16(f.d_cos_sin) || f.n_positions < 1) return fail(KVCOMP_ERR_INVALID_ARG, "d_cos_sin must be 16-byte aligned and hold a position");
        if (f.n_axes < 1 || f.n_axes > 3 || (f.n_axes > 1 && !f.d_positions))
            return fail(KVCOMP_ERR_INVALID_ARG, "n_axes must be 1 to 3, and several axes need positions");
        int sum = 0;
        for (int a = 0; a < f.n_axes; a++) {
            if (f.sections[a] < 0 || f.sections[a] % 4) return fail(KVCOMP_ERR_INVALID_ARG, "sections must be multiples of 4");
            sum += f.sections[a];
            if (a < 2) n.edge[a] = sum;
        }
        if (sum != f.rot_dim / 2) return fail(KVCOMP_ERR_INVALID_ARG, "sections must add up to rot_dim / 2");
        for (int a = f.n_axes - 1; a < 2; a++) n.edge[a] = 1 << 20;  // no such axis
        n.rot_dim = f.rot_dim;
        n.cos_sin = f.d_cos_sin;
        n.positions = f.d_positions;
        n.n_positions = f.n_positions;
        n.interleaved = f.interleaved != 0;
    }
    if (!g.batch || !f.n_tokens) return KVCOMP_OK;
    if ((st = check_rows("d_k", f.d_k, f.k_stride, cfg->n_kv_heads, cfg->head_dim))) return st;
    if ((st = check_rows("d_v", f.d_v, f.v_stride, cfg->n_kv_heads, cfg->head_dim))) return st;
    if (f.d_q || f.d_q_out) {
        if ((st = check_rows("d_q", f.d_q, f.q_stride, cfg->n_q_heads, cfg->head_dim))) return st;
        if ((st = check_rows("d_q_out", f.d_q_out, f.q_out_stride, cfg->n_q_heads, cfg->head_dim))) return st;
        const size_t wq = (size_t)cfg->n_q_heads * cfg->head_dim, wk = (size_t)cfg->n_kv_heads * cfg->head_dim;
        const bool in_place = f.d_q == f.d_q_out && f.q_stride == f.q_out_stride;
        if ((!in_place && overlap(f.d_q, f.q_stride, wq, f.d_q_out, f.q_out_stride, wq, f.n_tokens)) ||
            overlap(f.d_k, f.k_stride, wk, f.d_q_out, f.q_out_stride, wq, f.n_tokens) ||
            overlap(f.d_v, f.v_stride, wk, f.d_q_out, f.q_out_stride, wq, f.n_tokens))
            return fail(KVCOMP_ERR_INVALID_ARG, "d_q_out overlaps d_q (and is not the same rows), d_k or d_v");
    }
    n.n_tokens = f.n_tokens;
    n.starts = f.d_starts;
    n.k = static_cast<const uint16_t *>(f.d_k);
    n.v = static_cast<const uint16_t *>(f.d_v);
    n.q = static_cast<const uint16_t *>(f.d_q);
    n.q_out = static_cast<uint16_t *>(f.d_q_out);
    n.k_stride = f.k_stride;
    n.v_stride = f.v_stride;
    n.q_stride = f.q_stride;
    n.q_out_stride = f.q_out_stride;
    HIP_TRY(launch_paged_append(g, n, cfg->head_dim, cfg->data_type, cfg->code_type, static_cast<hipStream_t>(stream)));
    return KVCOMP_OK;
}

size_t kvcomp_paged_workspace_bytes(const kvcomp_paged_config *cfg) {
    if (check_config(cfg)) return 0;
    const size_t decode = (size_t)2 * kDecodeWGs * kDecodeRows, prefill = kPrefillStateRows;  // rows of states
    return 4 * (kTicketWords + (decode > prefill ? decode : prefill) * partial_pitch(cfg->head_dim));
}

// what both attention calls are given; sets up `a`
static kvcomp_status check_attn(const kvcomp_paged_config *cfg, long long rows, const void *d_q, size_t q_stride, float scale, int window, void *d_out,
                                size_t out_stride, void *d_workspace, size_t workspace_bytes, PagedAttn *a) {
    kvcomp_status st;
    if ((st = check_rows("d_q", d_q, q_stride, cfg->n_q_heads, cfg->head_dim))) return st;
    if ((st = check_rows("d_out", d_out, out_stride, cfg->n_q_heads, cfg->head_dim))) return st;
    const size_t width = (size_t)cfg->n_q_heads * cfg->head_dim;
    if (overlap(d_q, q_stride, width, d_out, out_stride, width, rows)) return fail(KVCOMP_ERR_INVALID_ARG, "d_q and d_out overlap");
    if (!d_workspace || !aligned16(d_workspace)) return fail(KVCOMP_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    if (workspace_bytes < kvcomp_paged_workspace_bytes(cfg)) return fail(KVCOMP_ERR_CAPACITY, "workspace too small");
    const float scale2 = scale * 1.44269504088896f;  // to powers of two
    if (!(scale2 - scale2 == 0.f)) return fail(KVCOMP_ERR_INVALID_ARG, "scale times log2(e) must be finite");
    if (window < 0) return fail(KVCOMP_ERR_INVALID_ARG, "window is negative");
    a->q = static_cast<const uint16_t *>(d_q);
    a->out = static_cast<uint16_t *>(d_out);
    a->q_stride = q_stride;
    a->out_stride = out_stride;
    a->scale = scale2;
    a->window = window > kMaxPagesPerSeq * kPBT ? 0 : window;
    a->tickets = static_cast<uint32_t *>(d_workspace);
    a->partials = static_cast<float *>(d_workspace) + kTicketWords;
    return KVCOMP_OK;
}

kvcomp_status kvcomp_paged_attn_decode(const kvcomp_paged_config *cfg, const kvcomp_paged_cache *cache,
                                       const kvcomp_paged_batch *seqs, const void *d_q, size_t q_stride, int q_len, float scale,
                                       int window, int max_len, void *d_out, size_t out_stride, void *d_workspace,
                                       size_t workspace_bytes, void *stream) {
    PagedGeo g;
    PagedAttn a;
    kvcomp_status st = check_all(cfg, cache, seqs, &g);
    if (st) return st;
    if (q_len < 1 || q_len > kDecodeRows || q_len * g.G > kDecodeRows)
        return fail(KVCOMP_ERR_INVALID_ARG, "q_len must be at least 1, and q_len times the group of query heads at most %d", kDecodeRows);
    if (g.batch > kMaxDecodeBatch) return fail(KVCOMP_ERR_INVALID_ARG, "more than %d sequences", kMaxDecodeBatch);
    if ((long long)g.batch * g.H * (g.max_pages + 8) > 0x7fffffffll)
        return fail(KVCOMP_ERR_INVALID_ARG, "more than 2^31 - 1 sequences times KV heads times max_pages");
    if (max_len < 0) return fail(KVCOMP_ERR_INVALID_ARG, "max_len is negative");
    if (!g.batch) return KVCOMP_OK;
    if ((st = check_attn(cfg, (long long)g.batch * q_len, d_q, q_stride, scale, window, d_out, out_stride, d_workspace, workspace_bytes, &a))) return st;
    HIP_TRY(launch_paged_decode(g, a, q_len, max_len, cfg->head_dim, cfg->data_type, cfg->code_type, static_cast<hipStream_t>(stream)));
    return KVCOMP_OK;
}

kvcomp_status kvcomp_paged_attn_prefill(const kvcomp_paged_config *cfg, const kvcomp_paged_cache *cache,
                                        const kvcomp_paged_batch *seqs, const void *d_q, size_t q_stride, const void *d_starts,
                                        int n_tokens, float scale, int window, int max_new, int max_len, void *d_out,
                                        size_t out_stride, void *d_workspace, size_t workspace_bytes, void *stream) {
    PagedGeo g;
    PagedAttn a;
    kvcomp_status st = check_all(cfg, cache, seqs, &g);
    if (st) return st;
    if (!d_starts || (reinterpret_cast<uintptr_t>(d_starts) & 3u)) return fail(KVCOMP_ERR_INVALID_ARG, "d_starts is NULL or not aligned");
    if (n_tokens < 0 || max_new < 0 || max_len < 0) return fail(KVCOMP_ERR_INVALID_ARG, "n_tokens, max_new or max_len is negative");
    if ((long long)n_tokens * cfg->n_q_heads > (1ll << 30)) return fail(KVCOMP_ERR_INVALID_ARG, "more than 2^30 tokens times query heads");
    if (!g.batch || !n_tokens) return KVCOMP_OK;
    if ((st = check_attn(cfg, n_tokens, d_q, q_stride, scale, window, d_out, out_stride, d_workspace, workspace_bytes, &a))) return st;
    HIP_TRY(launch_paged_prefill(g, a, static_cast<const int32_t *>(d_starts), n_tokens, max_new, max_len, cfg->head_dim,
                                 cfg->data_type, cfg->code_type, static_cast<hipStream_t>(stream)));
    return KVCOMP_OK;
}

kvcomp_status kvcomp_paged_check(const kvcomp_paged_cache *cache, void *stream) {
    if (!cache || !cache->d_fault) return fail(KVCOMP_ERR_INVALID_ARG, "NULL argument");
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint32_t fault = 0;
    HIP_TRY(hipMemcpyAsync(&fault, cache->d_fault, sizeof(fault), hipMemcpyDeviceToHost, s));
    HIP_TRY(hipStreamSynchronize(s));
    if (!fault) return KVCOMP_OK;
    // only what was read: kernels on other streams may have flagged something else since
    hipLaunchKernelGGL(paged_clear_kernel, dim3(1), dim3(1), 0, s, cache->d_fault, fault);
    HIP_TRY(hipGetLastError());
    HIP_TRY(hipStreamSynchronize(s));
    static const struct {
        uint32_t bit;
        const char *text;
    } kinds[] = {{kFaultPage, "a page that was needed is outside the cache"},
                 {kFaultTail, "a tail that was needed is outside the cache"},
                 {kFaultLength, "a length or a start does not fit"},
                 {kFaultPosition, "a position is outside the table of cosines and sines"},
                 {kFaultNonfinite, "an appended token held Inf or NaN"}};
    char text[256] = "";
    int at = 0;
    for (const auto &k : kinds)
        if (fault & k.bit) at += snprintf(text + at, sizeof(text) - at, "%s%s", at ? "; " : "", k.text);
    return fail(fault & ~kFaultNonfinite ? KVCOMP_ERR_STATE : KVCOMP_ERR_NONFINITE, "%s", text);
}

}  // extern "C"
