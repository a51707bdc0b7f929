// stride_abi.cpp -- the extern "C" entry points of libstride.so.
//
// Host-side argument checking (synchronous, before any launch), workspace
// carving and the launch sequence of each call.  Every launch is asynchronous
// on the caller's stream; nothing here synchronises or allocates.
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "common.hpp"

namespace stride {

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

WsLayout ws_layout(int64_t n_rollouts, int64_t n_tokens, int64_t n_units, int64_t fused_partials) {
    WsLayout w;
    size_t off = 0;
    w.counter = off;
    off += 256;
    w.unit_off = off;
    off += align256(sizeof(int64_t) * (size_t)(n_rollouts + 1));
    w.desc = off;
    const int64_t tiles = n_units > 0 ? (n_units + kScanTile - 1) / kScanTile : 0;
    off += align256(sizeof(TileDesc) * (size_t)tiles);
    w.stop_end = off;
    w.row_dom = off;
    off += align256((size_t)(n_tokens > 0 ? n_tokens : 0));
    w.fused = off;
    off += align256(8 * (size_t)(fused_partials > 0 ? fused_partials : 0));
    w.total = off;
    return w;
}

}  // namespace stride

using namespace stride;

namespace {

thread_local char g_err[512] = "";

stride_status fail(stride_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return st;
}

stride_status ok() {
    g_err[0] = '\0';
    return STRIDE_OK;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

stride_status check_layout(const stride_layout *L) {
    if (!L) return fail(STRIDE_ERR_INVALID_ARG, "layout is NULL");
    if (L->n_rollouts < 0 || L->n_turns < 0 || L->n_tokens < 0)
        return fail(STRIDE_ERR_INVALID_ARG, "negative layout size (R=%d T=%d N=%lld)", L->n_rollouts,
                    L->n_turns, (long long)L->n_tokens);
    if (!L->rollout_turn_off) return fail(STRIDE_ERR_INVALID_ARG, "rollout_turn_off is NULL");
    if (!L->turn_tok_off) return fail(STRIDE_ERR_INVALID_ARG, "turn_tok_off is NULL");
    if (L->n_tokens > 0 && L->n_turns == 0)
        return fail(STRIDE_ERR_INVALID_ARG, "N = %lld rows but no turns", (long long)L->n_tokens);
    if (L->n_turns > 0 && L->n_rollouts == 0)
        return fail(STRIDE_ERR_INVALID_ARG, "T = %d turns but no rollouts", L->n_turns);
    return STRIDE_OK;
}

stride_status check_ws(size_t need, void *ws, size_t ws_bytes) {
    if (!ws) return fail(STRIDE_ERR_WORKSPACE, "workspace is NULL (need %zu bytes)", need);
    if (!aligned(ws, 256)) return fail(STRIDE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < need)
        return fail(STRIDE_ERR_WORKSPACE, "workspace has %zu bytes, need %zu", ws_bytes, need);
    return STRIDE_OK;
}

// Bytes of workspace the row-domain table (scoring) or retained-row mask (gradient) needs.
size_t rows_ws_bytes(const stride_layout &L) { return ws_layout(L.n_rollouts, L.n_tokens, 0, 0).total; }

// Bytes of workspace the stop test needs: tile counter, unit offsets, tile descriptors.
size_t stop_ws_bytes(const stride_layout &L, int64_t n_units) {
    return ws_layout(L.n_rollouts, 0, n_units, 0).stop_end;
}

stride_status check_domains(const double *table, int32_t n_dom, const char *name) {
    if (!table) return fail(STRIDE_ERR_INVALID_ARG, "%s is NULL", name);
    if (n_dom < 1 || n_dom > STRIDE_MAX_DOMAINS)
        return fail(STRIDE_ERR_UNSUPPORTED, "n_dom = %d outside 1..%d", n_dom, STRIDE_MAX_DOMAINS);
    return STRIDE_OK;
}

// Keys of a sequence and rows of an attention call are counted in 32 bits, in tiles of up to 256.
constexpr int32_t kMaxCount = INT32_MAX - 255;
constexpr int32_t kMaxVocab = 1 << 30;  // that stride_sample takes

// A stride in elements, or a position in them, that keeps 16-byte accesses aligned.
bool whole_words(int64_t elements, int32_t dtype) { return elements % (dtype == STRIDE_BF16 ? 8 : 4) == 0; }

stride_status check_cache_sizes(const stride_kv_cache *c) {
    if (!c) return fail(STRIDE_ERR_INVALID_ARG, "cache is NULL");
    if (c->dtype != STRIDE_BF16 && c->dtype != STRIDE_F32)
        return fail(STRIDE_ERR_UNSUPPORTED, "dtype %d is neither STRIDE_BF16 nor STRIDE_F32", c->dtype);
    if (c->n_seqs < 0 || c->max_pages < 0 || c->n_pages < 0)
        return fail(STRIDE_ERR_INVALID_ARG, "negative cache size (n_seqs=%d max_pages=%d n_pages=%lld)",
                    c->n_seqs, c->max_pages, (long long)c->n_pages);
    if (c->n_heads < 1) return fail(STRIDE_ERR_INVALID_ARG, "n_heads = %d < 1", c->n_heads);
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
        return fail(STRIDE_ERR_UNSUPPORTED, "head_dim = %d is not 64, 96, 128 or 256", c->head_dim);
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(STRIDE_ERR_UNSUPPORTED, "page_size = %d is not a power of two in [1, 65536]", c->page_size);
    if ((int64_t)c->max_pages * c->page_size > kMaxCount)
        return fail(STRIDE_ERR_UNSUPPORTED, "max_pages * page_size = %lld passes 2^31 - 256",
                    (long long)c->max_pages * c->page_size);
    return STRIDE_OK;
}

stride_status check_cache(const stride_kv_cache *c) {
    const stride_status st = check_cache_sizes(c);
    if (st != STRIDE_OK) return st;
    if (c->n_seqs > 0) {
        if (!c->page_table) return fail(STRIDE_ERR_INVALID_ARG, "page_table is NULL");
        if (c->table_ld < c->max_pages)
            return fail(STRIDE_ERR_INVALID_ARG, "table_ld = %lld < max_pages = %d", (long long)c->table_ld,
                        c->max_pages);
    }
    if (c->n_pages > 0) {
        if (!c->k || !c->v) return fail(STRIDE_ERR_INVALID_ARG, "the cache's k or v is NULL");
        if (!aligned(c->k, 16) || !aligned(c->v, 16))
            return fail(STRIDE_ERR_UNSUPPORTED, "the cache's k and v must be 16-byte aligned");
    }
    for (const int64_t x : {c->k_page, c->k_slot, c->k_head, c->v_page, c->v_slot, c->v_head})
        if (!whole_words(x, c->dtype))
            return fail(STRIDE_ERR_UNSUPPORTED, "cache stride %lld is not a multiple of 16 bytes", (long long)x);
    return STRIDE_OK;
}

// The sizes of an attention call.
stride_status check_attention_sizes(const stride_kv_cache &c, int64_t n_q, int32_t n_heads_q) {
    if (n_q < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_q = %lld < 0", (long long)n_q);
    if (n_heads_q < 1 || n_heads_q % c.n_heads != 0)
        return fail(STRIDE_ERR_INVALID_ARG, "n_heads_q = %d is not a multiple of n_heads = %d", n_heads_q, c.n_heads);
    if (n_q > kMaxCount / n_heads_q)
        return fail(STRIDE_ERR_UNSUPPORTED, "n_q = %lld rows of %d heads pass 2^31 - 256", (long long)n_q, n_heads_q);
    if (n_q > 0 && c.n_seqs == 0) return fail(STRIDE_ERR_INVALID_ARG, "n_q = %lld rows but no sequences", (long long)n_q);
    if (n_q > 0 && (c.n_pages == 0 || c.max_pages == 0))
        return fail(STRIDE_ERR_INVALID_ARG, "n_q = %lld rows but a cache without pages", (long long)n_q);
    return STRIDE_OK;
}

// Rows [token, head, head_dim] of the cache's type.
stride_status check_rows(const char *name, const void *p, int64_t tok, int64_t head, int32_t dtype) {
    if (!p) return fail(STRIDE_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned(p, 16) || !whole_words(tok, dtype) || !whole_words(head, dtype))
        return fail(STRIDE_ERR_UNSUPPORTED, "%s and its strides (%lld, %lld elements) must be multiples of 16 bytes",
                    name, (long long)tok, (long long)head);
    return STRIDE_OK;
}

stride_status hip_fail(hipError_t e, const char *what) {
    return fail(STRIDE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

size_t stride_workspace_size(const stride_layout *layout, int32_t unit) {
    if (!layout) return 0;
    const int64_t n_units = (unit == STRIDE_UNIT_TOKEN) ? layout->n_tokens : layout->n_turns;
    return ws_layout(layout->n_rollouts, layout->n_tokens, n_units, 0).total;
}

const char *stride_last_error(void) { return g_err; }

stride_status stride_score(const stride_layout *layout, int32_t vocab, int64_t ld, int32_t dtype,
                           int32_t n_teachers, const void *const *teacher_logits,
                           const void *student_logits, const int32_t *token_ids, float *logp_t,
                           float *logp_s, float *kl, float *kl_full, double *turn_mean,
                           uint32_t *dev_flags, void *ws, size_t ws_bytes, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (vocab < 1) return fail(STRIDE_ERR_INVALID_ARG, "vocab = %d < 1", vocab);
    if (ld < vocab) return fail(STRIDE_ERR_INVALID_ARG, "ld = %lld < vocab = %d", (long long)ld, vocab);
    if (dtype != STRIDE_BF16 && dtype != STRIDE_F32)
        return fail(STRIDE_ERR_UNSUPPORTED, "dtype %d is neither STRIDE_BF16 nor STRIDE_F32", dtype);
    const int64_t esize = dtype == STRIDE_BF16 ? 2 : 4;
    if ((ld * esize) % 16 != 0)
        return fail(STRIDE_ERR_UNSUPPORTED, "row stride %lld bytes is not a multiple of 16",
                    (long long)(ld * esize));
    if (n_teachers < 1 || n_teachers > STRIDE_MAX_DOMAINS)
        return fail(STRIDE_ERR_UNSUPPORTED, "n_teachers = %d outside 1..%d", n_teachers,
                    STRIDE_MAX_DOMAINS);
    if (!student_logits && (logp_s || kl || kl_full))
        return fail(STRIDE_ERR_INVALID_ARG, "logp_s / kl / kl_full requested without student logits");
    // the student rows' results are written to logp_s, and kl is formed from it
    if (student_logits && !logp_s && L.n_tokens > 0)
        return fail(STRIDE_ERR_INVALID_ARG, "student_logits given without logp_s");
    if ((kl || kl_full) && !logp_s && L.n_tokens > 0)
        return fail(STRIDE_ERR_INVALID_ARG, "kl / kl_full need logp_s as well");
    if (L.n_tokens > 0) {
        if (!teacher_logits) return fail(STRIDE_ERR_INVALID_ARG, "teacher_logits is NULL");
        for (int d = 0; d < n_teachers; ++d) {
            if (!teacher_logits[d])
                return fail(STRIDE_ERR_INVALID_ARG, "teacher_logits[%d] is NULL", d);
            if (!aligned(teacher_logits[d], 16))
                return fail(STRIDE_ERR_UNSUPPORTED, "teacher_logits[%d] is not 16-byte aligned", d);
        }
        if (student_logits && !aligned(student_logits, 16))
            return fail(STRIDE_ERR_UNSUPPORTED, "student_logits is not 16-byte aligned");
        if (!token_ids) return fail(STRIDE_ERR_INVALID_ARG, "token_ids is NULL");
        if (!logp_t) return fail(STRIDE_ERR_INVALID_ARG, "logp_t is NULL");
    }
    if (L.n_turns > 0 && !turn_mean) return fail(STRIDE_ERR_INVALID_ARG, "turn_mean is NULL");
    const bool routed = n_teachers > 1 && L.domain != nullptr;
    if (routed) {
        st = check_ws(rows_ws_bytes(L), ws, ws_bytes);
        if (st != STRIDE_OK) return st;
    }

    PtrTable tp{};
    for (int d = 0; d < n_teachers && teacher_logits; ++d) tp.p[d] = teacher_logits[d];
    uint8_t *row_dom = nullptr;
    hipError_t e;
    if (routed && L.n_tokens > 0) {
        const WsLayout w = ws_layout(L.n_rollouts, L.n_tokens, 0, 0);
        row_dom = static_cast<uint8_t *>(ws) + w.row_dom;
        e = launch_row_domain(L, n_teachers, row_dom, dev_flags, stream);
        if (e != hipSuccess) return hip_fail(e, "row-domain launch");
    }
    if (kl_full)
        e = launch_score_pairs(dtype, tp, n_teachers, row_dom, student_logits, token_ids, logp_t,
                               logp_s, kl_full, L.n_tokens, vocab, ld, dev_flags, stream);
    else
        e = launch_score_rows(dtype, tp, n_teachers, row_dom, student_logits, token_ids, logp_t,
                              logp_s, L.n_tokens, vocab, ld, dev_flags, stream);
    if (e != hipSuccess) return hip_fail(e, "row-scoring launch");
    e = launch_turn_mean(L, logp_t, logp_s, kl, turn_mean, dev_flags, stream);
    if (e != hipSuccess) return hip_fail(e, "turn-mean launch");
    return ok();
}

size_t stride_fused_workspace_size(const stride_layout *layout, int32_t vocab) {
    if (!layout || vocab < 1 || layout->n_tokens < 0) return 0;
    return fused_ws_bytes(layout->n_tokens, vocab);
}

stride_status stride_score_fused(const stride_layout *layout, int32_t vocab, int32_t d,
                                 const void *hidden_t, const void *w_t, const void *student_logits,
                                 int64_t ld, const int32_t *token_ids, float *logp_t, float *logp_s,
                                 float *kl, double *turn_mean, uint32_t *dev_flags, void *ws,
                                 size_t ws_bytes, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (vocab < 1) return fail(STRIDE_ERR_INVALID_ARG, "vocab = %d < 1", vocab);
    if (d < 64 || d % 64 != 0 || d > kMaxFusedD)
        return fail(STRIDE_ERR_UNSUPPORTED,
                    "hidden size d = %d is not a multiple of 64 in [64, %d]", d, kMaxFusedD);
    if (!student_logits && (logp_s || kl))
        return fail(STRIDE_ERR_INVALID_ARG, "logp_s / kl requested without student logits");
    if (student_logits && !logp_s && L.n_tokens > 0)
        return fail(STRIDE_ERR_INVALID_ARG, "student_logits given without logp_s");
    if (L.n_tokens > 0) {
        if (!hidden_t || !w_t) return fail(STRIDE_ERR_INVALID_ARG, "hidden_t or w_t is NULL");
        if (!aligned(hidden_t, 16) || !aligned(w_t, 16))
            return fail(STRIDE_ERR_UNSUPPORTED, "hidden_t and w_t must be 16-byte aligned");
        if (!token_ids || !logp_t) return fail(STRIDE_ERR_INVALID_ARG, "token_ids or logp_t is NULL");
        if (student_logits) {
            if (ld < vocab)
                return fail(STRIDE_ERR_INVALID_ARG, "ld = %lld < vocab = %d", (long long)ld, vocab);
            if ((ld * 2) % 16 != 0 || !aligned(student_logits, 16))
                return fail(STRIDE_ERR_UNSUPPORTED, "student rows must be 16-byte aligned");
        }
    }
    if (L.n_turns > 0 && !turn_mean) return fail(STRIDE_ERR_INVALID_ARG, "turn_mean is NULL");
    const size_t need = fused_ws_bytes(L.n_tokens, vocab);
    if (!ws) return fail(STRIDE_ERR_WORKSPACE, "workspace is NULL (need %zu bytes)", need);
    if (!aligned(ws, 256)) return fail(STRIDE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (ws_bytes < need)
        return fail(STRIDE_ERR_WORKSPACE, "workspace has %zu bytes, need %zu", ws_bytes, need);

    hipError_t e = launch_fused_teacher(static_cast<const uint16_t *>(hidden_t),
                                        static_cast<const uint16_t *>(w_t), token_ids, logp_t,
                                        L.n_tokens, vocab, d, dev_flags, ws, stream);
    if (e != hipSuccess) return hip_fail(e, "fused projection launch");
    if (student_logits) {
        PtrTable sp{};
        sp.p[0] = student_logits;
        e = launch_score_rows(STRIDE_BF16, sp, 1, nullptr, nullptr, token_ids, logp_s, nullptr,
                              L.n_tokens, vocab, ld, dev_flags, stream);
        if (e != hipSuccess) return hip_fail(e, "student scoring launch");
    }
    e = launch_turn_mean(L, logp_t, logp_s, kl, turn_mean, dev_flags, stream);
    if (e != hipSuccess) return hip_fail(e, "turn-mean launch");
    return ok();
}

stride_status stride_stop(const stride_layout *layout, int32_t unit, const void *values,
                          const double *lambda, int32_t n_dom, const int32_t *start_unit,
                          double *cum, int32_t *stop_unit, int64_t *n_retained_tokens,
                          uint32_t *dev_flags, void *ws, size_t ws_bytes, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (unit != STRIDE_UNIT_TURN && unit != STRIDE_UNIT_TOKEN)
        return fail(STRIDE_ERR_INVALID_ARG, "unit %d is neither STRIDE_UNIT_TURN nor STRIDE_UNIT_TOKEN",
                    unit);
    st = check_domains(lambda, n_dom, "lambda");
    if (st != STRIDE_OK) return st;
    const int64_t n_units = (unit == STRIDE_UNIT_TURN) ? L.n_turns : L.n_tokens;
    if (n_units > 0 && (!values || !cum))
        return fail(STRIDE_ERR_INVALID_ARG, "values or cum is NULL");
    if (L.n_rollouts > 0 && !stop_unit) return fail(STRIDE_ERR_INVALID_ARG, "stop_unit is NULL");
    st = check_ws(stop_ws_bytes(L, n_units), ws, ws_bytes);
    if (st != STRIDE_OK) return st;
    DomainTable lt{};
    for (int i = 0; i < n_dom; ++i) lt.v[i] = lambda[i];
    const hipError_t e = launch_stop(L, unit, values, lt, n_dom, start_unit, cum, stop_unit,
                                     n_retained_tokens, dev_flags, ws, stream);
    if (e != hipSuccess) return hip_fail(e, "stop launch");
    return ok();
}

stride_status stride_stop_noalloc(const stride_layout *layout, int32_t unit, const void *values,
                                  const double *lambda, int32_t n_dom, const int32_t *start_unit,
                                  double *cum, int32_t *stop_unit, int64_t *n_retained_tokens,
                                  uint32_t *dev_flags, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (unit != STRIDE_UNIT_TURN && unit != STRIDE_UNIT_TOKEN)
        return fail(STRIDE_ERR_INVALID_ARG, "unit %d is neither STRIDE_UNIT_TURN nor STRIDE_UNIT_TOKEN",
                    unit);
    st = check_domains(lambda, n_dom, "lambda");
    if (st != STRIDE_OK) return st;
    const int64_t n_units = (unit == STRIDE_UNIT_TURN) ? L.n_turns : L.n_tokens;
    if (n_units > 0 && (!values || !cum))
        return fail(STRIDE_ERR_INVALID_ARG, "values or cum is NULL");
    if (L.n_rollouts > 0 && !stop_unit) return fail(STRIDE_ERR_INVALID_ARG, "stop_unit is NULL");
    const size_t need = stop_ws_bytes(L, n_units);
    if (need > (size_t)STRIDE_NOALLOC_SCRATCH_BYTES)
        return fail(STRIDE_ERR_UNSUPPORTED,
                    "layout needs %zu bytes of scratch (R = %d, %lld units); the fixed scratch "
                    "holds %zu: use stride_stop with a workspace",
                    need, L.n_rollouts, (long long)n_units, (size_t)STRIDE_NOALLOC_SCRATCH_BYTES);
    void *scratch = nullptr;
    hipError_t e = noalloc_scratch(&scratch);
    if (e != hipSuccess) return hip_fail(e, "scratch address lookup");
    DomainTable lt{};
    for (int i = 0; i < n_dom; ++i) lt.v[i] = lambda[i];
    e = launch_stop(L, unit, values, lt, n_dom, start_unit, cum, stop_unit, n_retained_tokens,
                    dev_flags, scratch, stream);
    if (e != hipSuccess) return hip_fail(e, "stop launch");
    return ok();
}

stride_status stride_stop_step(int32_t n_active, const int32_t *slot, const int64_t *new_off,
                               int32_t unit, const void *values, const int32_t *domain,
                               const double *lambda, int32_t n_dom, double *state_cum,
                               int32_t *state_units, int32_t *stop_unit, uint32_t *dev_flags,
                               hipStream_t stream) {
    if (n_active < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_active = %d < 0", n_active);
    if (unit != STRIDE_UNIT_TURN && unit != STRIDE_UNIT_TOKEN)
        return fail(STRIDE_ERR_INVALID_ARG, "unit %d is neither STRIDE_UNIT_TURN nor STRIDE_UNIT_TOKEN",
                    unit);
    stride_status st = check_domains(lambda, n_dom, "lambda");
    if (st != STRIDE_OK) return st;
    if (n_active > 0 && (!slot || !new_off || !values || !state_cum || !state_units || !stop_unit))
        return fail(STRIDE_ERR_INVALID_ARG, "slot, new_off, values and the state arrays are required");
    DomainTable lt{};
    for (int i = 0; i < n_dom; ++i) lt.v[i] = lambda[i];
    const hipError_t e = launch_stop_step(n_active, slot, new_off, unit, values, domain, lt, n_dom,
                                          state_cum, state_units, stop_unit, dev_flags, stream);
    if (e != hipSuccess) return hip_fail(e, "stop-step launch");
    return ok();
}

stride_status stride_restart_turn(const stride_layout *layout, int32_t unit, const void *values,
                                  const int32_t *stop_unit, const double *alpha, int32_t n_dom,
                                  const uint8_t *correct_mask, int32_t *k_star, int32_t *k0,
                                  int32_t *k_max, uint32_t *dev_flags, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (unit != STRIDE_UNIT_TURN && unit != STRIDE_UNIT_TOKEN)
        return fail(STRIDE_ERR_INVALID_ARG, "unit %d is neither STRIDE_UNIT_TURN nor STRIDE_UNIT_TOKEN",
                    unit);
    st = check_domains(alpha, n_dom, "alpha");
    if (st != STRIDE_OK) return st;
    const int64_t n_units = (unit == STRIDE_UNIT_TURN) ? L.n_turns : L.n_tokens;
    if (n_units > 0 && !values) return fail(STRIDE_ERR_INVALID_ARG, "values is NULL");
    if (L.n_rollouts > 0 && (!k_star || !k0))
        return fail(STRIDE_ERR_INVALID_ARG, "k_star or k0 is NULL");
    DomainTable at{};
    for (int i = 0; i < n_dom; ++i) at.v[i] = alpha[i];
    const hipError_t e = launch_restart(L, unit, values, stop_unit, at, n_dom, correct_mask, k_star,
                                        k0, k_max, dev_flags, stream);
    if (e != hipSuccess) return hip_fail(e, "restart launch");
    return ok();
}

stride_status stride_opd_grad(const stride_layout *layout, int32_t unit, int32_t vocab, int64_t ld,
                              int32_t dtype, const void *student_logits, const int32_t *token_ids,
                              const float *logp_t, const float *logp_s, const int32_t *start_unit,
                              const int32_t *stop_unit, float scale, void *grad, float *loss,
                              uint32_t *dev_flags, void *ws, size_t ws_bytes, hipStream_t stream) {
    stride_status st = check_layout(layout);
    if (st != STRIDE_OK) return st;
    const stride_layout &L = *layout;
    if (unit != STRIDE_UNIT_TURN && unit != STRIDE_UNIT_TOKEN)
        return fail(STRIDE_ERR_INVALID_ARG, "unit %d is neither STRIDE_UNIT_TURN nor STRIDE_UNIT_TOKEN",
                    unit);
    if (vocab < 1) return fail(STRIDE_ERR_INVALID_ARG, "vocab = %d < 1", vocab);
    if (ld < vocab) return fail(STRIDE_ERR_INVALID_ARG, "ld = %lld < vocab = %d", (long long)ld, vocab);
    if (dtype != STRIDE_BF16 && dtype != STRIDE_F32)
        return fail(STRIDE_ERR_UNSUPPORTED, "dtype %d is neither STRIDE_BF16 nor STRIDE_F32", dtype);
    const int64_t esize = dtype == STRIDE_BF16 ? 2 : 4;
    if ((ld * esize) % 16 != 0)
        return fail(STRIDE_ERR_UNSUPPORTED, "row stride %lld bytes is not a multiple of 16",
                    (long long)(ld * esize));
    if (L.n_tokens > 0) {
        if (!student_logits || !grad || !token_ids || !logp_t || !logp_s)
            return fail(STRIDE_ERR_INVALID_ARG, "student_logits, grad, token_ids, logp_t and logp_s are required");
        if (!aligned(student_logits, 16) || !aligned(grad, 16))
            return fail(STRIDE_ERR_UNSUPPORTED, "student_logits and grad must be 16-byte aligned");
    }
    st = check_ws(rows_ws_bytes(L), ws, ws_bytes);
    if (st != STRIDE_OK) return st;
    const WsLayout w = ws_layout(L.n_rollouts, L.n_tokens, 0, 0);
    uint8_t *mask = static_cast<uint8_t *>(ws) + w.row_dom;
    const hipError_t e = launch_opd_grad(L, unit, dtype, vocab, ld, student_logits, token_ids,
                                         logp_t, logp_s, start_unit, stop_unit, scale, grad, loss,
                                         dev_flags, mask, stream);
    if (e != hipSuccess) return hip_fail(e, "gradient launch");
    return ok();
}

stride_status stride_kv_append(const stride_kv_cache *cache, int64_t n_tokens, const int32_t *seq,
                               const int32_t *slot, const int32_t *pos, const void *k, int64_t k_tok,
                               int64_t k_head, const void *v, int64_t v_tok, int64_t v_head,
                               int32_t n_heads_q, const void *q, int64_t q_tok, int64_t q_head, void *q_out,
                               int64_t qo_tok, int64_t qo_head, const void *k_weight, const void *q_weight,
                               float eps, const float *rope, int32_t max_pos, int32_t rot,
                               int32_t rope_style, uint32_t *dev_flags, hipStream_t stream) {
    stride_status st = check_cache(cache);
    if (st != STRIDE_OK) return st;
    const stride_kv_cache &c = *cache;
    if (n_tokens < 0 || n_heads_q < 0 || max_pos < 0)
        return fail(STRIDE_ERR_INVALID_ARG, "negative size (n_tokens=%lld n_heads_q=%d max_pos=%d)",
                    (long long)n_tokens, n_heads_q, max_pos);
    if (rot < 0 || rot > c.head_dim || rot % 16 != 0)
        return fail(STRIDE_ERR_UNSUPPORTED, "rot = %d is not a multiple of 16 in [0, head_dim = %d]", rot, c.head_dim);
    if (rope_style != STRIDE_ROPE_HALF && rope_style != STRIDE_ROPE_PAIRS)
        return fail(STRIDE_ERR_INVALID_ARG, "rope_style %d is neither STRIDE_ROPE_HALF nor STRIDE_ROPE_PAIRS",
                    rope_style);
    if (!(eps >= 0.0f)) return fail(STRIDE_ERR_INVALID_ARG, "eps = %g is not >= 0", (double)eps);
    if (n_heads_q == 0 && (q || q_out || q_weight))
        return fail(STRIDE_ERR_INVALID_ARG, "q, q_out or q_weight given with n_heads_q = 0");
    if (n_tokens > INT32_MAX / ((int64_t)n_heads_q + 2 * (int64_t)c.n_heads))
        return fail(STRIDE_ERR_UNSUPPORTED, "n_tokens = %lld of %lld heads pass 2^31 - 1", (long long)n_tokens,
                    (long long)n_heads_q + 2 * (long long)c.n_heads);
    if (!aligned(k_weight, 16) || !aligned(q_weight, 16) || !aligned(rope, 16))
        return fail(STRIDE_ERR_UNSUPPORTED, "weights and rope must be 16-byte aligned");
    if (n_tokens > 0) {
        if (!seq || !slot) return fail(STRIDE_ERR_INVALID_ARG, "seq or slot is NULL");
        if (rot > 0 && (!rope || !pos)) return fail(STRIDE_ERR_INVALID_ARG, "rope or pos is NULL with rot = %d", rot);
        st = check_rows("k", k, k_tok, k_head, c.dtype);
        if (st != STRIDE_OK) return st;
        st = check_rows("v", v, v_tok, v_head, c.dtype);
        if (st != STRIDE_OK) return st;
        if (n_heads_q > 0) {
            st = check_rows("q", q, q_tok, q_head, c.dtype);
            if (st != STRIDE_OK) return st;
            st = check_rows("q_out", q_out, qo_tok, qo_head, c.dtype);
            if (st != STRIDE_OK) return st;
        }
    }
    AppendArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.q_out = q_out;
    a.k_cache = c.k;
    a.v_cache = c.v;
    a.seq = seq;
    a.slot = slot;
    a.pos = pos;
    a.page_table = c.page_table;
    a.rope = rope;
    a.flags = dev_flags;
    a.q_tok = q_tok;
    a.q_head = q_head;
    a.qo_tok = qo_tok;
    a.qo_head = qo_head;
    a.k_tok = k_tok;
    a.k_head = k_head;
    a.v_tok = v_tok;
    a.v_head = v_head;
    a.k_page = c.k_page;
    a.k_slot = c.k_slot;
    a.k_chead = c.k_head;
    a.v_page = c.v_page;
    a.v_slot = c.v_slot;
    a.v_chead = c.v_head;
    a.table_ld = c.table_ld;
    a.n_pages = c.n_pages;
    a.n_heads_q = n_heads_q;
    a.n_heads = c.n_heads;
    a.head_dim = c.head_dim;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.n_seqs = c.n_seqs;
    a.max_pages = c.max_pages;
    a.max_pos = max_pos;
    a.rot = rot;
    a.eps = eps;
    const hipError_t e = launch_kv_append(a, c.dtype, n_tokens, rope_style, stream);
    if (e != hipSuccess) return hip_fail(e, "cache append launch");
    return ok();
}

size_t stride_attention_workspace_size(const stride_kv_cache *cache, int64_t n_q, int32_t n_heads_q) {
    if (check_cache_sizes(cache) != STRIDE_OK || check_attention_sizes(*cache, n_q, n_heads_q) != STRIDE_OK) return 0;
    return attention_ws_bytes(*cache, n_q, n_heads_q);
}

stride_status stride_tree_attention(const stride_kv_cache *cache, int64_t n_q, int32_t n_heads_q,
                                    const void *q, int64_t q_tok, int64_t q_head, const int32_t *q_off,
                                    const int32_t *ctx_len, const uint64_t *tree_mask, int32_t mask_words,
                                    float scale, void *out, int64_t out_tok, int64_t out_head, float *lse,
                                    uint32_t *dev_flags, void *ws, size_t ws_bytes, hipStream_t stream) {
    stride_status st = check_cache(cache);
    if (st != STRIDE_OK) return st;
    const stride_kv_cache &c = *cache;
    st = check_attention_sizes(c, n_q, n_heads_q);
    if (st != STRIDE_OK) return st;
    if (!(scale > 0.0f && scale < INFINITY)) return fail(STRIDE_ERR_INVALID_ARG, "scale = %g is not > 0", (double)scale);
    if (tree_mask && mask_words < 1) return fail(STRIDE_ERR_INVALID_ARG, "mask_words = %d < 1", mask_words);
    if (c.n_seqs > 0 && (!q_off || !ctx_len)) return fail(STRIDE_ERR_INVALID_ARG, "q_off or ctx_len is NULL");
    if (n_q > 0) {
        st = check_rows("q", q, q_tok, q_head, c.dtype);
        if (st != STRIDE_OK) return st;
        st = check_rows("out", out, out_tok, out_head, c.dtype);
        if (st != STRIDE_OK) return st;
    }
    st = check_ws(attention_ws_bytes(c, n_q, n_heads_q), ws, ws_bytes);
    if (st != STRIDE_OK) return st;
    const hipError_t e = launch_tree_attention(c, n_q, n_heads_q, q, q_tok, q_head, q_off, ctx_len, tree_mask,
                                               mask_words, scale, out, out_tok, out_head, lse, dev_flags, ws,
                                               stream);
    if (e != hipSuccess) return hip_fail(e, "attention launch");
    return ok();
}

size_t stride_sample_workspace_size(int64_t n_rows, int32_t vocab) {
    if (n_rows < 0 || vocab < 1 || vocab > kMaxVocab) return 0;
    return sample_ws_bytes(n_rows, vocab);
}

stride_status stride_sample(int64_t n_rows, int32_t vocab, int64_t ld, int32_t dtype, const void *logits,
                            const float *noise, int64_t noise_ld, const float *temperature,
                            const int32_t *top_k, const float *top_p, const float *min_p,
                            int32_t *token_ids, uint32_t *dev_flags, void *ws, size_t ws_bytes,
                            hipStream_t stream) {
    if (n_rows < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_rows = %lld < 0", (long long)n_rows);
    if (vocab < 1) return fail(STRIDE_ERR_INVALID_ARG, "vocab = %d < 1", vocab);
    if (vocab > kMaxVocab) return fail(STRIDE_ERR_UNSUPPORTED, "vocab = %d passes 2^30", vocab);
    if (ld < vocab) return fail(STRIDE_ERR_INVALID_ARG, "ld = %lld < vocab = %d", (long long)ld, vocab);
    if (dtype != STRIDE_BF16 && dtype != STRIDE_F32)
        return fail(STRIDE_ERR_UNSUPPORTED, "dtype %d is neither STRIDE_BF16 nor STRIDE_F32", dtype);
    if (!whole_words(ld, dtype))
        return fail(STRIDE_ERR_UNSUPPORTED, "row stride of %lld elements is not a multiple of 16 bytes", (long long)ld);
    if (n_rows > 0) {
        if (!logits || !token_ids) return fail(STRIDE_ERR_INVALID_ARG, "logits or token_ids is NULL");
        if (!aligned(logits, 16)) return fail(STRIDE_ERR_UNSUPPORTED, "logits is not 16-byte aligned");
        if (temperature) {
            if (!noise) return fail(STRIDE_ERR_INVALID_ARG, "temperature given without noise");
            if (noise_ld < vocab)
                return fail(STRIDE_ERR_INVALID_ARG, "noise_ld = %lld < vocab = %d", (long long)noise_ld, vocab);
            if (noise_ld % 4 != 0 || !aligned(noise, 16))
                return fail(STRIDE_ERR_UNSUPPORTED, "noise rows must be 16-byte aligned");
        }
    }
    const stride_status st = check_ws(sample_ws_bytes(n_rows, vocab), ws, ws_bytes);
    if (st != STRIDE_OK) return st;
    const hipError_t e = launch_sample(n_rows, vocab, ld, dtype, logits, noise, noise_ld, temperature, top_k,
                                       top_p, min_p, token_ids, dev_flags, ws, stream);
    if (e != hipSuccess) return hip_fail(e, "sampling launch");
    return ok();
}

stride_status stride_probe_read(const void *a, const void *b, int64_t n_rows, int64_t row_bytes,
                                int64_t read_bytes, uint32_t *sink, hipStream_t stream) {
    if (n_rows < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_rows = %lld < 0", (long long)n_rows);
    if (n_rows == 0) return ok();
    if (!a || !sink) return fail(STRIDE_ERR_INVALID_ARG, "a or sink is NULL");
    if (read_bytes < 16 || read_bytes > row_bytes)
        return fail(STRIDE_ERR_INVALID_ARG, "read_bytes = %lld outside [16, row_bytes = %lld]",
                    (long long)read_bytes, (long long)row_bytes);
    if (row_bytes % 16 != 0 || !aligned(a, 16) || (b && !aligned(b, 16)))
        return fail(STRIDE_ERR_UNSUPPORTED, "rows must be 16-byte aligned");
    hipError_t e = launch_probe_read(a, b, n_rows, row_bytes, read_bytes, sink, stream);
    if (e != hipSuccess) return hip_fail(e, "probe launch");
    return ok();
}

stride_status stride_probe_read_flat(const void *a, const void *b, int64_t n_bytes, uint32_t *sink,
                                     int64_t sink_len, hipStream_t stream) {
    if (n_bytes < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_bytes = %lld < 0", (long long)n_bytes);
    if (n_bytes == 0) return ok();
    if (!a || !sink) return fail(STRIDE_ERR_INVALID_ARG, "a or sink is NULL");
    if (sink_len < 4) return fail(STRIDE_ERR_INVALID_ARG, "sink_len = %lld < 4", (long long)sink_len);
    if (n_bytes % 16 != 0 || !aligned(a, 16) || (b && !aligned(b, 16)))
        return fail(STRIDE_ERR_UNSUPPORTED, "ranges must be 16-byte aligned multiples of 16 bytes");
    hipError_t e = launch_probe_flat(a, b, n_bytes, sink, sink_len, stream);
    if (e != hipSuccess) return hip_fail(e, "probe launch");
    return ok();
}

stride_status stride_probe_copy(const void *src, void *dst, const uint8_t *row_mask, int64_t n_rows,
                                int64_t row_bytes, int64_t copy_bytes, hipStream_t stream) {
    if (n_rows < 0) return fail(STRIDE_ERR_INVALID_ARG, "n_rows = %lld < 0", (long long)n_rows);
    if (n_rows == 0) return ok();
    if (!src || !dst) return fail(STRIDE_ERR_INVALID_ARG, "src or dst is NULL");
    if (copy_bytes < 16 || copy_bytes > row_bytes)
        return fail(STRIDE_ERR_INVALID_ARG, "copy_bytes = %lld outside [16, row_bytes = %lld]",
                    (long long)copy_bytes, (long long)row_bytes);
    if (row_bytes % 16 != 0 || !aligned(src, 16) || !aligned(dst, 16))
        return fail(STRIDE_ERR_UNSUPPORTED, "rows must be 16-byte aligned");
    hipError_t e = launch_probe_copy(src, dst, row_mask, n_rows, row_bytes, copy_bytes, stream);
    if (e != hipSuccess) return hip_fail(e, "probe launch");
    return ok();
}

}  // extern "C"
