// C-ABI of libstc: host-side argument validation and dispatch.  Nothing here
// allocates device memory; every launch goes to the caller's stream.
#include <nvtx3/nvToolsExt.h>

#include <cmath>

#include "common.cuh"

using namespace stc;

namespace {

int32_t make_geom(const stc_shape* s, Geom* g) {
    if (!s) return STC_ERR_INVALID_ARG;
    if (s->batch < 0 || s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->t_cap < 0 || s->reserved != 0)
        return STC_ERR_INVALID_ARG;
    if (s->n_q_heads % s->n_kv_heads != 0) return STC_ERR_INVALID_ARG;
    if (s->head_dim != kHeadDim || s->page_size != kPage) return STC_ERR_UNSUPPORTED;
    if (s->n_groups != 4 && s->n_groups != 8 && s->n_groups != 16) return STC_ERR_UNSUPPORTED;
    if (s->n_q_heads / s->n_kv_heads > 8) return STC_ERR_UNSUPPORTED;
    if ((int64_t)s->t_cap * 16 >= (int64_t)1 << 31) return STC_ERR_UNSUPPORTED;   // u32 offsets
    if ((int64_t)s->batch * s->n_kv_heads >= (int64_t)1 << 24) return STC_ERR_UNSUPPORTED;
    g->B = s->batch; g->Hq = s->n_q_heads; g->Hkv = s->n_kv_heads; g->Gq = g->Hq / g->Hkv;
    g->S = s->n_groups; g->g = kHeadDim / g->S; g->T = s->t_cap; g->P = (g->T + kPage - 1) / kPage;
    g->problems = g->B * g->Hkv;
    g->seq_len = s->seq_len;
    return STC_OK;
}

bool empty(const Geom& g) { return g.problems == 0 || g.T == 0; }

int32_t check_ws(const void* ws, size_t have, size_t need) {
    if (need == 0) return STC_OK;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || have < need) return STC_ERR_WORKSPACE;
    return STC_OK;
}

int32_t cuda_rc(cudaError_t e) { return e == cudaSuccess ? STC_OK : STC_ERR_CUDA; }

// NVTX range around the host side of a call (what it enqueues shows under it in a timeline).
struct Range {
    explicit Range(const char* name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

}  // namespace

namespace {
// The kernels move keys, values, queries, page metadata and scores in 16-byte pieces.
template <typename... P>
bool aligned16(P... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) == 0; }
}  // namespace

extern "C" {

const char* stc_status_string(int32_t status) {
    switch (status) {
        case STC_OK: return "ok";
        case STC_ERR_INVALID_ARG: return "invalid argument";
        case STC_ERR_UNSUPPORTED: return "unsupported shape";
        case STC_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case STC_ERR_CAPACITY: return "packed value store too small";
        case STC_ERR_BUDGET: return "group budget below one group per routed token";
        case STC_ERR_CUDA: return "CUDA runtime error";
        case STC_ERR_TIMEOUT: return "timeout";
        case STC_ERR_SCRATCH_LIMIT: return "shape needs more than the built-in scratch array";
        default: return "unknown status";
    }
}

int32_t stc_version(void) { return 100; }

int32_t stc_workspace_bytes(const stc_shape* shape, int32_t op, int64_t arg, size_t* bytes_host) {
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!bytes_host) return STC_ERR_INVALID_ARG;
    if (op == STC_OP_PREFIX_ATTN) {                 // rows have outputs even where the prefixes have no tokens
        if (arg < 0 || arg > 0x7FFFFFFF) return STC_ERR_INVALID_ARG;
        *bytes_host = g.problems == 0 || arg == 0 ? 0 : prefix_ws_bytes(g);
        return STC_OK;
    }
    if (op == STC_OP_TREE_ATTN) {                   // nodes attend their ancestors even where the cache has no tokens
        if (arg < 0 || arg > STC_TREE_MAX_NODES) return STC_ERR_INVALID_ARG;
        *bytes_host = g.problems == 0 || arg == 0 ? 0 : tree_attn_ws_bytes();
        return STC_OK;
    }
    if (empty(g)) { *bytes_host = 0; return STC_OK; }
    switch (op) {
        case STC_OP_QUEST_SELECT: *bytes_host = select_ws_bytes(g); break;
        case STC_OP_ROUTE_PACK: *bytes_host = route_ws_bytes(g); break;
        case STC_OP_DECODE_ATTN:
            if (arg < 0 || arg > g.P) return STC_ERR_INVALID_ARG;
            *bytes_host = attn_ws_bytes(g, (int)arg);
            break;
        default: return STC_ERR_INVALID_ARG;
    }
    return STC_OK;
}

int32_t stc_build_page_meta(const stc_shape* shape, const stc_cache* cache, int32_t page_begin,
                            int32_t page_end, void* stream) {
    Range nvtx_range("stc_build_page_meta");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!cache->k || !cache->kmin || !cache->kmax || page_begin < 0) return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->kmin, cache->kmax)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_page_meta(g, cache->k, cache->kmin, cache->kmax, page_begin, page_end,
                                    static_cast<cudaStream_t>(stream)));
}

int32_t stc_quest_select(const stc_shape* shape, const stc_cache* cache, const void* q,
                         int32_t token_budget, int32_t max_pages, int32_t* page_ids,
                         int32_t* n_pages, float* scores_opt, void* ws, size_t ws_bytes,
                         void* stream) {
    return stc_quest_select_window(shape, cache, q, token_budget, 0, max_pages, page_ids, n_pages, scores_opt, ws,
                                   ws_bytes, stream);
}

int32_t stc_quest_select_window(const stc_shape* shape, const stc_cache* cache, const void* q,
                                int32_t token_budget, int32_t n_recent_pages, int32_t max_pages,
                                int32_t* page_ids, int32_t* n_pages, float* scores_opt, void* ws,
                                size_t ws_bytes, void* stream) {
    Range nvtx_range("stc_quest_select_window");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || token_budget < 0 || max_pages < 0 || n_recent_pages < 0) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!cache->kmin || !cache->kmax || !q || !page_ids || !n_pages) return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->kmin, cache->kmax, q)) return STC_ERR_INVALID_ARG;
    const int want = token_budget / kPage < g.P ? token_budget / kPage : g.P;
    if (max_pages < want) return STC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, select_ws_bytes(g));
    if (rc != STC_OK) return rc;
    return cuda_rc(launch_quest_select(g, cache->kmin, cache->kmax, q, token_budget, n_recent_pages, max_pages,
                                       page_ids, n_pages, scores_opt, ws,
                                       static_cast<cudaStream_t>(stream)));
}

int32_t stc_pages_to_class(const stc_shape* shape, const int32_t* page_ids, const int32_t* n_pages,
                           int32_t max_pages, uint8_t* tok_class, void* stream) {
    Range nvtx_range("stc_pages_to_class");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (max_pages < 0) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!tok_class || (max_pages > 0 && (!page_ids || !n_pages))) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_pages_to_class(g, page_ids, n_pages, max_pages, tok_class,
                                         static_cast<cudaStream_t>(stream)));
}

namespace {
int32_t route_pack_phases(const stc_shape* shape, const void* v, const float* scores,
                          const uint8_t* tok_class, int64_t class_head_stride, int32_t k_nominal,
                          int32_t min_per_token, int32_t mode, const stc_cache* out,
                          int64_t* total_groups, int32_t* status, void* ws, size_t ws_bytes, int phases,
                          void* stream) {
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!out || k_nominal < 0 || k_nominal > g.S || (min_per_token != 0 && min_per_token != 1) ||
        (mode != STC_MODE_GLOBAL && mode != STC_MODE_PER_TOKEN))
        return STC_ERR_INVALID_ARG;
    if (class_head_stride != 0 && class_head_stride != g.T) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!out->v_mask) return STC_ERR_INVALID_ARG;
    if ((phases & 1) && (!scores || !aligned16(scores))) return STC_ERR_INVALID_ARG;
    if ((phases & 2) && !aligned16(v, out->v_packed)) return STC_ERR_INVALID_ARG;
    if ((phases & 2) && (!v || !out->v_packed || !out->v_offs || !total_groups || !status || out->cap_groups < 0))
        return STC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, route_ws_bytes(g));
    if (rc != STC_OK) return rc;
    return cuda_rc(launch_route_pack(g, v, scores, tok_class, class_head_stride, k_nominal,
                                     min_per_token, mode, out->v_packed, out->v_mask, out->v_offs,
                                     out->cap_groups, total_groups, status, ws, phases,
                                     static_cast<cudaStream_t>(stream)));
}
}  // namespace

int32_t stc_route_pack(const stc_shape* shape, const void* v, const float* scores,
                       const uint8_t* tok_class, int64_t class_head_stride, int32_t k_nominal,
                       int32_t min_per_token, int32_t mode, const stc_cache* out,
                       int64_t* total_groups, int32_t* status, void* ws, size_t ws_bytes,
                       void* stream) {
    Range nvtx_range("stc_route_pack");
    return route_pack_phases(shape, v, scores, tok_class, class_head_stride, k_nominal, min_per_token, mode,
                             out, total_groups, status, ws, ws_bytes, 3, stream);
}

int32_t stc_route_mask(const stc_shape* shape, const float* scores, const uint8_t* tok_class,
                       int64_t class_head_stride, int32_t k_nominal, int32_t min_per_token, int32_t mode,
                       const stc_cache* out, void* ws, size_t ws_bytes, void* stream) {
    Range nvtx_range("stc_route_mask");
    return route_pack_phases(shape, nullptr, scores, tok_class, class_head_stride, k_nominal, min_per_token,
                             mode, out, nullptr, nullptr, ws, ws_bytes, 1, stream);
}

int32_t stc_pack_values(const stc_shape* shape, const void* v, int32_t mode, const stc_cache* out,
                        int64_t* total_groups, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
    Range nvtx_range("stc_pack_values");
    return route_pack_phases(shape, v, nullptr, nullptr, 0, 0, 0, mode, out, total_groups, status, ws,
                             ws_bytes, 2, stream);
}

int32_t stc_router_logits(const stc_shape* shape, const void* h, const void* w, const float* bias_opt,
                          int32_t d_model, float* scores, int32_t* status_word, void* stream) {
    Range nvtx_range("stc_router_logits");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (d_model <= 0) return STC_ERR_INVALID_ARG;
    const int n = g.Hkv * g.S;
    if (d_model % 64 != 0 || n % 16 != 0 || (n > 256 && n % 256 != 0)) return STC_ERR_UNSUPPORTED;
    if (empty(g)) return STC_OK;
    if (!h || !w || !scores || !status_word) return STC_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(h) | reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(scores) |
          reinterpret_cast<uintptr_t>(bias_opt)) & 15u) != 0)
        return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_router_logits(g, h, w, bias_opt, d_model, scores, status_word,
                                        static_cast<cudaStream_t>(stream)));
}

int32_t stc_query_bias(int32_t batch, int32_t q_cap, int32_t d_model, int32_t n_logits, const void* h_q,
                       const int32_t* q_len_opt, const void* w_q, float* s_q, float* bias, void* stream) {
    Range nvtx_range("stc_query_bias");
    if (batch < 0 || q_cap < 0 || d_model <= 0 || n_logits < 0 || batch > 65535) return STC_ERR_INVALID_ARG;
    if (d_model % 8 != 0) return STC_ERR_UNSUPPORTED;
    if (batch == 0) return STC_OK;
    if (!s_q || (n_logits > 0 && (!w_q || !bias)) || (q_cap > 0 && !h_q)) return STC_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(h_q) | reinterpret_cast<uintptr_t>(w_q) | reinterpret_cast<uintptr_t>(s_q)) & 15u) != 0)
        return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_query_bias(batch, q_cap, d_model, n_logits, h_q, q_len_opt, w_q, s_q, bias,
                                     static_cast<cudaStream_t>(stream)));
}

int32_t stc_append_tokens(const stc_shape* shape, const stc_cache* cache, const void* v,
                          const int32_t* old_len, int32_t max_new, int64_t* total_groups, int32_t* status,
                          void* stream) {
    Range nvtx_range("stc_append_tokens");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || max_new < 0) return STC_ERR_INVALID_ARG;
    if (empty(g) || max_new == 0) return STC_OK;
    if (!cache->k || !cache->kmin || !cache->kmax || !cache->v_packed || !cache->v_mask || !cache->v_offs ||
        cache->cap_groups < 0 || !v || !old_len || !total_groups || !status)
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->kmin, cache->kmax, cache->v_packed, v)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_append(g, cache->k, cache->kmin, cache->kmax, v, old_len, max_new, cache->v_packed,
                                 cache->v_mask, cache->v_offs, cache->cap_groups, total_groups, status,
                                 static_cast<cudaStream_t>(stream)));
}

int32_t stc_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                             double low, double high, double* inv_freq_host, float* scale_host) {
    if (rot_dim < 0 || rot_dim > kHeadDim || !inv_freq_host || !scale_host || !(base > 1.0) || !std::isfinite(base))
        return STC_ERR_INVALID_ARG;
    if (rot_dim % 16 != 0) return STC_ERR_UNSUPPORTED;
    if (scaling < STC_ROPE_NONE || scaling > STC_ROPE_YARN) return STC_ERR_INVALID_ARG;
    if (scaling != STC_ROPE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return STC_ERR_INVALID_ARG;
    if (scaling >= STC_ROPE_BANDS && !(original_len > 0.0 && low > 0.0 && high > low && std::isfinite(original_len) &&
                                       std::isfinite(high)))
        return STC_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    // pair (as a real number) that makes `turns` turns over the original context
    auto pair_of = [&](double turns) {
        return rot_dim * std::log(original_len / (turns * two_pi)) / (2.0 * std::log(base));
    };
    double lo = 0.0, hi = 0.0;
    if (scaling == STC_ROPE_YARN) {
        lo = std::fmax(std::floor(pair_of(high)), 0.0);
        hi = std::fmin(std::ceil(pair_of(low)), rot_dim - 1.0);
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double keep = 1.0;                          // share of the unscaled frequency; the rest is divided by factor
        if (scaling == STC_ROPE_LINEAR) keep = 0.0;
        if (scaling == STC_ROPE_BANDS) {
            const double turns = original_len * f / two_pi;
            keep = std::fmin(std::fmax((turns - low) / (high - low), 0.0), 1.0);
        }
        if (scaling == STC_ROPE_YARN)
            keep = 1.0 - std::fmin(std::fmax((i - lo) / std::fmax(hi - lo, 1e-3), 0.0), 1.0);
        inv_freq_host[i] = keep * f + (1.0 - keep) * f / factor;
    }
    *scale_host = scaling == STC_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return STC_OK;
}

int32_t stc_rope_write(const stc_shape* shape, const stc_rope* rope, const int32_t* old_len, int32_t max_new,
                       const int32_t* positions_opt, const void* q_in, int64_t q_stride, const void* k_in,
                       int64_t k_stride, const void* v_in, int64_t v_stride, void* q_out, void* k, void* v,
                       int32_t* status, void* stream) {
    Range nvtx_range("stc_rope_write");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!rope || max_new < 0 || rope->rot_dim < 0 || rope->rot_dim > kHeadDim || rope->reserved != 0 ||
        (rope->interleaved != 0 && rope->interleaved != 1))
        return STC_ERR_INVALID_ARG;
    if (rope->rot_dim % 16 != 0) return STC_ERR_UNSUPPORTED;
    if (empty(g) || max_new == 0) return STC_OK;
    if (!old_len || !status || (rope->rot_dim > 0 && !rope->inv_freq)) return STC_ERR_INVALID_ARG;
    if ((!q_in) != (!q_out) || (!k_in) != (!k) || (!v_in) != (!v) || (!q_in && !k_in && !v_in))
        return STC_ERR_INVALID_ARG;
    if (!aligned16(q_in, q_out, k_in, k, v_in, v) || (reinterpret_cast<uintptr_t>(rope->inv_freq) & 7u) != 0)
        return STC_ERR_INVALID_ARG;
    auto stride_ok = [&](const void* in, int64_t stride, int heads) {
        return !in || (stride >= (int64_t)heads * kHeadDim && stride % 8 == 0 && stride < ((int64_t)1 << 40));
    };
    if (!stride_ok(q_in, q_stride, g.Hq) || !stride_ok(k_in, k_stride, g.Hkv) || !stride_ok(v_in, v_stride, g.Hkv))
        return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_rope_write(g, *rope, old_len, max_new, positions_opt, q_in, q_stride, k_in, k_stride,
                                     v_in, v_stride, q_out, k, v, status, static_cast<cudaStream_t>(stream)));
}

int32_t stc_route_new_pages(const stc_shape* shape, const stc_cache* cache, const float* scores,
                            const int32_t* first_page, int32_t k_nominal, int32_t min_per_token,
                            int32_t mode, int64_t* total_groups, int32_t* status, void* stream) {
    Range nvtx_range("stc_route_new_pages");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || k_nominal < 0 || k_nominal > g.S || (min_per_token != 0 && min_per_token != 1) ||
        (mode != STC_MODE_GLOBAL && mode != STC_MODE_PER_TOKEN))
        return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!cache->v_packed || !cache->v_mask || !cache->v_offs || cache->cap_groups < 0 || !scores || !first_page ||
        !total_groups || !status)
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->v_packed, scores)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_route_new_pages(g, scores, first_page, k_nominal, min_per_token, mode, cache->v_packed,
                                          cache->v_mask, cache->v_offs, cache->cap_groups, total_groups, status,
                                          static_cast<cudaStream_t>(stream)));
}

namespace {
// Checked options of the scored calls; *plain = nothing is set and the call is the unscored one.
int32_t score_args(const stc_score* score, float sm_scale, ScoreArgs* out, bool* plain) {
    *out = ScoreArgs{};
    *plain = true;
    if (!score) return STC_OK;
    if (!(score->softcap >= 0.f) || !std::isfinite(score->softcap) || score->window < 0) return STC_ERR_INVALID_ARG;
    // the kernels multiply by sm_scale / softcap (a subnormal one has lost bits) and by softcap log2(e)
    if (score->softcap > 0.f) {
        const float in = sm_scale / score->softcap;
        if (!(std::isnormal(in) || sm_scale == 0.f) || !std::isfinite(score->softcap * 1.4426950408889634f)) return STC_ERR_INVALID_ARG;
    }
    if ((!score->tok_doc) != (!score->q_doc)) return STC_ERR_INVALID_ARG;
    out->softcap = score->softcap; out->window = score->window; out->slopes = score->slopes;
    out->q_pos = score->q_pos; out->tok_doc = score->tok_doc; out->q_doc = score->q_doc;
    *plain = score->softcap == 0.f && score->window == 0 && !score->slopes && !score->q_pos && !score->tok_doc;
    return STC_OK;
}

int32_t decode_attn(const stc_shape* shape, const stc_cache* cache, const void* q, const int32_t* page_ids,
                    const int32_t* n_pages, int32_t max_pages, float sm_scale, const stc_score* score, float* out,
                    float* lse_opt, void* ws, size_t ws_bytes, void* stream) {
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || max_pages < 0 || !(sm_scale == sm_scale)) return STC_ERR_INVALID_ARG;
    ScoreArgs sc;
    bool plain;
    rc = score_args(score, sm_scale, &sc, &plain);
    if (rc != STC_OK) return rc;
    if (g.problems == 0) return STC_OK;
    if (!q || !out) return STC_ERR_INVALID_ARG;
    if (page_ids && !n_pages) return STC_ERR_INVALID_ARG;
    if (!page_ids) max_pages = g.P;
    if (max_pages > g.P && !page_ids) return STC_ERR_INVALID_ARG;
    if (g.T > 0 && (!cache->k || !cache->v_packed || !cache->v_mask || !cache->v_offs || cache->cap_groups < 0))
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->v_packed, q, out)) return STC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, attn_ws_bytes(g, max_pages));
    if (rc != STC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_rc(plain ? launch_decode_attn(g, cache->k, cache->v_packed, cache->v_mask, cache->v_offs, cache->cap_groups,
                                              q, page_ids, n_pages, max_pages, sm_scale, out, lse_opt, ws, st)
                         : launch_scored_attn(g, cache->k, cache->v_packed, cache->v_mask, cache->v_offs, cache->cap_groups,
                                              q, page_ids, n_pages, max_pages, sm_scale, sc, out, lse_opt, ws, st));
}
}  // namespace

int32_t stc_decode_attn(const stc_shape* shape, const stc_cache* cache, const void* q,
                        const int32_t* page_ids, const int32_t* n_pages, int32_t max_pages,
                        float sm_scale, float* out, float* lse_opt, void* ws, size_t ws_bytes,
                        void* stream) {
    Range nvtx_range("stc_decode_attn");
    return decode_attn(shape, cache, q, page_ids, n_pages, max_pages, sm_scale, nullptr, out, lse_opt, ws, ws_bytes,
                       stream);
}

int32_t stc_decode_attn_scored(const stc_shape* shape, const stc_cache* cache, const void* q,
                               const int32_t* page_ids, const int32_t* n_pages, int32_t max_pages,
                               float sm_scale, const stc_score* score, float* out, float* lse_opt, void* ws,
                               size_t ws_bytes, void* stream) {
    Range nvtx_range("stc_decode_attn_scored");
    return decode_attn(shape, cache, q, page_ids, n_pages, max_pages, sm_scale, score, out, lse_opt, ws, ws_bytes,
                       stream);
}

int32_t stc_prefix_attn(const stc_shape* shape, const stc_cache* cache, int32_t n_rows, const void* q,
                        const int32_t* row_start, float sm_scale, const stc_score* score, const float* own_out,
                        const float* own_lse, float* out, float* lse_opt, void* ws, size_t ws_bytes, void* stream) {
    Range nvtx_range("stc_prefix_attn");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || n_rows < 0 || !(sm_scale == sm_scale)) return STC_ERR_INVALID_ARG;
    ScoreArgs sc;
    bool plain;
    rc = score_args(score, sm_scale, &sc, &plain);
    if (rc != STC_OK) return rc;
    if ((sc.slopes || sc.window > 0) && !sc.q_pos) return STC_ERR_INVALID_ARG;    // no position to count from
    if ((int64_t)g.problems * g.T > 0x7FFFFFFFLL || (int64_t)n_rows * g.Hq > 0x7FFFFFFFLL) return STC_ERR_UNSUPPORTED;
    if (g.problems == 0 || n_rows == 0) return STC_OK;
    if (!q || !row_start || !out || (!own_out) != (!own_lse)) return STC_ERR_INVALID_ARG;
    if (own_out == out || (own_lse && own_lse == lse_opt)) return STC_ERR_INVALID_ARG;
    if (g.T > 0 && (!cache->k || !cache->v_packed || !cache->v_mask || !cache->v_offs || cache->cap_groups < 0))
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->v_packed, q, own_out, out)) return STC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, prefix_ws_bytes(g));
    if (rc != STC_OK) return rc;
    return cuda_rc(launch_prefix_attn(g, cache->k, cache->v_packed, cache->v_mask, cache->v_offs, cache->cap_groups,
                                      n_rows, q, row_start, sm_scale, plain ? nullptr : &sc, own_out, own_lse, out,
                                      lse_opt, ws, static_cast<cudaStream_t>(stream)));
}

namespace {
int32_t check_tree(const stc_tree* t) {
    if (!t || t->reserved != 0 || t->n_cap < 1 || t->n_cap > STC_TREE_MAX_NODES) return STC_ERR_INVALID_ARG;
    return STC_OK;
}
bool complete(const stc_cache* c) { return c->k && c->v_packed && c->v_mask && c->v_offs && c->cap_groups >= 0 && (!c->kmin) == (!c->kmax); }
bool aligned(const stc_cache* c) { return aligned16(c->k, c->v_packed, c->kmin, c->kmax); }
}  // namespace

int32_t stc_tree_attn(const stc_shape* shape, const stc_cache* cache, const stc_tree* tree, const void* q,
                      const int32_t* page_ids, const int32_t* n_pages, int32_t max_pages, float sm_scale,
                      const stc_score* score, float* out, float* lse_opt, int32_t* status, void* ws, size_t ws_bytes,
                      void* stream) {
    Range nvtx_range("stc_tree_attn");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc == STC_OK) rc = check_tree(tree);
    if (rc != STC_OK) return rc;
    if (!cache || max_pages < 0 || !(sm_scale == sm_scale)) return STC_ERR_INVALID_ARG;
    ScoreArgs sc;
    bool plain;
    rc = score_args(score, sm_scale, &sc, &plain);
    if (rc != STC_OK) return rc;
    if ((int64_t)g.problems * g.T > 0x7FFFFFFFLL || (int64_t)g.B * tree->n_cap * g.Hq > 0x7FFFFFFFLL)
        return STC_ERR_UNSUPPORTED;
    // tiles of the call, counted in 32 bits: eight pages each, for every block of at least 32 / 8 nodes
    const int64_t most_pages = page_ids && max_pages > g.P ? max_pages : g.P;
    if ((int64_t)g.problems * (most_pages / 8 + 2) > 0x7FFFFFFFLL / ((tree->n_cap + 3) / 4)) return STC_ERR_UNSUPPORTED;
    if (g.problems == 0) return STC_OK;
    if (!q || !out || !status || !tree->k || !tree->v || (page_ids && !n_pages)) return STC_ERR_INVALID_ARG;
    if (g.T > 0 && (!cache->k || !cache->v_packed || !cache->v_mask || !cache->v_offs || cache->cap_groups < 0))
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->v_packed, q, out, tree->k, tree->v)) return STC_ERR_INVALID_ARG;
    rc = check_ws(ws, ws_bytes, tree_attn_ws_bytes());
    if (rc != STC_OK) return rc;
    return cuda_rc(launch_tree_attn(g, *cache, *tree, q, page_ids, n_pages, max_pages, sm_scale, sc, out, lse_opt, status, ws,
                                    static_cast<cudaStream_t>(stream)));
}

int32_t stc_tree_accept(int32_t batch, int32_t n_cap, int32_t vocab, const void* logits, int32_t logits_type,
                        int64_t row_stride, const int32_t* tokens, const int32_t* parent, const int32_t* n_nodes_opt,
                        int32_t* path, int32_t* n_accepted, int32_t* next_token, void* stream) {
    Range nvtx_range("stc_tree_accept");
    if (batch < 0 || n_cap < 1 || n_cap > STC_TREE_MAX_NODES || vocab < 1 || row_stride < vocab ||
        row_stride >= (int64_t)1 << 40 || (logits_type != STC_LOGITS_BF16 && logits_type != STC_LOGITS_F32))
        return STC_ERR_INVALID_ARG;
    if (batch >= 1 << 24) return STC_ERR_UNSUPPORTED;
    if (batch == 0) return STC_OK;
    if (!logits || !tokens || !path || !n_accepted || !next_token) return STC_ERR_INVALID_ARG;
    const bool bf16 = logits_type == STC_LOGITS_BF16;
    if ((reinterpret_cast<uintptr_t>(logits) & (bf16 ? 1u : 3u)) != 0) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_tree_accept(batch, n_cap, vocab, logits, bf16, row_stride, tokens, parent, n_nodes_opt, path, n_accepted,
                                      next_token, static_cast<cudaStream_t>(stream)));
}

int32_t stc_tree_commit(const stc_shape* shape, const stc_cache* cache, const stc_tree* tree, const int32_t* path,
                        const int32_t* n_accepted, int32_t* new_len, int64_t* total_groups, int32_t* status,
                        void* stream) {
    Range nvtx_range("stc_tree_commit");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc == STC_OK) rc = check_tree(tree);
    if (rc != STC_OK) return rc;
    if (!cache) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    if (!complete(cache) || !tree->k || !tree->v || !path || !n_accepted || !new_len || !total_groups || !status ||
        new_len == g.seq_len)
        return STC_ERR_INVALID_ARG;
    if (!aligned(cache) || !aligned16(tree->k, tree->v)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_tree_commit(g, *tree, path, n_accepted, const_cast<void*>(cache->k), cache->kmin, cache->kmax,
                                      cache->v_packed, cache->v_mask, cache->v_offs, cache->cap_groups, new_len, total_groups,
                                      status, static_cast<cudaStream_t>(stream)));
}

int32_t stc_cache_fork(const stc_shape* src_shape, const stc_cache* src, const stc_shape* dst_shape, const stc_cache* dst,
                       int32_t n_pairs, const int32_t* src_row, const int32_t* dst_row, int32_t* new_len,
                       int64_t* total_groups, int32_t* status, void* stream) {
    Range nvtx_range("stc_cache_fork");
    Geom gs, gd;
    int32_t rc = make_geom(src_shape, &gs);
    if (rc == STC_OK) rc = make_geom(dst_shape, &gd);
    if (rc != STC_OK) return rc;
    if (!src || !dst || n_pairs < 0 || gs.Hkv != gd.Hkv || gs.Hq != gd.Hq || gs.S != gd.S) return STC_ERR_INVALID_ARG;
    if (n_pairs > 4096 || gs.Hkv > 65535) return STC_ERR_UNSUPPORTED;
    if (n_pairs == 0 || empty(gs) || empty(gd)) return STC_OK;
    if (!complete(src) || !complete(dst) || !src_row || !dst_row || !new_len || !total_groups || !status || new_len == gs.seq_len ||
        (dst->kmin && !src->kmin))
        return STC_ERR_INVALID_ARG;
    if (src->k == dst->k && (gs.B != gd.B || gs.T != gd.T || src->v_packed != dst->v_packed || src->v_mask != dst->v_mask ||
                             src->v_offs != dst->v_offs || src->cap_groups != dst->cap_groups))
        return STC_ERR_INVALID_ARG;
    if (!aligned(src) || !aligned(dst)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_cache_fork(gs, *src, gd, *dst, n_pairs, src_row, dst_row, new_len, total_groups, status,
                                     static_cast<cudaStream_t>(stream)));
}

int32_t stc_cache_compact(const stc_shape* src_shape, const stc_cache* src, const int32_t* page_ids,
                          const int32_t* n_pages, int32_t max_pages, const stc_shape* dst_shape, const stc_cache* dst,
                          int32_t* new_len, int64_t* total_groups, int32_t* status, void* stream) {
    Range nvtx_range("stc_cache_compact");
    Geom gs, gd;
    int32_t rc = make_geom(src_shape, &gs);
    if (rc == STC_OK) rc = make_geom(dst_shape, &gd);
    if (rc != STC_OK) return rc;
    if (!src || !dst || max_pages < 0 || gs.B != gd.B || gs.Hkv != gd.Hkv || gs.Hq != gd.Hq || gs.S != gd.S)
        return STC_ERR_INVALID_ARG;
    if (empty(gs) || empty(gd)) return STC_OK;
    if (!complete(src) || !complete(dst) || (max_pages > 0 && !page_ids) || !n_pages || !new_len || !total_groups || !status ||
        new_len == gs.seq_len || (dst->kmin && !src->kmin))
        return STC_ERR_INVALID_ARG;
    if (src->k == dst->k && (gs.T != gd.T || src->kmin != dst->kmin || src->kmax != dst->kmax || src->v_packed != dst->v_packed ||
                             src->v_mask != dst->v_mask || src->v_offs != dst->v_offs || src->cap_groups != dst->cap_groups))
        return STC_ERR_INVALID_ARG;
    if (!aligned(src) || !aligned(dst)) return STC_ERR_INVALID_ARG;
    return cuda_rc(launch_cache_compact(gs, *src, page_ids, n_pages, max_pages, gd, *dst, new_len, total_groups, status,
                                        static_cast<cudaStream_t>(stream)));
}

int32_t stc_decode_step(const stc_shape* shape, const stc_cache* cache, const void* q, int32_t token_budget,
                        int32_t max_pages, int32_t* page_ids, int32_t* n_pages, float sm_scale, float* out,
                        float* lse_opt, void* ws_select, size_t ws_select_bytes, void* ws_attn,
                        size_t ws_attn_bytes, void* stream) {
    Range nvtx_range("stc_decode_step");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || token_budget < 0 || max_pages < 0 || !(sm_scale == sm_scale)) return STC_ERR_INVALID_ARG;
    if (g.problems == 0) return STC_OK;
    if (!q || !out || !page_ids || !n_pages) return STC_ERR_INVALID_ARG;
    if (g.T == 0 || max_pages < 1) {              // nothing to select or attend: the two plain calls handle it
        rc = stc_quest_select(shape, cache, q, token_budget, max_pages, page_ids, n_pages, nullptr, ws_select,
                              ws_select_bytes, stream);
        if (rc != STC_OK) return rc;
        return stc_decode_attn(shape, cache, q, page_ids, n_pages, max_pages, sm_scale, out, lse_opt, ws_attn,
                               ws_attn_bytes, stream);
    }
    if (!cache->kmin || !cache->kmax || !cache->k || !cache->v_packed || !cache->v_mask || !cache->v_offs ||
        cache->cap_groups < 0)
        return STC_ERR_INVALID_ARG;
    if (!aligned16(cache->k, cache->v_packed, cache->kmin, cache->kmax, q, out)) return STC_ERR_INVALID_ARG;
    const int want = token_budget / kPage < g.P ? token_budget / kPage : g.P;
    if (max_pages < want || max_pages > g.P) return STC_ERR_INVALID_ARG;
    rc = check_ws(ws_select, ws_select_bytes, select_ws_bytes(g));
    if (rc == STC_OK) rc = check_ws(ws_attn, ws_attn_bytes, attn_ws_bytes(g, max_pages));
    if (rc != STC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // both workspaces are cleared first, so that nothing stands between the two kernels
    cudaError_t e = clear_two(ws_select, quest_select_clear_bytes(g), ws_attn, decode_attn_clear_bytes(g), st);
    if (e == cudaSuccess)
        e = launch_quest_select(g, cache->kmin, cache->kmax, q, token_budget, 0, max_pages, page_ids, n_pages,
                                nullptr, ws_select, st, kLaunchNoClear);
    if (e == cudaSuccess)
        e = launch_decode_attn(g, cache->k, cache->v_packed, cache->v_mask, cache->v_offs, cache->cap_groups, q,
                               page_ids, n_pages, max_pages, sm_scale, out, lse_opt, ws_attn, st,
                               kLaunchNoClear);
    return cuda_rc(e);
}

int32_t stc_cache_bytes(int64_t n_tokens_retained, int64_t n_groups_kept, int32_t n_groups,
                        int64_t* kv_bytes_host, int64_t* index_bytes_host) {
    if (n_tokens_retained < 0 || n_groups_kept < 0 || !kv_bytes_host) return STC_ERR_INVALID_ARG;
    if (n_groups != 4 && n_groups != 8 && n_groups != 16) return STC_ERR_UNSUPPORTED;
    *kv_bytes_host = n_tokens_retained * kRowBytes + n_groups_kept * (kHeadDim / n_groups) * 2;
    if (index_bytes_host) {
        const int64_t pages = (n_tokens_retained + kPage - 1) / kPage;
        *index_bytes_host = n_tokens_retained * 2 + (n_tokens_retained + 1) * 4 + pages * 2 * kRowBytes;
    }
    return STC_OK;
}

}  // extern "C"

namespace {

struct Arena {
    char *k, *v, *scores, *cls, *q, *kmin, *kmax, *packed, *mask, *offs, *ids, *npages, *out, *total,
        *status, *ws;
    size_t ws_bytes, total_bytes;
    int max_pages;
};

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

Arena carve_arena(const Geom& g, int64_t cap_groups, int token_budget, void* base) {
    Arena a;
    char* p = static_cast<char*>(base);
    size_t o = 0;
    auto take = [&](size_t bytes) { char* r = p + o; o += up256(bytes); return r; };
    const size_t rows = (size_t)g.problems * g.T;
    a.max_pages = token_budget < 0 ? g.P : (token_budget / kPage < g.P ? token_budget / kPage : g.P);
    if (a.max_pages < 1) a.max_pages = 1;
    a.k = take(rows * kRowBytes);
    a.v = take(rows * kRowBytes);
    a.scores = take(rows * g.S * 4);
    a.cls = take((size_t)g.B * g.T);
    a.q = take((size_t)g.B * g.Hq * kRowBytes);
    a.kmin = take((size_t)g.problems * g.P * kRowBytes);
    a.kmax = take((size_t)g.problems * g.P * kRowBytes);
    a.packed = take((size_t)g.problems * cap_groups * g.g * 2);
    a.mask = take(rows * 2);
    a.offs = take((size_t)g.problems * (g.T + 1) * 4);
    a.ids = take((size_t)g.problems * a.max_pages * 4);
    a.npages = take((size_t)g.problems * 4);
    a.out = take((size_t)g.B * g.Hq * kHeadDim * 4);
    a.total = take((size_t)g.problems * 8);
    a.status = take((size_t)g.problems * 4);
    size_t w = select_ws_bytes(g);
    if (route_ws_bytes(g) > w) w = route_ws_bytes(g);
    if (attn_ws_bytes(g, a.max_pages) > w) w = attn_ws_bytes(g, a.max_pages);
    a.ws_bytes = up256(w);
    a.ws = take(a.ws_bytes);
    a.total_bytes = o;
    return a;
}

}  // namespace

extern "C" {

int32_t stc_pass_host_arena_bytes(const stc_shape* shape, int64_t cap_groups, int32_t token_budget,
                                  size_t* bytes_host) {
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!bytes_host || cap_groups < 0) return STC_ERR_INVALID_ARG;
    *bytes_host = empty(g) ? 0 : carve_arena(g, cap_groups, token_budget, nullptr).total_bytes;
    return STC_OK;
}

int32_t stc_pass_host(const stc_shape* shape, const void* k_host, const void* v_host,
                      const float* scores_host, const uint8_t* tok_class_host, const void* q_host,
                      int32_t token_budget, int32_t k_nominal, int32_t min_per_token, int32_t mode,
                      float sm_scale, int64_t cap_groups, void* arena, size_t arena_bytes,
                      float* out_host, int64_t* total_groups_host, int32_t* status_host,
                      void* stream) {
    Range nvtx_range("stc_pass_host");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (cap_groups < 0 || !k_host || !v_host || !scores_host || !q_host || !out_host ||
        !total_groups_host || !status_host)
        return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    const Arena a = carve_arena(g, cap_groups, token_budget, arena);
    rc = check_ws(arena, arena_bytes, a.total_bytes);
    if (rc != STC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t rows = (size_t)g.problems * g.T;
    cudaError_t e = cudaMemcpyAsync(a.k, k_host, rows * kRowBytes, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess) e = cudaMemcpyAsync(a.v, v_host, rows * kRowBytes, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess) e = cudaMemcpyAsync(a.scores, scores_host, rows * g.S * 4, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess && tok_class_host)
        e = cudaMemcpyAsync(a.cls, tok_class_host, (size_t)g.B * g.T, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess)
        e = cudaMemcpyAsync(a.q, q_host, (size_t)g.B * g.Hq * kRowBytes, cudaMemcpyHostToDevice, st);
    if (e != cudaSuccess) return STC_ERR_CUDA;

    stc_cache c;
    c.k = a.k; c.kmin = a.kmin; c.kmax = a.kmax; c.v_packed = a.packed;
    c.v_mask = reinterpret_cast<uint16_t*>(a.mask);
    c.v_offs = reinterpret_cast<uint32_t*>(a.offs);
    c.cap_groups = cap_groups;
    rc = stc_build_page_meta(shape, &c, 0, -1, stream);
    if (rc != STC_OK) return rc;
    rc = stc_route_pack(shape, a.v, reinterpret_cast<const float*>(a.scores),
                        tok_class_host ? reinterpret_cast<const uint8_t*>(a.cls) : nullptr, 0, k_nominal,
                        min_per_token, mode, &c, reinterpret_cast<int64_t*>(a.total),
                        reinterpret_cast<int32_t*>(a.status), a.ws, a.ws_bytes, stream);
    if (rc != STC_OK) return rc;
    const int32_t* ids = nullptr;
    if (token_budget >= 0) {
        rc = stc_quest_select(shape, &c, a.q, token_budget, a.max_pages, reinterpret_cast<int32_t*>(a.ids),
                              reinterpret_cast<int32_t*>(a.npages), nullptr, a.ws, a.ws_bytes, stream);
        if (rc != STC_OK) return rc;
        ids = reinterpret_cast<const int32_t*>(a.ids);
    }
    rc = stc_decode_attn(shape, &c, a.q, ids, reinterpret_cast<const int32_t*>(a.npages), a.max_pages,
                         sm_scale, reinterpret_cast<float*>(a.out), nullptr, a.ws, a.ws_bytes, stream);
    if (rc != STC_OK) return rc;
    e = cudaMemcpyAsync(out_host, a.out, (size_t)g.B * g.Hq * kHeadDim * 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess)
        e = cudaMemcpyAsync(total_groups_host, a.total, (size_t)g.problems * 8, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess)
        e = cudaMemcpyAsync(status_host, a.status, (size_t)g.problems * 4, cudaMemcpyDeviceToHost, st);
    return cuda_rc(e);
}


namespace {
struct StepArena { char *q, *ids, *npages, *out, *ws; size_t ws_bytes, total_bytes; int max_pages; };
StepArena carve_step_arena(const Geom& g, int token_budget, void* base) {
    StepArena a;
    char* p = static_cast<char*>(base);
    size_t o = 0;
    auto take = [&](size_t bytes) { char* r = p + o; o += up256(bytes); return r; };
    a.max_pages = token_budget < 0 ? g.P : (token_budget / kPage < g.P ? token_budget / kPage : g.P);
    if (a.max_pages < 1) a.max_pages = 1;
    a.q = take((size_t)g.B * g.Hq * kRowBytes);
    a.ids = take((size_t)g.problems * a.max_pages * 4);
    a.npages = take((size_t)g.problems * 4);
    a.out = take((size_t)g.B * g.Hq * kHeadDim * 4);
    // selection and attention keep separate workspaces: the attention status word must survive
    const size_t ws_sel = up256(select_ws_bytes(g)), ws_att = up256(attn_ws_bytes(g, a.max_pages));
    a.ws_bytes = ws_att;
    a.ws = take(ws_att);
    take(ws_sel);
    a.total_bytes = o;
    return a;
}
}  // namespace

int32_t stc_decode_step_host_arena_bytes(const stc_shape* shape, int32_t token_budget, size_t* bytes_host) {
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!bytes_host) return STC_ERR_INVALID_ARG;
    *bytes_host = empty(g) ? 0 : carve_step_arena(g, token_budget, nullptr).total_bytes;
    return STC_OK;
}

int32_t stc_decode_step_host(const stc_shape* shape, const stc_cache* cache, const void* q_host,
                             int32_t token_budget, float sm_scale, void* arena, size_t arena_bytes,
                             float* out_host, int32_t* status_host, void* stream) {
    Range nvtx_range("stc_decode_step_host");
    Geom g;
    int32_t rc = make_geom(shape, &g);
    if (rc != STC_OK) return rc;
    if (!cache || !q_host || !out_host || !status_host) return STC_ERR_INVALID_ARG;
    if (empty(g)) return STC_OK;
    const StepArena a = carve_step_arena(g, token_budget, arena);
    rc = check_ws(arena, arena_bytes, a.total_bytes);
    if (rc != STC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(a.q, q_host, (size_t)g.B * g.Hq * kRowBytes, cudaMemcpyHostToDevice, st) != cudaSuccess)
        return STC_ERR_CUDA;
    if (token_budget >= 0) {
        rc = stc_decode_step(shape, cache, a.q, token_budget, a.max_pages, reinterpret_cast<int32_t*>(a.ids),
                             reinterpret_cast<int32_t*>(a.npages), sm_scale, reinterpret_cast<float*>(a.out), nullptr,
                             a.ws + a.ws_bytes, up256(select_ws_bytes(g)), a.ws, a.ws_bytes, stream);
    } else {
        rc = stc_decode_attn(shape, cache, a.q, nullptr, nullptr, a.max_pages, sm_scale,
                             reinterpret_cast<float*>(a.out), nullptr, a.ws, a.ws_bytes, stream);
    }
    if (rc != STC_OK) return rc;
    cudaError_t e = cudaMemcpyAsync(out_host, a.out, (size_t)g.B * g.Hq * kHeadDim * 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemcpyAsync(status_host, a.ws, 4, cudaMemcpyDeviceToHost, st);
    return cuda_rc(e);
}

}  // extern "C"
