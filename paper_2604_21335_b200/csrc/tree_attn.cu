// Attention for trees of drafted tokens over a routed cache.
//
//   Row r = (sequence b, node i, query head h):  softmax over the valid tokens of the listed pages and the nodes N_i (node i and
//   its ancestors) of s = sm_scale * q.k (+ options of stc_score),  out = sum p v~,  lse = log sum exp s.
//
// Simplest form: one warp per row, a lane owns four channels, tokens one by one with a running maximum.
#include "common.cuh"

namespace stc {
namespace {

constexpr int kThreads = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct TreeArgs {
    const uint2* q;
    const uint2* k;
    const uint2* k_new;
    const uint2* v_new;
    const __nv_bfloat16* v_packed;
    const uint16_t* v_mask;
    const uint32_t* v_offs;
    const int32_t* seq_len;
    const int32_t* parent;
    const int32_t* n_nodes;
    const int32_t* page_ids;
    const int32_t* n_pages;
    float* out;
    float* lse;
    int32_t* status;
    int32_t* word;
    int64_t cap_groups;
    int B, Hq, Hkv, Gq, T, P, S, n_cap, max_pages;
    float scale;
    ScoreArgs sc;
};

__global__ void __launch_bounds__(kThreads) tree_attn_kernel(const TreeArgs a) {
    const long long row = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.word = STC_OK;
    if (row >= (long long)a.B * a.n_cap * a.Hq) return;
    const int h = (int)(row % a.Hq), node = (int)(row / a.Hq % a.n_cap), b = (int)(row / a.Hq / a.n_cap);
    const int len = clamp_len(a.seq_len, b, a.T), n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.n_cap) : a.n_cap;
    const int32_t* parent = a.parent ? a.parent + (size_t)b * a.n_cap : nullptr;
    bool bad = false;
    for (int i = lane; i < n && parent; i += 32) bad |= parent[i] < -1 || parent[i] >= i;
    bad = __any_sync(0xFFFFFFFFu, bad);
    if (h == 0 && node == 0 && lane == 0) a.status[b] = bad ? STC_ERR_INVALID_ARG : STC_OK;
    if (bad || node >= n) return;
    auto up = [&](int i) { return parent ? parent[i] : i - 1; };
    auto depth = [&](int i) { int d = 0; for (i = up(i); i >= 0; i = up(i)) ++d; return d; };
    auto pos_of = [&](int i) { return a.sc.q_pos ? a.sc.q_pos[(size_t)b * a.n_cap + i] : len + depth(i); };
    const int hk = h / a.Gq, pos = pos_of(node);
    const size_t problem = (size_t)b * a.Hkv + hk;
    const float slope = a.sc.slopes ? a.sc.slopes[h] : 0.f;
    const uint2 qw = a.q[(size_t)row * 32 + lane];
    float m = -INFINITY, l = 0.f, o[4] = {};
    auto take = [&](uint2 kw, const float (&v)[4], int t) {
        float s = bf16lo(qw.x) * bf16lo(kw.x);
        s = fmaf(bf16hi(qw.x), bf16hi(kw.x), s);
        s = fmaf(bf16lo(qw.y), bf16lo(kw.y), s);
        s = fmaf(bf16hi(qw.y), bf16hi(kw.y), s);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        s *= a.scale;
        if (a.sc.softcap > 0.f) s = a.sc.softcap * tanh_f32(s / a.sc.softcap);
        s += slope * (float)(t - pos);
        const float top = s > m ? s : m, f = m == -INFINITY ? 0.f : expf(m - top), w = s == -INFINITY ? 0.f : expf(s - top);
        l = fmaf(l, f, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], f, w * v[e]);
        m = top;
    };
    auto hidden = [&](int t) { return t > pos || (a.sc.window > 0 && pos - t >= a.sc.window); };
    const int pages = (len + kPage - 1) / kPage, listed = a.page_ids ? min(max(a.n_pages[problem], 0), a.max_pages) : pages;
    for (int i = 0; i < listed; ++i) {
        const int page = a.page_ids ? a.page_ids[problem * a.max_pages + i] : i;
        if (page < 0 || page >= pages) continue;
        for (int t = page * kPage; t < min(len, (page + 1) * kPage); ++t) {
            if (hidden(t)) continue;
            if (a.sc.tok_doc) {
                const int d = a.sc.tok_doc[(size_t)b * a.T + t];
                if (d >= 0 && d != a.sc.q_doc[b]) continue;
            }
            const uint32_t mask = a.v_mask[problem * a.T + t];
            const int g = kHeadDim / a.S, grp = 4 * lane / g;
            const int64_t at = (int64_t)a.v_offs[problem * (a.T + 1) + t] + __popc(mask & ((1u << grp) - 1u));
            float v[4] = {};
            if ((mask >> grp & 1u) && at < a.cap_groups)
                for (int e = 0; e < 4; ++e) v[e] = __bfloat162float(a.v_packed[(problem * a.cap_groups + at) * g + (4 * lane) % g + e]);
            take(a.k[(problem * a.T + t) * 32 + lane], v, t);
        }
    }
    for (int i = node; i >= 0; i = up(i)) {
        const int t = pos_of(i);
        if (hidden(t)) continue;
        const uint2 vw = a.v_new[(problem * a.n_cap + i) * 32 + lane];
        const float v[4] = {bf16lo(vw.x), bf16hi(vw.x), bf16lo(vw.y), bf16hi(vw.y)};
        take(a.k_new[(problem * a.n_cap + i) * 32 + lane], v, t);
    }
    const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
    reinterpret_cast<float4*>(a.out)[(size_t)row * 32 + lane] = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (a.lse && lane == 0) a.lse[row] = l == l ? (l > 0.f ? m + logf(l) : -INFINITY) : l;
}

}  // namespace

size_t tree_attn_ws_bytes(const Geom&, int) { return 256; }

cudaError_t launch_tree_attn(const Geom& g, const stc_cache& cache, const stc_tree& tree, const void* q, const int32_t* page_ids,
                             const int32_t* n_pages, int max_pages, float sm_scale, const ScoreArgs& score, float* out, float* lse,
                             int32_t* status, void* ws, cudaStream_t st) {
    TreeArgs a;
    a.q = static_cast<const uint2*>(q); a.k = static_cast<const uint2*>(cache.k);
    a.k_new = static_cast<const uint2*>(tree.k); a.v_new = static_cast<const uint2*>(tree.v);
    a.v_packed = static_cast<const __nv_bfloat16*>(cache.v_packed); a.v_mask = cache.v_mask; a.v_offs = cache.v_offs;
    a.seq_len = g.seq_len; a.parent = tree.parent; a.n_nodes = tree.n_nodes; a.page_ids = page_ids; a.n_pages = n_pages;
    a.out = out; a.lse = lse; a.status = status; a.word = static_cast<int32_t*>(ws); a.cap_groups = cache.cap_groups;
    a.B = g.B; a.Hq = g.Hq; a.Hkv = g.Hkv; a.Gq = g.Gq; a.T = g.T; a.P = g.P; a.S = g.S; a.n_cap = tree.n_cap;
    a.max_pages = max_pages; a.scale = sm_scale; a.sc = score;
    const long long rows = (long long)g.B * tree.n_cap * g.Hq;
    tree_attn_kernel<<<(unsigned)((rows + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace stc
