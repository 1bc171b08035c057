// Scored decode attention: the routed decode attention with capped scores, a bias linear in the distance, a sliding
// window and a document mask (stc_score).  Per query head h of sequence b with position p, over the valid tokens t
// of the listed pages that the query sees (t <= p, p - t < window, document of t shared or the query's):
//     x_t = sm_scale q_h.k_t,   x_t <- cap tanh(x_t / cap),   s_t = x_t + slope_h (t - p),
//     out = softmax(s) V~ (dropped value groups add zero),   lse = log sum exp s.
//
// What bounds it.  HBM for the largest calls (256 bytes of key and the kept groups per token; 16 x 32/8 heads over whole caches of
// 131072 tokens: 1.13 ms, 0.89 of the copy rate).  A few hundred pages per problem leave a warp few pages and the machine few warps: 8 x
// 28/4 heads, 256 pages of 16 groups, take 18.2 us for 6.6 us' worth of bytes (21 to 22 us with cold caches; DRAM at a quarter of its rate),
// 5.5 of them the start and the join.  Small calls are the chain of dependent steps: a decode step of one sequence moves half a
// microsecond's worth, and what counts is how few round trips stand between the launch and the result (1 x 8 heads: 5.9 us).
//
// Work split.  One cluster of C CTAs (4 warps each) per (sequence, KV head); warp i of the cluster takes the listed
// pages i, i + 4 C, ...  C is chosen so that the clusters fill the machine (plan below).  Each warp keeps its own
// running maximum, sum and accumulator; the four of a CTA are joined in shared memory and the CTAs of a cluster through
// each other's shared memory (distributed shared memory), each CTA finishing its share of the outputs: one launch,
// nothing in global memory, no atomics, and the same order of additions every time.  Few problems with long lists (one
// sequence that attends all of its cache) take several clusters each, whose results a second small kernel joins.
//
// (One KV head, 131072 tokens: 20.7 us for one query head, 23.4 for eight, 7.8 us' worth of bytes; 263 with one cluster.)
//
// Which pages a warp needs at all is settled before any copy: 32 listed pages at a time, one per lane, the lane
// works out which of the page's 16 tokens the query sees (window and documents included) and drops the page from the
// work if none; what is left streams through a ring of bulk asynchronous copies (a page's keys and its packed values)
// on the warp's own mbarriers.  Values of tokens that are not seen are never used, whatever they hold.
//
// Arithmetic as in the plain decode attention: several query heads per KV head on mma.sync tiles (16 tokens x 8 heads,
// softmax weights as three bf16 parts), a single head on the fp32 pipes.  The options are a handful of fp32 operations
// on at most four scores per lane and page.  The bias is taken against the last visible token instead of the query, which
// cancels in the softmax and keeps it small for the tokens that count even if the query stands far behind them;
// lse gets the difference back.
//
// The running maximum only moves when a page exceeds it by more than 2^8 (a vote instead of a reduction, and no
// rescaling of the accumulator, on most pages); weights are then at most 2^8, far from fp32's limits.
//
// Waits for copies are bounded (about a second); one that expires raises STC_ERR_TIMEOUT in the workspace status word
// and the warp goes on without the rest of its pages (outputs are then unspecified).
#include "warp_mma.cuh"

namespace stc {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxGq = 8;
constexpr int kMaxCluster = 8;
constexpr uint32_t kKeyBytes = kPage * kRowBytes;          // 4096
constexpr uint32_t kStageBytes = 2 * kKeyBytes;            // keys + worst-case value span
constexpr int kHeadStride = kHeadDim + 4;                  // floats from head to head of an exchanged accumulator (banks)
constexpr unsigned long long kWaitLimitNs = 1000000000ull;
constexpr float kSlack = 8.f;                              // log2 units the maximum may be exceeded by
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__host__ __device__ constexpr uint32_t ring_bytes(int stages) { return kWarps * stages * kStageBytes; }
__host__ __device__ constexpr uint32_t smem_bytes(int stages) { return ring_bytes(stages) + 64 + kWarps * stages * 8; }   // + zero row, mbarriers
// the exchange buffers reuse the ring: [warps][Gq][kHeadStride] accumulators, then [Gq][kHeadStride] of the CTA
static_assert((kWarps + 1) * kMaxGq * kHeadStride * 4 <= ring_bytes(2), "exchange buffers fit the ring");

struct ScoredArgs {
    const unsigned char* k;
    const unsigned char* v_packed;
    const uint16_t* v_mask;
    const uint32_t* v_offs;
    const uint4* q;
    const int32_t* page_ids;
    const int32_t* n_pages;
    const int32_t* seq_len;
    float* out;
    float* lse;
    int32_t* status;
    int64_t cap_groups;
    float* part_o;               // splits > 1: [problems][splits][Gq][128] sums, as they stand
    float2* part_ml;             // [problems][splits][Gq] maximum (log2 units) and sum
    int Hq, Hkv, Gq, T, max_pages, cluster, splits;
    float scale_log2, cap_in, cap_log2;    // sm_scale log2(e); sm_scale / cap; cap log2(e)
    ScoreArgs sc;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// fp32 at `addr` of this CTA's shared memory, but of CTA `rank` of the cluster.
__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank) {
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}"
                 : "=f"(v) : "r"(addr), "r"(rank) : "memory");
    return v;
}

// What scores are weighed against: the running maximum, or 0 as long as all of them were -inf (a seen key may hold one).
__device__ __forceinline__ float above(float m) { return m == -INFINITY ? 0.f : m; }

template <int S, bool MMA, int kStages, int kPerSm>
__global__ void __launch_bounds__(kThreads, kPerSm)
scored_attn_kernel(const ScoredArgs a) {
    constexpr uint32_t kRingBytes = ring_bytes(kStages);
    constexpr int OPG = kOctets / S;             // 16-byte chunks per value group
    constexpr uint32_t kGroupBytes = OPG * 16;
    constexpr int HEADS = MMA ? kMaxGq : 1;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float2 sh_ml[kWarps][kMaxGq];     // maximum (log2 units) and sum per warp and head
    __shared__ float sh_m[kMaxGq], sh_l[kMaxGq]; // of the CTA

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = lane >> 2, c = lane & 3;
    const int rank = (int)(blockIdx.x % (unsigned)a.cluster), cluster_id = (int)(blockIdx.x / (unsigned)a.cluster);
    const int problem = cluster_id / a.splits, split = cluster_id - problem * a.splits;
    if (a.splits > 1) asm volatile("griddepcontrol.launch_dependents;");
    const int b = problem / a.Hkv, hk = problem - b * a.Hkv;
    const uint32_t ring = smem_u32(smem) + (uint32_t)warp * kStages * kStageBytes;
    const uint32_t zero_row = smem_u32(smem) + kRingBytes;
    const uint32_t bars = smem_u32(smem) + kRingBytes + 64 + (uint32_t)warp * kStages * 8;

    // The reads the first window needs go out together: the page list does not wait for the lengths (a listed slot below
    // max_pages is readable whatever it holds).
    const int W = a.splits * a.cluster * kWarps, first_slot = (split * a.cluster + rank) * kWarps + warp;
    const int32_t* const list = a.page_ids ? a.page_ids + (size_t)problem * a.max_pages : nullptr;
    const long long slot0 = first_slot + (long long)W * lane;
    int listed = list && slot0 < a.max_pages ? list[slot0] : -1;             // this lane's entry of the next window

    // the query and what it sees
    const int len = clamp_len(a.seq_len, b, a.T), pos = a.sc.q_pos ? a.sc.q_pos[b] : len - 1;
    const int my_doc = a.sc.tok_doc ? a.sc.q_doc[b] : 0;
    const int n_list = a.page_ids ? min(max(a.n_pages[problem], 0), a.max_pages) : (len + kPage - 1) / kPage;
    uint4 qa[4];                                 // lane (r, c): chunks c, c + 4, c + 8, c + 12 of head r (zeros past Gq; FMA: head 0)
    float slope2[2] = {0.f, 0.f};                // log2 units; heads 2 c, 2 c + 1 (FMA: head 0)
    {
        const int head = MMA ? r : 0;
        const bool ok = head < a.Gq;
        const uint4* qrow = a.q + ((size_t)b * a.Hq + (size_t)hk * a.Gq + (ok ? head : 0)) * kOctets;
#pragma unroll
        for (int j = 0; j < 4; ++j) qa[j] = ok ? __ldg(qrow + c + 4 * j) : make_uint4(0, 0, 0, 0);
        if (a.sc.slopes) {
#pragma unroll
            for (int e = 0; e < (MMA ? 2 : 1); ++e) {
                const int h = MMA ? 2 * c + e : 0;
                slope2[e] = h < a.Gq ? a.sc.slopes[hk * a.Gq + h] * kLog2e : 0.f;
            }
        }
    }
    if (tid < 4) reinterpret_cast<uint32_t*>(smem + kRingBytes)[tid] = 0u;
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < kStages; ++s) mbar_init(bars + 8 * s, 1);
        fence_mbar_init();
    }
    if (blockIdx.x == 0 && tid == 0) *a.status = STC_OK;
    int see_lo, see_hi;
    visible_range(len, pos, a.sc.window, see_lo, see_hi);
    __syncthreads();

    // ---- lookahead window: lane i describes the i-th of the warp's next 32 listed pages -----------------------
    int page = -1;                               // page id of this lane's entry
    uint32_t seen = 0, first = 0, groups = 0;    // bit t = token t of the page is seen; its span of the packed store
    uint32_t todo = 0;                           // entries with something to attend, not issued yet (same in all lanes)
    long long next_slot = first_slot;
    auto fill = [&]() {
        const long long slot = next_slot + (long long)W * lane;
        page = -1;
        if (slot < n_list) page = list ? listed : (int)slot;
        seen = 0;
        // (an id outside the sequence is skipped; see_hi <= len)
        if (page >= 0 && page < (len + kPage - 1) / kPage) {
            const int t0 = page * kPage, lo = max(see_lo - t0, 0), hi = min(see_hi - t0, kPage);
            if (lo < hi) seen = (0xFFFFu >> (kPage - hi)) & ~((1u << lo) - 1u);
            if (seen) {
                const int nv = min(kPage, len - t0);
                const uint32_t* o = a.v_offs + (size_t)problem * (a.T + 1) + t0;
                const long long ob = min((long long)o[0], (long long)a.cap_groups);
                const long long oe = min((long long)o[nv], (long long)a.cap_groups);
                first = (uint32_t)ob;
                groups = (uint32_t)min(oe > ob ? oe - ob : 0LL, (long long)(kPage * S));       // never past the stage
                if (a.sc.tok_doc) {
                    const int32_t* doc = a.sc.tok_doc + (size_t)b * a.T + t0;
                    uint32_t keep = 0;
#pragma unroll
                    for (int t = 0; t < kPage; ++t) {
                        const int d = t < nv ? __ldg(doc + t) : 0;
                        if (d < 0 || d == my_doc) keep |= 1u << t;
                    }
                    seen &= keep;
                }
            }
        }
        todo = __ballot_sync(0xFFFFFFFFu, seen != 0);
        next_slot += 32 * W;
        const long long ahead = next_slot + (long long)W * lane;
        listed = list && ahead < n_list ? list[ahead] : -1;
    };

    // ---- the pages in flight: a register FIFO, oldest first -----------------------------------------------------
    struct InFlight {
        uint32_t seen;       // 0 = empty
        uint32_t chunks;     // 16-byte chunks of the value span present in the stage
        uint32_t mask;       // lanes 0..15: group mask of token `lane`
        uint32_t at;         // lanes 0..15: its first group in the packed store
        uint32_t first;      // the page's first group
        int t0;
    };
    auto issue = [&](int s, bool reuse) -> InFlight {
        InFlight f{0u, 0u, 0u, 0u, 0u, 0};
        while (todo == 0) {
            if (next_slot >= n_list) return f;
            fill();
        }
        const int src = __ffs(todo) - 1;
        todo &= todo - 1;
        const int id = __shfl_sync(0xFFFFFFFFu, page, src);
        f.seen = __shfl_sync(0xFFFFFFFFu, seen, src);
        const uint32_t at = __shfl_sync(0xFFFFFFFFu, first, src), n = __shfl_sync(0xFFFFFFFFu, groups, src);
        f.t0 = id * kPage;
        f.chunks = n * OPG;
        const int nv = min(kPage, len - f.t0);
        const size_t row0 = (size_t)problem * a.T + (size_t)f.t0;
        f.first = at;
        if (lane < nv) {
            f.mask = a.v_mask[row0 + lane];
            f.at = a.v_offs[(size_t)problem * (a.T + 1) + (size_t)f.t0 + lane];
        }
        if (lane == 0) {
            const uint32_t kb = (uint32_t)nv * kRowBytes, vb = n * kGroupBytes;
            const uint32_t bar = bars + 8 * s, dst = ring + (uint32_t)s * kStageBytes;
            if (reuse) fence_proxy_async();      // the stage's earlier reads precede the new writes
            mbar_expect_tx(bar, kb + vb);
            bulk_g2s(dst, a.k + row0 * kRowBytes, kb, bar);
            if (vb) bulk_g2s(dst + kKeyBytes, a.v_packed + ((size_t)problem * a.cap_groups + at) * kGroupBytes, vb, bar);
        }
        return f;
    };

    // ---- running state ----------------------------------------------------------------------------------------------
    // MMA: acc[dt][0..3] = (dim 16dt+r, head 2c), (16dt+r, 2c+1), (16dt+r+8, 2c), (16dt+r+8, 2c+1);
    //      m_run/l_run[e] belong to head 2c+e (l_run summed over the lane's own tokens only).
    // FMA: acc[j][2q2+e] -> dim 8(c+4j)+2q2+e, summed over the lane's own two tokens; m_run[0], l_run[0].
    float acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};

    // N raw products of tokens t[i] -> scores in log2 units (one branch per page, not per score)
    auto score = [&](auto& x, const int* t, const int* e, int n) {
        if (a.sc.softcap > 0.f) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) x[i] = a.cap_log2 * tanh_f32(x[i] * a.cap_in);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) x[i] *= a.scale_log2;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) x[i] = fmaf(slope2[e[i]], (float)(t[i] - (see_hi - 1)), x[i]);
    };

    auto compute = [&](int s, const InFlight& f) {
        const uint32_t kst = ring + (uint32_t)s * kStageBytes, vst = kst + kKeyBytes;
        const uint32_t pre = f.at - f.first;     // groups of the page before the token (lanes 0..15)
        const uint32_t mask = (f.seen >> (lane & 15)) & 1u ? f.mask : 0u;     // groups that may be read
        const bool v0 = (f.seen >> r) & 1u, v1 = (f.seen >> (r + 8)) & 1u;

        if constexpr (MMA) {
            // S^T = K . Q^T : rows = tokens (r, r+8), columns = heads (2c, 2c+1)
            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 k0 = lds16(kst + (uint32_t)r * kRowBytes + (uint32_t)(c + 4 * j) * 16u);
                const uint4 k1 = lds16(kst + (uint32_t)(r + 8) * kRowBytes + (uint32_t)(c + 4 * j) * 16u);
                mma_bf16(s0, k0.x, k1.x, k0.y, k1.y, qa[j].x, qa[j].y);
                mma_bf16(s1, k0.z, k1.z, k0.w, k1.w, qa[j].z, qa[j].w);
            }
            float sv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sv[i] = s0[i] + s1[i];
            const int t[4] = {f.t0 + r, f.t0 + r, f.t0 + r + 8, f.t0 + r + 8}, e[4] = {0, 1, 0, 1};
            score(sv, t, e, 4);
            sv[0] = v0 ? sv[0] : -INFINITY; sv[1] = v0 ? sv[1] : -INFINITY;
            sv[2] = v1 ? sv[2] : -INFINITY; sv[3] = v1 ? sv[3] : -INFINITY;
            float al0 = 1.f, al1 = 1.f;
            bool moved = false;
            if (__any_sync(0xFFFFFFFFu, fmaxf(sv[0], sv[2]) > m_run[0] + kSlack || fmaxf(sv[1], sv[3]) > m_run[1] + kSlack)) {
                float pm0 = fmaxf(sv[0], sv[2]), pm1 = fmaxf(sv[1], sv[3]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    pm0 = fmaxf(pm0, __shfl_xor_sync(0xFFFFFFFFu, pm0, d));
                    pm1 = fmaxf(pm1, __shfl_xor_sync(0xFFFFFFFFu, pm1, d));
                }
                const float mn0 = fmaxf(m_run[0], pm0), mn1 = fmaxf(m_run[1], pm1);
                al0 = ex2(m_run[0] - above(mn0)); al1 = ex2(m_run[1] - above(mn1));
                m_run[0] = mn0; m_run[1] = mn1;
                moved = true;
            }
            const float ref0 = above(m_run[0]), ref1 = above(m_run[1]);
            const float p0 = ex2(sv[0] - ref0), p1 = ex2(sv[1] - ref1), p2 = ex2(sv[2] - ref0), p3 = ex2(sv[3] - ref1);
            l_run[0] = fmaf(l_run[0], al0, p0 + p2);
            l_run[1] = fmaf(l_run[1], al1, p1 + p3);
            if (moved) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) { acc[dt][0] *= al0; acc[dt][1] *= al1; acc[dt][2] *= al0; acc[dt][3] *= al1; }
            }
            // P^T as B fragments: a weight is the sum of three bf16 parts (24 bits, so the weights are as good as fp32; the third
            // part costs a page 8 of 32 MMAs)
            uint32_t wb[3][2];
            {
                float x0 = p0, x1 = p1, x2 = p2, x3 = p3;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const uint32_t u0 = pack_bf16(x0, x1), u1 = pack_bf16(x2, x3);
                    wb[k][0] = movmatrix_trans(u0);
                    wb[k][1] = movmatrix_trans(u1);
                    x0 -= bf16lo(u0); x1 -= bf16hi(u0); x2 -= bf16lo(u1); x3 -= bf16hi(u1);
                }
            }
            // value rows: this lane addresses token tau, chunk 2dt + hb of every dim tile
            const int tau = (lane & 7) + 8 * (lane >> 4), hb = (lane >> 3) & 1;
            const uint32_t m = __shfl_sync(0xFFFFFFFFu, mask, tau);
            const uint32_t base = __shfl_sync(0xFFFFFFFFu, pre, tau) * OPG;
            // the low half of a masked token's own groups does not matter: its prefix counts all of them
            const uint32_t all = __shfl_sync(0xFFFFFFFFu, f.mask, tau);
            // The page's product starts from zero and is added by the fp32 pipes, which round to nearest: mma.sync truncates the sum
            // it adds to, and over hundreds of pages that takes a share of the result away (683 pages per warp, 16 x 32/8 heads:
            // error 5.5e-5 when acc itself was the sum, 1.4e-7 now).  Small parts first, so that only the last product truncates
            // at the sum's full size; the eight tiles' chains side by side (8 x 28/4 heads: acc as the sum 17.6 us, one chain
            // after the other 18.9, side by side 18.3).
            uint32_t vr[8][4];
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const int oct = 2 * dt + hb, grp = oct / OPG;
                const uint32_t idx = base + __popc(all & ((1u << grp) - 1u)) * OPG + (uint32_t)(oct % OPG);
                const bool kept = ((m >> grp) & 1u) && idx < f.chunks;
                ldmatrix_x4_trans(kept ? vst + idx * 16u : zero_row, vr[dt][0], vr[dt][1], vr[dt][2], vr[dt][3]);
            }
            float sum[8][4] = {};
#pragma unroll
            for (int k = 2; k >= 0; --k)
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) mma_bf16(sum[dt], vr[dt][0], vr[dt][1], vr[dt][2], vr[dt][3], wb[k][0], wb[k][1]);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[dt][i] += sum[dt][i];
        } else {
            // one head on the fp32 pipes: lane = tokens r, r+8 x chunks c, c+4, c+8, c+12
            float sd[4];
            uint4 kr[2][4];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    kr[hf][j] = lds16(kst + (uint32_t)(r + 8 * hf) * kRowBytes + (uint32_t)(c + 4 * j) * 16u);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                float d0 = 0.f, d1 = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    d0 = fmaf(bf16lo(qa[j].x), bf16lo(kr[hf][j].x), d0);
                    d1 = fmaf(bf16hi(qa[j].x), bf16hi(kr[hf][j].x), d1);
                    d0 = fmaf(bf16lo(qa[j].y), bf16lo(kr[hf][j].y), d0);
                    d1 = fmaf(bf16hi(qa[j].y), bf16hi(kr[hf][j].y), d1);
                    d0 = fmaf(bf16lo(qa[j].z), bf16lo(kr[hf][j].z), d0);
                    d1 = fmaf(bf16hi(qa[j].z), bf16hi(kr[hf][j].z), d1);
                    d0 = fmaf(bf16lo(qa[j].w), bf16lo(kr[hf][j].w), d0);
                    d1 = fmaf(bf16hi(qa[j].w), bf16hi(kr[hf][j].w), d1);
                }
                float d = d0 + d1;
                d += __shfl_xor_sync(0xFFFFFFFFu, d, 1);
                d += __shfl_xor_sync(0xFFFFFFFFu, d, 2);
                sd[hf] = d;
            }
            const int t[4] = {f.t0 + r, f.t0 + r + 8, 0, 0}, e[4] = {0, 0, 0, 0};
            score(sd, t, e, 2);
            sd[0] = v0 ? sd[0] : -INFINITY;
            sd[1] = v1 ? sd[1] : -INFINITY;
            float al = 1.f;
            if (__any_sync(0xFFFFFFFFu, fmaxf(sd[0], sd[1]) > m_run[0] + kSlack)) {
                float pm = fmaxf(sd[0], sd[1]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) pm = fmaxf(pm, __shfl_xor_sync(0xFFFFFFFFu, pm, d));
                const float mn = fmaxf(m_run[0], pm);
                al = ex2(m_run[0] - above(mn));
                m_run[0] = mn;
            }
            const float ref = above(m_run[0]), p0 = ex2(sd[0] - ref), p1 = ex2(sd[1] - ref);
            l_run[0] = fmaf(l_run[0], al, p0 + p1);
            uint4 vr[2][4];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint32_t m = __shfl_sync(0xFFFFFFFFu, mask, r + 8 * hf);
                const uint32_t base = __shfl_sync(0xFFFFFFFFu, pre, r + 8 * hf) * OPG;
                const uint32_t all = __shfl_sync(0xFFFFFFFFu, f.mask, r + 8 * hf);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int oct = c + 4 * j, grp = oct / OPG;
                    const uint32_t idx = base + __popc(all & ((1u << grp) - 1u)) * OPG + (uint32_t)(oct % OPG);
                    const bool kept = ((m >> grp) & 1u) && idx < f.chunks;
                    vr[hf][j] = kept ? lds16(vst + idx * 16u) : make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t u0[4] = {vr[0][j].x, vr[0][j].y, vr[0][j].z, vr[0][j].w};
                const uint32_t u1[4] = {vr[1][j].x, vr[1][j].y, vr[1][j].z, vr[1][j].w};
#pragma unroll
                for (int q2 = 0; q2 < 4; ++q2) {
                    float& lo = acc[2 * j + (q2 >> 1)][2 * (q2 & 1)];
                    float& hi = acc[2 * j + (q2 >> 1)][2 * (q2 & 1) + 1];
                    lo = fmaf(p1, bf16lo(u1[q2]), fmaf(p0, bf16lo(u0[q2]), lo * al));
                    hi = fmaf(p1, bf16hi(u1[q2]), fmaf(p0, bf16hi(u0[q2]), hi * al));
                }
            }
        }
    };

    // ---- main loop ----------------------------------------------------------------------------------------------
    {
        InFlight f[kStages];                     // f[0] = oldest page in flight, in stage s
#pragma unroll
        for (int i = 0; i < kStages; ++i) f[i] = issue(i, false);
        uint32_t phase = 0;                      // bit s = parity to wait for on stage s
        int s = 0;
#pragma unroll 1
        while (f[0].seen) {
            const uint32_t par = (phase >> s) & 1u;
            phase ^= 1u << s;
            if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(bars + 8 * s, par, kWaitLimitNs))) {
                // A copy did not land in time.  Report it and give the copies still in flight one more bounded wait each, so
                // that they do not land in the exchange buffers or a dead CTA's memory.
                if (lane == 0) atomicExch(a.status, (int)STC_ERR_TIMEOUT);
                int s2 = s;
#pragma unroll
                for (int i = 1; i < kStages; ++i) {
                    s2 = s2 + 1 == kStages ? 0 : s2 + 1;
                    if (f[i].seen) mbar_wait_bounded(bars + 8 * s2, (phase >> s2) & 1u, kWaitLimitNs);
                }
                break;
            }
            compute(s, f[0]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i + 1 < kStages; ++i) f[i] = f[i + 1];
            f[kStages - 1] = issue(s, true);
            s = s + 1 == kStages ? 0 : s + 1;
        }
    }

    // ---- join: the warps of the CTA, then the CTAs of the cluster --------------------------------------------------
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
        l_run[0] += __shfl_xor_sync(0xFFFFFFFFu, l_run[0], d);
        if (MMA) l_run[1] += __shfl_xor_sync(0xFFFFFFFFu, l_run[1], d);
    }
    if constexpr (!MMA) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][e], d);
    }
    __syncthreads();                             // every warp is through with its ring
    float* const ex = reinterpret_cast<float*>(smem);                    // [kWarps][HEADS][kHeadStride]
    float* const cta = ex + kWarps * HEADS * kHeadStride;                // [HEADS][kHeadStride]
    {
        float* mine = ex + warp * HEADS * kHeadStride;
        if constexpr (MMA) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int h = 2 * c + e;
                if (r == 0) sh_ml[warp][h] = make_float2(m_run[e], l_run[e]);
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    mine[h * kHeadStride + 16 * dt + r] = acc[dt][e];
                    mine[h * kHeadStride + 16 * dt + r + 8] = acc[dt][2 + e];
                }
            }
        } else if (r == 0) {                     // lanes 0..3 hold the reduced 128 channels
            if (c == 0) sh_ml[warp][0] = make_float2(m_run[0], l_run[0]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) mine[8 * (c + 4 * j) + e] = acc[2 * j + (e >> 2)][e & 3];
        }
    }
    __syncthreads();
    const int share = a.cluster;
    const size_t row_base = (size_t)b * a.Hq + (size_t)hk * a.Gq;
    // what lse lacks: slope * (last visible token - position of the query)
    auto lse_of = [&](int h, float m, float l) {
        const float shift = a.sc.slopes ? a.sc.slopes[hk * a.Gq + h] * (float)(see_hi - 1 - pos) : 0.f;
        return l != 0.f ? (m + log2f(l)) * kLn2 + shift : -INFINITY;
    };
    // channel d of head h is finished (or this cluster's part of it)
    const size_t part_row = (size_t)cluster_id * a.Gq;
    auto put = [&](int h, int d, float m, float l, float o) {
        if (a.splits > 1) {
            a.part_o[(part_row + h) * kHeadDim + d] = o;
            if (d == 0) a.part_ml[part_row + h] = make_float2(m, l);
        } else {
            a.out[(row_base + h) * kHeadDim + d] = l != 0.f ? o / l : 0.f;     // (a NaN among the seen is an answer)
            if (a.lse && d == 0) a.lse[row_base + h] = lse_of(h, m, l);
        }
    };
#pragma unroll 1
    for (int h = 0; h < a.Gq; ++h) {             // thread = channel
        float2 p[kWarps];
        float m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { p[w] = sh_ml[w][h]; m = fmaxf(m, p[w].x); }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = ex2(p[w].x - above(m));
            l = fmaf(p[w].y, f, l);
            o = fmaf(ex[(w * HEADS + h) * kHeadStride + tid], f, o);
        }
        if (share == 1) {
            put(h, tid, m, l, o);
        } else {
            cta[h * kHeadStride + tid] = o;
            if (tid == 0) { sh_m[h] = m; sh_l[h] = l; }
        }
    }
    if (share == 1) return;
    cluster_sync();
    const uint32_t at_m = smem_u32(sh_m), at_l = smem_u32(sh_l), at_o = smem_u32(cta);
#pragma unroll 1
    for (int i = rank * kThreads + tid; i < a.Gq * kHeadDim; i += share * kThreads) {
        const int h = i >> 7, d = i & (kHeadDim - 1);
        float pm[kMaxCluster], pl[kMaxCluster], po[kMaxCluster], m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k) {
            if (k >= share) { pm[k] = -INFINITY; pl[k] = po[k] = 0.f; continue; }
            pm[k] = ld_cluster(at_m + 4u * h, k);
            pl[k] = ld_cluster(at_l + 4u * h, k);
            po[k] = ld_cluster(at_o + 4u * (uint32_t)(h * kHeadStride + d), k);
            m = fmaxf(m, pm[k]);
        }
#pragma unroll
        for (int k = 0; k < kMaxCluster; ++k) {
            const float f = ex2(pm[k] - above(m));
            l = fmaf(pl[k], f, l);
            o = fmaf(po[k], f, o);
        }
        put(h, d, m, l, o);
    }
    cluster_sync();                              // no CTA leaves while another still reads its shared memory
}

// Joins the clusters of a problem: one warp per (problem, head), a lane four channels; lane = cluster for the weights.
__global__ void __launch_bounds__(128)
scored_join_kernel(const ScoredArgs a, int rows) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int task = (int)blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (task >= rows) return;
    const int problem = task / a.Gq, h = task - problem * a.Gq, b = problem / a.Hkv, hk = problem - b * a.Hkv;
    const size_t first = (size_t)problem * a.splits * a.Gq + h;
    const float2 p = lane < a.splits ? a.part_ml[first + (size_t)lane * a.Gq] : make_float2(-INFINITY, 0.f);
    float m = p.x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    const float f = ex2(p.x - above(m));
    float l = p.y * f;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int k = 0; k < a.splits; ++k) {
        const float4 v = reinterpret_cast<const float4*>(a.part_o + (first + (size_t)k * a.Gq) * kHeadDim)[lane];
        const float w = __shfl_sync(0xFFFFFFFFu, f, k);
        o.x = fmaf(v.x, w, o.x); o.y = fmaf(v.y, w, o.y); o.z = fmaf(v.z, w, o.z); o.w = fmaf(v.w, w, o.w);
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    const size_t row = (size_t)b * a.Hq + (size_t)hk * a.Gq + h;
    reinterpret_cast<float4*>(a.out + row * kHeadDim)[lane] = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.lse && lane == 0) {
        float shift = 0.f;
        if (a.sc.slopes) {
            const int len = clamp_len(a.seq_len, b, a.T), pos = a.sc.q_pos ? a.sc.q_pos[b] : len - 1;
            int lo, hi;
            visible_range(len, pos, a.sc.window, lo, hi);
            shift = a.sc.slopes[hk * a.Gq + h] * (float)(hi - 1 - pos);
        }
        a.lse[row] = l != 0.f ? (m + log2f(l)) * kLn2 + shift : -INFINITY;
    }
}

// CTAs per cluster and clusters per problem.  A call takes waves x (pages of a warp + 3) page times: CTAs resident at
// once, and about three page times to start, to fill the ring and to join; several clusters cost three more for the second
// kernel and are looked at where a warp of the largest cluster would have 16 pages or more, up to as many as the
// workspace has partial slots for.  (Single-head and 4-head problems of 2048 to 8192 pages: 20 to 84 us against 74 to
// 290 with one cluster or the plain kernel's split.)
void plan(int problems, int max_pages, int resident, int slots, int* cluster, int* splits) {
    double least = 0.0;
    *splits = 1;
    for (int c = 1; c <= kMaxCluster; ++c) {
        if (c == 5 || c == 7) continue;          // they pack badly into the machine's groups of SMs
        const double waves = (double)(((long long)problems * c + resident - 1) / resident);
        const double cost = waves * ((max_pages + kWarps * c - 1) / (kWarps * c) + 3.0);
        if (c == 1 || cost < least) { least = cost; *cluster = c; }
    }
    if (max_pages < kWarps * kMaxCluster * 16) return;
    for (int n = 2; n <= 32 && n <= slots && (long long)problems * n <= resident; ++n) {
        const int room = resident / (problems * n);
        const int c = room >= 8 ? 8 : room >= 4 ? 4 : room >= 2 ? 2 : 1;     // (seven CTAs to a cluster: 125 us where eight take 84)
        const double cost = (max_pages + kWarps * c * n - 1) / (kWarps * c * n) + 6.0;
        if (cost < least) { least = cost; *cluster = c; *splits = n; }
    }
}

template <int S, bool MMA, int kStages, int kPerSm>
cudaError_t launch(const ScoredArgs& a, int problems, cudaStream_t st) {
    auto kernel = scored_attn_kernel<S, MMA, kStages, kPerSm>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(kStages));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(problems * a.splits * a.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes(kStages);
    cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)a.cluster;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess || a.splits == 1) return e;
    const int rows = problems * a.Gq;
    cudaLaunchConfig_t join = {};
    join.gridDim = dim3((unsigned)((rows + 3) / 4));
    join.blockDim = dim3(128);
    join.stream = st;
    cudaLaunchAttribute early;                       // its blocks wait in place instead of behind a launch
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    join.attrs = &early;
    join.numAttrs = 1;
    return cudaLaunchKernelEx(&join, scored_join_kernel, a, rows);
}

}  // namespace

cudaError_t launch_scored_attn(const Geom& g, const void* k, const void* v_packed, const uint16_t* v_mask,
                               const uint32_t* v_offs, int64_t cap_groups, const void* q, const int32_t* page_ids,
                               const int32_t* n_pages, int max_pages, float sm_scale, const ScoreArgs& score, float* out,
                               float* lse, void* ws, cudaStream_t st) {
    if (g.problems == 0) return cudaSuccess;
    ScoredArgs a;
    a.k = static_cast<const unsigned char*>(k);
    a.v_packed = static_cast<const unsigned char*>(v_packed);
    a.v_mask = v_mask; a.v_offs = v_offs;
    a.q = static_cast<const uint4*>(q);
    a.page_ids = page_ids; a.n_pages = n_pages; a.seq_len = g.seq_len;
    a.out = out; a.lse = lse;
    a.status = static_cast<int32_t*>(ws);
    a.cap_groups = cap_groups;
    a.Hq = g.Hq; a.Hkv = g.Hkv; a.Gq = g.Gq; a.T = g.T; a.max_pages = max_pages;
    a.sc = score;
    a.scale_log2 = sm_scale * kLog2e;
    a.cap_in = score.softcap > 0.f ? sm_scale / score.softcap : 0.f;
    a.cap_log2 = score.softcap * kLog2e;
    int sms = 0;
    cudaError_t e = device_sm_count(&sms);
    if (e != cudaSuccess) return e;
    // three CTAs per SM with two stages per warp: a page's arithmetic outlasts a copy, so twelve warps per SM beat eight with
    // three stages (8 sequences, 28 / 4 heads, 256 pages, their state in L2: 15.3 against 15.9 us); six or twelve warps per CTA took
    // 14.4 us there, but 5.9 and 6.3 instead of 5.6 for one sequence of 8 heads, and clusters of 9 to 16 CTAs 16.8 to 27 us
    plan(g.problems, max_pages, sms * 3, attn_plan(g, max_pages).slots_cap, &a.cluster, &a.splits);
    a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + 256);
    a.part_o = reinterpret_cast<float*>(a.part_ml) + ((size_t)g.problems * a.splits * g.Gq * 2 + 63) / 64 * 64;
#define STC_SCORED(S_) \
    case S_: return g.Gq > 1 ? launch<S_, true, 2, 3>(a, g.problems, st) : launch<S_, false, 2, 3>(a, g.problems, st);
    switch (g.S) {
        STC_SCORED(4) STC_SCORED(8) STC_SCORED(16)
        default: return cudaErrorInvalidValue;
    }
#undef STC_SCORED
}

}  // namespace stc
