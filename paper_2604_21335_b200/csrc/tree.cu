// Speculative decoding around the attention: greedy verification of drafted trees, and the accepted nodes' way into the cache.
//
// stc_tree_accept.  Only the logits of accepted nodes matter, and which they are is known step by step: the root's row
// gives a token, the token a child, the child's row the next token.  So a cluster of CTAs walks one sequence: each CTA
// takes a slice of the row, every warp tells all CTAs its best through distributed shared memory, every warp finds the child by
// itself.  Bound by that chain: a row from HBM, one meeting, the child, eight times over for 16 trees of 64 over 152064 words in
// bf16 (25 us, 3.3 us of bytes).  A thread keeps the 16 bytes with its largest logit and looks for the place in them once, at the
// end of the row; key and index reduce as two 32-bit words (place by place, 64-bit words and a stage per CTA: 49 us).
//
// stc_tree_commit.  One CTA per (sequence, KV head): rows of 256 bytes from the draft buffers to the cache, a few kilobytes
// per problem; the time is one launch and two dependent round trips (path, rows): 6 us on the device for 64x8 problems.
#include <cooperative_groups.h>

#include "common.cuh"

namespace stc {
namespace {

namespace cg = cooperative_groups;

constexpr int kAcceptThreads = 512, kAcceptCtas = 8, kAcceptWarps = kAcceptThreads / 32;

// The best of a set of logits: the largest key (NaN above everything), the lowest index among equals.
struct Best {
    uint32_t key = 0, index = 0xFFFFFFFFu;                   // (key 0: none; of a logit it is at least float_key(-inf) > 0)
    __device__ __forceinline__ void take(float x, uint32_t i) { take(x != x ? 0xFFFFFFFFu : float_key(x + 0.f), i); }    // (-0 is 0)
    __device__ __forceinline__ void take(uint32_t k, uint32_t i) {
        if (k > key || (k == key && i < index)) {
            key = k;
            index = i;
        }
    }
    __device__ __forceinline__ void over_warp() {
        const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, key);
        index = __reduce_min_sync(0xFFFFFFFFu, key == top ? index : 0xFFFFFFFFu);
        key = top;
    }
};

template <bool BF16>
__device__ __forceinline__ float logit_at(const void* row, uint32_t i) {
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[i] << 16);
    else return static_cast<const float*>(row)[i];
}
// Maximum of the logits of 16 bytes; NaN if there is one.
template <bool BF16>
__device__ __forceinline__ float top_of(const uint4& w) {
    if constexpr (BF16) {
        auto top2 = [](uint32_t a, uint32_t b) {
            uint32_t r;
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        };
        const uint32_t t = top2(top2(w.x, w.y), top2(w.z, w.w)), u = top2(t, t >> 16 | t << 16);
        return bf16lo(u);
    } else {
        auto top = [](float a, float b) {
            float r;
            asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
            return r;
        };
        return top(top(__uint_as_float(w.x), __uint_as_float(w.y)), top(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
}

template <bool BF16>
__global__ void __launch_bounds__(kAcceptThreads)
tree_accept_kernel(const void* __restrict__ logits, int n_cap, int vocab, int64_t row_stride, const int32_t* __restrict__ tokens,
                   const int32_t* __restrict__ parent, const int32_t* __restrict__ n_nodes, int32_t* __restrict__ path,
                   int32_t* __restrict__ n_accepted, int32_t* __restrict__ next_token) {
    constexpr int kPer = BF16 ? 8 : 4, kAtOnce = 8;          // logits per 16 bytes; loads in flight
    __shared__ uint2 sh_best[2][kAcceptCtas * kAcceptWarps]; // (key, index) per step parity and warp of the cluster
    __shared__ int sh_token[STC_TREE_MAX_NODES], sh_parent[STC_TREE_MAX_NODES];
    cg::cluster_group cluster = cg::this_cluster();
    const int b = blockIdx.x / kAcceptCtas, rank = (int)cluster.block_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = n_nodes ? min(max(n_nodes[b], 0), n_cap) : n_cap;
    if (threadIdx.x < n) {
        sh_token[threadIdx.x] = tokens[(size_t)b * n_cap + threadIdx.x];
        sh_parent[threadIdx.x] = parent ? parent[(size_t)b * n_cap + threadIdx.x] : (int)threadIdx.x - 1;
    }
    cluster.sync();                                          // every CTA runs, its shared memory can be written
    int node = n > 0 ? 0 : -1, count = 0, choice = -1;
    while (node >= 0) {
        if (rank == 0 && threadIdx.x == 0) path[(size_t)b * n_cap + count] = node;
        const char* row = static_cast<const char*>(logits) + ((size_t)b * n_cap + node) * row_stride * (BF16 ? 2 : 4);
        // the row from its first 16-byte boundary on, in 16-byte pieces dealt out in turn; the ends one by one
        const uint32_t head = min((uint32_t)vocab, (uint32_t)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / (BF16 ? 2u : 4u));
        const uint32_t pieces = ((uint32_t)vocab - head) / kPer, tail = head + pieces * kPer;
        const uint32_t me = (uint32_t)rank * kAcceptThreads + threadIdx.x;
        const uint4* src = reinterpret_cast<const uint4*>(row + head * (BF16 ? 2 : 4));
        // the piece with the thread's largest logit, the first of equal ones; within it the place is looked for once, at the end
        float top = 0.f;
        uint32_t top_at = 0xFFFFFFFFu;
        uint4 top_piece = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
        for (uint32_t i0 = me; i0 < pieces; i0 += kAtOnce * kAcceptCtas * kAcceptThreads) {
            uint4 w[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t i = i0 + (uint32_t)u * kAcceptCtas * kAcceptThreads;
                w[u] = ldg_nc16(src + (i < pieces ? i : i0));
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t i = i0 + (uint32_t)u * kAcceptCtas * kAcceptThreads;
                const float x = top_of<BF16>(w[u]);
                if (i < pieces && (top_at == 0xFFFFFFFFu || x > top || (x != x && top == top))) {
                    top = x;
                    top_at = i;
                    top_piece = w[u];
                }
            }
        }
        Best best;
        if (me < head) best.take(logit_at<BF16>(row, me), me);
        if (tail + me < (uint32_t)vocab) best.take(logit_at<BF16>(row, tail + me), tail + me);
        if (top_at != 0xFFFFFFFFu) {
            const uint32_t r[4] = {top_piece.x, top_piece.y, top_piece.z, top_piece.w};
            int at = kPer - 1;
#pragma unroll
            for (int e = kPer - 2; e >= 0; --e) {
                const float x = BF16 ? (e & 1 ? bf16hi(r[e / 2]) : bf16lo(r[e / 2])) : __uint_as_float(r[e % 4]);
                if (x == top || (x != x && top != top)) at = e;
            }
            best.take(top, head + top_at * kPer + at);
        }
        best.over_warp();
        if (lane < kAcceptCtas) *cluster.map_shared_rank(&sh_best[count & 1][rank * kAcceptWarps + warp], lane) = make_uint2(best.key, best.index);
        cluster.sync();
        best = Best();
#pragma unroll
        for (int i = 0; i < kAcceptCtas * kAcceptWarps / 32; ++i) {
            const uint2 of_warp = sh_best[count & 1][i * 32 + lane];
            best.take(of_warp.x, of_warp.y);
        }
        best.over_warp();
        choice = (int)best.index;
        ++count;
        // the lowest child with that token; every warp looks for itself
        int child = STC_TREE_MAX_NODES;
#pragma unroll
        for (int k = 0; k < STC_TREE_MAX_NODES / 32; ++k) {
            const int i = k * 32 + lane;
            if (i > node && i < n && sh_parent[i] == node && sh_token[i] == choice) child = min(child, i);
        }
        child = __reduce_min_sync(0xFFFFFFFFu, child);
        node = child < n ? child : -1;
    }
    if (rank == 0 && threadIdx.x == 0) {
        n_accepted[b] = count;
        next_token[b] = choice;
    }
    cluster.sync();                                          // no CTA leaves while another may still write to it
}

constexpr int kCommitThreads = 256;

template <int S>
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(const uint4* __restrict__ k_new, const uint4* __restrict__ v_new, const int32_t* __restrict__ n_nodes, int n_cap,
                   const int32_t* __restrict__ path, const int32_t* __restrict__ n_accepted, const int32_t* __restrict__ seq_len,
                   int Hkv, int T, int P, uint4* k, uint4* kmin, uint4* kmax, uint16_t* v_mask, uint32_t* v_offs, uint4* v_packed,
                   int64_t cap_groups, int32_t* __restrict__ new_len, int64_t* __restrict__ total_groups,
                   int32_t* __restrict__ status) {
    constexpr int OPG = kOctets / S;
    __shared__ int sh_node[STC_TREE_MAX_NODES];
    const int problem = blockIdx.x, b = problem / Hkv;
    const int len = clamp_len(seq_len, b, T), n = n_accepted[b];
    const int nodes = n_nodes ? min(max(n_nodes[b], 0), n_cap) : n_cap;
    bool bad = n < 0 || n > n_cap || n > T - len;
    if (!bad && threadIdx.x < n) {
        const int node = path[(size_t)b * n_cap + threadIdx.x];
        bad = node < 0 || node >= nodes;
        sh_node[threadIdx.x] = bad ? 0 : node;
    }
    uint32_t* offs = v_offs + (size_t)problem * (T + 1);
    const int64_t base = offs[len];
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        const int64_t total = base + (int64_t)n * S;
        if (!bad) total_groups[problem] = total;
        status[problem] = bad ? STC_ERR_INVALID_ARG : total > cap_groups ? STC_ERR_CAPACITY : STC_OK;
        if (problem == b * Hkv) new_len[b] = bad ? len : len + n;
    }
    if (bad) return;
    const uint4* kd = k_new + (size_t)problem * n_cap * kOctets;
    const uint4* vd = v_new + (size_t)problem * n_cap * kOctets;
    uint4* kc = k + (size_t)problem * T * kOctets;
    uint4* vp = v_packed + (size_t)problem * cap_groups * OPG;
    const int oct = threadIdx.x & 15;
#pragma unroll 2
    for (int i = threadIdx.x >> 4; i < n; i += kCommitThreads / 16) {
        const int node = sh_node[i];
        const uint4 key = ldg_nc16(kd + (size_t)node * kOctets + oct), value = ldg_nc16(vd + (size_t)node * kOctets + oct);
        kc[(size_t)(len + i) * kOctets + oct] = key;
        const int64_t first = base + (int64_t)i * S;
        if (first + oct / OPG < cap_groups) vp[first * OPG + oct] = value;
        if (oct == 0) {
            v_mask[(size_t)problem * T + len + i] = (uint16_t)((1u << S) - 1u);
            offs[len + i + 1] = (uint32_t)(first + S);
        }
    }
    if (!kmin || n == 0) return;
    // half a warp per touched page: old tokens from the cache, new ones from the draft
    for (int page = len / kPage + (int)(threadIdx.x >> 4); page <= (len + n - 1) / kPage; page += kCommitThreads / 16) {
        uint4 lo, hi;
        const int t0 = page * kPage, valid = min(kPage, len + n - t0);
        for (int t = 0; t < valid; ++t) {
            const int i = t0 + t - len;
            const uint4 r = i < 0 ? kc[(size_t)(t0 + t) * kOctets + oct] : ldg_nc16(kd + (size_t)sh_node[i] * kOctets + oct);
            if (t == 0) lo = hi = r;
            lo.x = bmin2(lo.x, r.x); hi.x = bmax2(hi.x, r.x);
            lo.y = bmin2(lo.y, r.y); hi.y = bmax2(hi.y, r.y);
            lo.z = bmin2(lo.z, r.z); hi.z = bmax2(hi.z, r.z);
            lo.w = bmin2(lo.w, r.w); hi.w = bmax2(hi.w, r.w);
        }
        kmin[((size_t)problem * P + page) * kOctets + oct] = lo;
        kmax[((size_t)problem * P + page) * kOctets + oct] = hi;
    }
}

}  // namespace

cudaError_t launch_tree_accept(int B, int n_cap, int vocab, const void* logits, bool bf16, int64_t row_stride, const int32_t* tokens,
                               const int32_t* parent, const int32_t* n_nodes, int32_t* path, int32_t* n_accepted,
                               int32_t* next_token, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)B * kAcceptCtas);
    cfg.blockDim = dim3(kAcceptThreads);
    cfg.stream = st;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = kAcceptCtas;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
    return bf16 ? cudaLaunchKernelEx(&cfg, tree_accept_kernel<true>, logits, n_cap, vocab, row_stride, tokens, parent, n_nodes, path,
                                     n_accepted, next_token)
                : cudaLaunchKernelEx(&cfg, tree_accept_kernel<false>, logits, n_cap, vocab, row_stride, tokens, parent, n_nodes, path,
                                     n_accepted, next_token);
}

cudaError_t launch_tree_commit(const Geom& g, const stc_tree& tree, const int32_t* path, const int32_t* n_accepted, void* k,
                               void* kmin, void* kmax, void* v_packed, uint16_t* v_mask, uint32_t* v_offs, int64_t cap_groups,
                               int32_t* new_len, int64_t* total_groups, int32_t* status, cudaStream_t st) {
#define STC_COMMIT(S_)                                                                                                       \
    case S_:                                                                                                                 \
        tree_commit_kernel<S_><<<g.problems, kCommitThreads, 0, st>>>(                                                       \
            static_cast<const uint4*>(tree.k), static_cast<const uint4*>(tree.v), tree.n_nodes, tree.n_cap, path,            \
            n_accepted, g.seq_len, g.Hkv, g.T, g.P, static_cast<uint4*>(k), static_cast<uint4*>(kmin),                       \
            static_cast<uint4*>(kmax), v_mask, v_offs, static_cast<uint4*>(v_packed), cap_groups, new_len, total_groups,     \
            status);                                                                                                         \
        break;
    switch (g.S) {
        STC_COMMIT(4) STC_COMMIT(8) STC_COMMIT(16)
        default: return cudaErrorInvalidValue;
    }
#undef STC_COMMIT
    return cudaGetLastError();
}

}  // namespace stc
