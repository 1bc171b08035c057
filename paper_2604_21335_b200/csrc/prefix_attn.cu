// Attention over shared prefixes: the sequences of a batch that continue the same cached prefix attend it
// together, so that the prefix is read once for all of them instead of once per sequence.
//
//   For every prefix g, KV head and query row r = (sequence, query head of that KV head) of the prefix's sequences:
//     s_t = sm_scale * q_r.k_t (+ options of stc_score),  p = softmax over the prefix's tokens of s
//     out_r = sum_t p_t v~_t   (v~: routed values, dropped groups zero),  lse_r = log sum exp s
//   optionally joined with (own_out, own_lse) of the sequence's own tokens by their log-sum-exps.
//
// Rows of one KV head form tiles of 128, tokens tiles of 128; both products run on the 5th-generation tensor
// cores with their accumulators in tensor memory:
//   S[row][token] = Q . K^T     Q, K tiles by TMA (128-byte swizzle), M = N = 128, K = 128
//   O[row][dim]  += P . V~      P from tensor memory, written over S by the softmax; V~ rebuilt from the packed
//                               groups in shared memory, token rows of 128 dims = N-major operand
// P enters as a bf16 high part plus a bf16 residual (two MMAs): the output is fp32, and one bf16 weight alone would
// leave it 2^-9 off; the pair leaves 2^-17.
//
// What bounds it.  Up to 128 rows per KV head the two products of a token tile take 1536 cycles of the tensor pipe
// and its bytes (K 32 KiB, V up to 32 KiB) 2100 to 2800 cycles of an SM's share of HBM: memory-bound; at 256 rows
// the pipe needs 3072 cycles and binds, so a work unit is at most two row tiles (one pass over K and V for 256
// rows) and larger batches take more units, whose K and V come from L2.
//
// Work split.  Unit = (prefix, KV head, block of up to two row tiles); the token tiles of all units form one flat
// sequence that is cut into equal contiguous ranges, one per CTA (one CTA per SM).  A CTA walks the segments of its
// range; a segment that is a whole unit is finished in place, another one leaves a partial (max, sum,
// accumulator) which a second small kernel joins in CTA order: no atomics, bitwise repeatable.
//
// Roles (16 warps): warp 0 = TMA producer of Q and K; warp 1 = MMA issuer; warps 4..7 and 8..11 = two softmax
// groups, thread = row; warps 12..15 rebuild the value tiles with 16-byte
// asynchronous copies straight from the packed store into the swizzled tile.  Two row tiles: group w owns row tile w and
// both see every token tile.  One row tile: the groups take the token tiles in turn, each with its own running
// maximum, sum and accumulator, joined at the end of the segment: the products of one overlap the softmax of the
// other in both modes.
//
// The running maximum only moves when a tile exceeds it by more than 2^8, so the accumulator in tensor memory is
// rescaled a few times per segment and not per tile; weights are then at most 2^8, far from fp32's limits.
//
// Every wait is bounded (about a second); one that expires raises a CTA-wide flag and STC_ERR_TIMEOUT in the
// status word, the roles leave, the producer waits (bounded) for its copies, tensor memory is freed.
#include "umma.cuh"

namespace stc {
namespace {

constexpr int kRows = 128;                        // rows per tile = tensor-memory lanes
constexpr int kTok = 128;                         // tokens per tile
constexpr int kThreads = 512;
constexpr int kKStages = 3;                       // key tiles of 128 tokens
constexpr int kVStages = 4;                       // value tiles of 64 tokens: finer, so that more of the ring is in flight
constexpr int kVTok = 64;
constexpr uint32_t kHalf = kRows * 128;           // 64 columns of a tile: 128 rows of 128 bytes
constexpr uint32_t kTile = 2 * kHalf;             // 32 KiB
constexpr uint32_t kVHalf = kVTok * 128, kVTile = 2 * kVHalf;
constexpr uint32_t kOffK = 2 * kTile, kOffV = kOffK + kKStages * kTile, kOffCtl = kOffV + kVStages * kVTile;
constexpr uint32_t kCtlBytes = 512 + 2 * kRows * 8;
constexpr uint32_t kSmem = kOffCtl + kCtlBytes;
static_assert(kSmem <= 232448, "shared memory of a block");
constexpr unsigned long long kWaitNs = 1000000000ull;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;                     // log2 units the maximum may be exceeded by

// barriers, in 8-byte words of the control block
enum { kQFull, kQEmpty, kKFull, kKEmpty = kKFull + kKStages, kVFull = kKEmpty + kKStages, kVEmpty = kVFull + kVStages,
       kSFull = kVEmpty + kVStages, kPFull = kSFull + 2, kOFull = kPFull + 2, kXchg = kOFull + 2, kBars };
static_assert(kBars * 8 <= 256, "control block");

struct PrefixArgs {
    const int32_t* row_start;    // [G + 1]
    const int32_t* seq_len;
    const uint16_t* v_mask;
    const uint32_t* v_offs;
    const uint4* v_packed;
    const float* own_out;        // or nullptr
    const float* own_lse;
    float* out;
    float* lse;                  // or nullptr
    int32_t* status;
    long long* base;             // [G + 2]: first flat tile of each prefix; [G] = total; [G + 1] = 1 if row_start is bad
    float* part_o;               // [2 * grid][slot_rows][128]
    float2* part_ml;             // [2 * grid][slot_rows]
    int64_t cap_groups;
    int G, Hq, Hkv, Gq, T, n_rows, slot_rows;
    int seqs;                    // sequences per row tile = 128 / Gq
    float scale_log2, cap_in, cap_log2;
    ScoreArgs sc;
};

// 2^x to 2 units of fp32; results below the normal range become zero.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Group {
    int row0, n_seq, len, tiles, blocks;
};
__device__ __forceinline__ Group load_group(const PrefixArgs& a, int g) {
    Group r;
    r.row0 = a.row_start[g];
    r.n_seq = a.row_start[g + 1] - r.row0;
    r.len = clamp_len(a.seq_len, g, a.T);
    r.tiles = (r.len + kTok - 1) / kTok;
    r.blocks = (r.n_seq + 2 * a.seqs - 1) / (2 * a.seqs);
    return r;
}
__device__ __forceinline__ long long group_tiles(const PrefixArgs& a, const Group& g) {
    return (long long)g.tiles * g.blocks * a.Hkv;
}

// One segment: tiles [tile0, tile1) of one unit.
struct Segment {
    int g, hk, row0, n_seq, len, tile0, tile1;
    int slot;                    // partial slot, -1 = the whole unit
};
// Walks the segments of the CTA's range [x, x_end).
struct Walker {
    long long x, x_end, x_begin, off;  // off = x - base of group g
    int g;
    Group grp;
    bool loaded;
    __device__ __forceinline__ bool next(const PrefixArgs& a, Segment& s) {
        if (x >= x_end) return false;
        if (!loaded) { grp = load_group(a, g); loaded = true; }
        while (off >= group_tiles(a, grp)) {
            off -= group_tiles(a, grp);
            grp = load_group(a, ++g);
        }
        const long long unit = off / grp.tiles;
        s.tile0 = (int)(off - unit * grp.tiles);
        const long long left = x_end - x;
        s.tile1 = (int)min((long long)grp.tiles, s.tile0 + left);
        s.hk = (int)(unit / grp.blocks);
        const int blk = (int)(unit - (long long)s.hk * grp.blocks);
        s.g = g;
        s.row0 = grp.row0 + blk * 2 * a.seqs;
        s.n_seq = min(2 * a.seqs, grp.n_seq - blk * 2 * a.seqs);
        s.len = grp.len;
        const bool whole = s.tile0 == 0 && s.tile1 == grp.tiles;
        s.slot = whole ? -1 : 2 * (int)blockIdx.x + (x == x_begin ? 0 : 1);
        const int n = s.tile1 - s.tile0;
        x += n;
        off += n;
        return true;
    }
};

// Joins an attention result (m in log2 units, l, unnormalised o) with the sequence's own (own, own_lse): factors
// for o and own, and the joined lse.  An empty side gets the factor 0 and is not to be multiplied.
struct Join { float fo, fown, lse; };
__device__ __forceinline__ Join join(float m, float l, float shift, bool has_own, float own_lse) {
    const float a2 = l > 0.f ? m + log2f(l) + shift * kLog2e : -INFINITY;
    const float b2 = has_own ? own_lse * kLog2e : -INFINITY;
    const float top = fmaxf(a2, b2);
    if (!(top > -INFINITY)) return Join{0.f, 0.f, -INFINITY};
    const float wa = exp2f(a2 - top), wb = exp2f(b2 - top), inv = 1.f / (wa + wb);
    return Join{l > 0.f ? wa * inv / l : 0.f, wb * inv, (top + log2f(wa + wb)) * kLn2};
}

// lse of the scores lacks slope * (reference - position): the bias is taken against the last visible token.
__device__ __forceinline__ float bias_shift(const PrefixArgs& a, int len, int seq, int head) {
    if (!a.sc.slopes) return 0.f;
    int lo, hi;
    const int pos = a.sc.q_pos[seq];
    visible_range(len, pos, a.sc.window, lo, hi);
    return a.sc.slopes[head] * (float)(hi - 1 - pos);
}

// Caps 16 scores of a row (raw products in, log2 units out).  Scores far below the cap, the usual case, need only the
// polynomial of tanh_f32; the warp votes once per 16 instead of branching per score.
__device__ __forceinline__ void cap_scores(uint32_t (&r)[16], float cap_in, float cap_log2) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) big = fmaxf(big, fabsf(__uint_as_float(r[i])));
    const bool small = __all_sync(0xFFFFFFFFu, big * fabsf(cap_in) <= kTanhSmall);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {                // tanh_small, two at a time
        const float2 z = mul2(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), both(cap_in));
        const float2 u = mul2(z, z);
        float2 p = fma2(both(kTanh4), u, both(kTanh3));
        p = fma2(p, u, both(kTanh2));
        p = fma2(p, u, both(kTanh1));
        p = fma2(p, u, both(kTanh0));
        const float2 t = fma2(mul2(z, u), p, z);
        float2 y = mul2(t, both(cap_log2));
        if (!small) {                                // uniform
            if (fabsf(z.x) > kTanhSmall) y.x = cap_log2 * tanh_large(z.x);
            if (fabsf(z.y) > kTanhSmall) y.y = cap_log2 * tanh_large(z.y);
        }
        r[i] = __float_as_uint(y.x);
        r[i + 1] = __float_as_uint(y.y);
    }
}

// CAP: capped scores; BIAS: finished scores are needed for the maximum (slopes, or a scale that is not positive).
// The window, positions and documents of the rows are masks and looked at in every variant.
template <int S, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const PrefixArgs a) {
    constexpr int OPG = kOctets / S;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const uint32_t bars = base + kOffCtl;
    unsigned char* ctl = smem + kOffCtl;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctl + 256);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctl + 260);
    volatile long long* plan = reinterpret_cast<volatile long long*>(ctl + 272);      // x, x_end, off, g
    float2* ml = reinterpret_cast<float2*>(ctl + 512);                                // [2][128]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // ---- set-up: barriers, tensor memory, this CTA's range ------------------------------------------
    if (threadIdx.x == 0) {
        mbar_init(bars + 8 * kQFull, 1);
        mbar_init(bars + 8 * kQEmpty, 1);
        for (int i = 0; i < kKStages; ++i) { mbar_init(bars + 8 * (kKFull + i), 1); mbar_init(bars + 8 * (kKEmpty + i), 1); }
        for (int i = 0; i < kVStages; ++i) { mbar_init(bars + 8 * (kVFull + i), 2); mbar_init(bars + 8 * (kVEmpty + i), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bars + 8 * (kSFull + i), 1);
            mbar_init(bars + 8 * (kPFull + i), kRows);
            mbar_init(bars + 8 * (kOFull + i), 1);
        }
        mbar_init(bars + 8 * kXchg, 2 * kRows);
        *abort_flag = (base & 1023u) != 0;           // swizzled tiles need 1024-byte aligned bases
        if (base & 1023u) atomicExch(a.status, (int)STC_ERR_CUDA);
        fence_mbar_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(bars + 256), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 2) {                                 // flat tile sequence: prefix sums over the prefixes, 32 at a time
        long long total = 0;
        bool bad = false;
        auto scan = [&](auto&& use) {
            long long run = 0;
            for (int g0 = 0; g0 < a.G; g0 += 32) {
                const int g = g0 + lane;
                long long n = 0;
                if (g < a.G) {
                    const int r0 = a.row_start[g], r1 = a.row_start[g + 1];
                    if (r0 < 0 || r1 < r0 || r1 > a.n_rows) bad = true;
                    else n = group_tiles(a, load_group(a, g));
                }
                long long incl = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const long long o = __shfl_up_sync(0xFFFFFFFFu, incl, d);
                    if (lane >= d) incl += o;
                }
                use(g, run + incl - n, run + incl);
                run += __shfl_sync(0xFFFFFFFFu, incl, 31);
            }
            return run;
        };
        total = scan([&](int g, long long lo, long long) {
            if (blockIdx.x == 0 && g < a.G) a.base[g] = lo;
        });
        bad = __any_sync(0xFFFFFFFFu, bad);
        if (bad) total = 0;
        const long long lo = total * blockIdx.x / gridDim.x, hi = total * (blockIdx.x + 1) / gridDim.x;
        if (lane == 0) {
            plan[0] = lo; plan[1] = hi; plan[2] = 0; plan[3] = 0;
            if (blockIdx.x == 0) {
                a.base[a.G] = total;
                a.base[a.G + 1] = bad;
                if (bad) atomicExch(a.status, (int)STC_ERR_INVALID_ARG);
            }
        }
        __syncwarp();
        if (hi > lo)
            scan([&](int g, long long first, long long end) {
                if (g < a.G && first <= lo && lo < end) { plan[2] = lo - first; plan[3] = g; }
            });
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_slot;
    Walker walk;
    walk.x = walk.x_begin = plan[0];
    walk.x_end = plan[1];
    walk.off = plan[2];
    walk.g = (int)plan[3];
    walk.loaded = false;
    Segment s;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto wait = [&](int i, uint32_t parity) { return mbar_wait_or_abort(bar(i), parity & 1u, abort_flag, kWaitNs); };
    // the same for a whole warp: lane 0 waits and hands the answer on
    auto warp_wait = [&](int i, uint32_t parity) -> bool {
        int got = 0;
        if (lane == 0) got = wait(i, parity);
        return __shfl_sync(0xFFFFFFFFu, got, 0) != 0;
    };
    auto give_up = [&]() { *abort_flag = 1; atomicCAS(a.status, 0, (int)STC_ERR_TIMEOUT); };

    if (*abort_flag) {
        // nothing was started
    } else if (warp == 0) {
        // ---- producer of Q and K ---------------------------------------------------------------------
        if (lane == 0) {
            int kc = 0, seg = 0;
            bool ok = true;
            const uint32_t q_bytes = 2u * 128u * (uint32_t)(a.Gq * a.seqs);       // per row tile
            while (ok && walk.next(a, s)) {
                const int row_tiles = s.n_seq > a.seqs ? 2 : 1;
                if (seg > 0 && !wait(kQEmpty, (uint32_t)(seg - 1))) { give_up(); break; }
                mbar_expect_tx(bar(kQFull), q_bytes * row_tiles);
                for (int i = 0; i < row_tiles; ++i)
                    for (int h = 0; h < 2; ++h)
                        tma_3d(base + i * kTile + h * kHalf, &map_q, 64 * h, s.hk * a.Gq, s.row0 + i * a.seqs, bar(kQFull));
                ++seg;
                const int row = (s.g * a.Hkv + s.hk) * a.T;
                for (int t = s.tile0; t < s.tile1; ++t, ++kc) {
                    const int st = kc % kKStages;
                    if (kc >= kKStages && !wait(kKEmpty + st, (uint32_t)(kc / kKStages - 1))) { give_up(); ok = false; break; }
                    mbar_expect_tx(bar(kKFull + st), kTile);
                    for (int h = 0; h < 2; ++h)
                        tma_2d(base + kOffK + st * kTile + h * kHalf, &map_k, 64 * h, row + t * kTok, bar(kKFull + st));
                }
            }
            if (*abort_flag) {                       // copies still in flight get one more bounded wait each
                int none = 0;
                if (seg > 0) mbar_wait_or_abort(bar(kQFull), (uint32_t)(seg - 1) & 1u, &none, kWaitNs);
                for (int i = max(0, kc - kKStages); i < kc; ++i)
                    mbar_wait_or_abort(bar(kKFull + i % kKStages), (uint32_t)(i / kKStages) & 1u, &none, kWaitNs);
            }
        }
    } else if (warp == 1) {
        // ---- MMA issuer ----------------------------------------------------------------------------------
        // (loops are kept rolled here and in the other roles: the roles of an SM partition share its small first-level
        // instruction cache, and unrolled they evict each other; the issuer then took 3200 cycles per step)
        if (lane == 0) {
            constexpr uint32_t id_qk = idesc_bf16(kRows, kTok, false), id_pv = idesc_bf16(kRows, kHeadDim, true);
            int kc0 = 0, seg = 0;                    // tiles of the segments before; segments before
            uint32_t n_o0 = 0, n_o1 = 0;             // P tiles consumed per group
            bool ok = true;
            while (ok && walk.next(a, s)) {
                const int tiles = s.tile1 - s.tile0;
                const bool two = s.n_seq > a.seqs;   // two row tiles: every token tile goes to both groups
                const int steps = two ? 2 * tiles : tiles;
                if (!wait(kQFull, (uint32_t)seg)) { ok = false; break; }
                // step i belongs to group w = i & 1; it is S = Q K^T now, and O += P V two iterations on
#pragma unroll 1
                for (int n = 0; n < steps + 2; ++n) {
                    const int w = n & 1;
                    const uint32_t n_o = w ? n_o1 : n_o0;
                    const uint32_t ts = tmem + (uint32_t)w * 128u;
                    if (n >= 2) {                    // O += P V of step n - 2
                        const int j = kc0 + (two ? (n - 2) >> 1 : n - 2);
                        ok = wait(kPFull + w, n_o);
                        uint32_t acc = n >= 4;       // the group's first product of a segment starts O anew
#pragma unroll 1
                        for (int jv = 2 * j; ok && jv < 2 * j + 2; ++jv) {   // two value tiles of 64 tokens
                            const int st = jv % kVStages;
                            if (!two || w == 0) ok = wait(kVFull + st, (uint32_t)(jv / kVStages));
                            tc_after();
                            uint64_t dv = smem_desc_128(base + kOffV + st * kVTile, kVHalf);
                            uint32_t pk = ts + 64u * (jv & 1);
#pragma unroll 1
                            for (int k = 0; k < 4; ++k) {    // 16 tokens: 16 rows of 128 bytes; P: 8 columns high, 8 residual
                                tc_mma_ts(ts + 256, pk, dv, id_pv, acc);
                                tc_mma_ts(ts + 256, pk + 8, dv, id_pv, 1);
                                acc = 1;
                                pk += 16;
                                dv += 2048 >> 4;
                            }
                            if (!two || w == 1) tc_commit_to(bar(kVEmpty + st));
                        }
                        if (!ok) break;
                        tc_commit_to(bar(kOFull + w));
                        if (w) ++n_o1; else ++n_o0;
                    }
                    if (n < steps) {                 // S = Q K^T of step n
                        const int j = kc0 + (two ? n >> 1 : n), st = j % kKStages;
                        if (!two || w == 0) ok = wait(kKFull + st, (uint32_t)(j / kKStages));
                        // S and P share their columns: the product that read the group's last P has to be through
                        const uint32_t done = w ? n_o1 : n_o0;
                        if (ok && done > 0) ok = wait(kOFull + w, done - 1);
                        if (!ok) break;
                        tc_after();
                        uint64_t dq = smem_desc_128(base + (two ? w * kTile : 0u), 16);
                        uint64_t dk = smem_desc_128(base + kOffK + st * kTile, 16);
#pragma unroll 1
                        for (int k = 0; k < 2; ++k) {        // 64 dims: one half tile
#pragma unroll
                            for (int e = 0; e < 4; ++e)      // 16 dims: 32 bytes, 2 units
                                tc_mma_ss(ts, dq + 2 * e, dk + 2 * e, id_qk, k + e != 0);
                            dq += kHalf >> 4;
                            dk += kHalf >> 4;
                        }
                        tc_commit_to(bar(kSFull + w));
                        if (!two || w == 1) tc_commit_to(bar(kKEmpty + st));
                        if (n == steps - 1) tc_commit_to(bar(kQEmpty));
                    }
                }
                kc0 += tiles;
                ++seg;
            }
            if (!ok) give_up();
        }
    } else if (warp >= 4 && warp < 12) {
        // ---- softmax: thread = row -----------------------------------------------------------------------
        const int w = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t ts = lane_base + w * 128, to = lane_base + 256 + w * 128;
        uint32_t n_s = 0, n_x = 0;
        bool ok = true;
        while (ok && walk.next(a, s)) {
            const int tiles = s.tile1 - s.tile0;
            const bool two = s.n_seq > a.seqs;
            const int mine = two ? tiles : (tiles + 1 - w) >> 1, stride = two ? 1 : 2, first = s.tile0 + (two ? 0 : w);
            // this thread's row: sequence and head
            const int in_tile = row / a.Gq, seq_i = (two ? w * a.seqs : 0) + in_tile;
            const bool live = in_tile < a.seqs && seq_i < s.n_seq;
            const int seq = s.row0 + (live ? seq_i : 0), head = s.hk * a.Gq + row % a.Gq;
            int lo = 0, hi = s.len, my_doc = 0;
            float slope2 = 0.f;
            if (a.sc.q_pos) visible_range(s.len, a.sc.q_pos[seq], a.sc.window, lo, hi);
            if (BIAS && a.sc.slopes) slope2 = a.sc.slopes[head] * kLog2e;
            const int32_t* doc = a.sc.tok_doc ? a.sc.tok_doc + (size_t)s.g * a.T : nullptr;
            if (doc) my_doc = a.sc.q_doc[seq];
            // -inf for the tokens t .. t + 15 that the row does not see
            auto hide = [&](uint32_t (&r)[16], int t) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (t + i < lo || t + i >= hi) r[i] = __float_as_uint(-INFINITY);
                if (doc) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int d = __ldg(doc + min(t + i, a.T - 1));
                        if (d >= 0 && d != my_doc) r[i] = __float_as_uint(-INFINITY);
                    }
                }
            };
            float m = -INFINITY, l = 0.f;
            for (int n = 0; n < mine; ++n) {
                ok = warp_wait(kSFull + w, n_s);
                if (!ok) break;
                tc_after();
                const int t0 = (first + n * stride) * kTok;
                // does every row of the warp see the whole tile?
                const bool open = __all_sync(0xFFFFFFFFu, lo <= t0 && hi >= t0 + kTok) && !doc;
                // pass 1: the tile's maximum.  A cap alone keeps the order, so the raw products do; with a bias the finished
                // scores are compared, and kept if capping them again would cost more than tensor memory
                float top = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < kTok; c += 16) {
                    uint32_t r[16];
                    tmem_ld16(ts + c, r);
                    tmem_wait_ld();
                    if constexpr (BIAS) {
                        const float far = (float)(t0 + c - (hi - 1));
                        if constexpr (CAP) cap_scores(r, a.cap_in, a.cap_log2);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x = CAP ? __uint_as_float(r[i]) : __uint_as_float(r[i]) * a.scale_log2;
                            r[i] = __float_as_uint(fmaf(slope2, far + (float)i, x));
                        }
                    }
                    if (!open) hide(r, t0 + c);
                    if constexpr (CAP && BIAS) tmem_st16(ts + c, r);
                    float t2[2] = {top, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 16; i += 2)
                        t2[(i >> 1) & 1] = fmaxf(fmaxf(t2[(i >> 1) & 1], __uint_as_float(r[i])), __uint_as_float(r[i + 1]));
                    top = fmaxf(t2[0], t2[1]);
                }
                if constexpr (CAP && BIAS) tmem_wait_st();
                if constexpr (!BIAS)
                    if (top > -INFINITY) top = CAP ? a.cap_log2 * tanh_f32(top * a.cap_in) : top * a.scale_log2;
                // move the maximum only if it is exceeded by much; the accumulator follows
                const bool move = top > m + kSlack || (m == -INFINITY && top > -INFINITY);
                if (__any_sync(0xFFFFFFFFu, move)) {
                    const float to_m = move ? top : m;
                    const float f = (m == -INFINITY) ? 0.f : exp2f(m - to_m);
                    l *= f;
                    if (n > 0) {
#pragma unroll 1
                        for (int c = 0; c < kHeadDim; c += 16) {
                            uint32_t r[16];
                            tmem_ld16(to + c, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                r[i] = move ? __float_as_uint(__uint_as_float(r[i]) * f) : r[i];
                            tmem_st16(to + c, r);
                        }
                    }
                    m = to_m;
                }
                // pass 2: weights, their sum, and P over S: per 16 tokens 8 columns of bf16 pairs high, 8 residual
                const float ref = m == -INFINITY ? 0.f : m;
                float2 la = make_float2(0.f, 0.f), lb = la;
#pragma unroll 1
                for (int c = 0; c < kTok; c += 16) {
                    uint32_t r[16];
                    tmem_ld16(ts + c, r);
                    tmem_wait_ld();
                    if constexpr (CAP && !BIAS) cap_scores(r, a.cap_in, a.cap_log2);
                    const float far = (float)(t0 + c - (hi - 1));
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float2 x = make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                        float2 y;
                        if constexpr (CAP) y = add2(x, both(-ref));
                        else if constexpr (BIAS)
                            y = fma2(x, both(a.scale_log2), fma2(both(slope2), make_float2(far + (float)i, far + (float)(i + 1)), both(-ref)));
                        else y = fma2(x, both(a.scale_log2), both(-ref));
                        r[i] = __float_as_uint(y.x);
                        r[i + 1] = __float_as_uint(y.y);
                    }
                    if (!(CAP && BIAS) && !open) hide(r, t0 + c);
                    uint32_t o[16];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 p = make_float2(ex2(__uint_as_float(r[2 * i])), ex2(__uint_as_float(r[2 * i + 1])));
                        if (i & 1) lb = add2(lb, p); else la = add2(la, p);
                        const __nv_bfloat162 h2 = __floats2bfloat162_rn(p.x, p.y);
                        o[i] = *reinterpret_cast<const uint32_t*>(&h2);
                        const float2 d = fma2(make_float2(bf16lo(o[i]), bf16hi(o[i])), both(-1.f), p);
                        const __nv_bfloat162 r2 = __floats2bfloat162_rn(d.x, d.y);
                        o[8 + i] = *reinterpret_cast<const uint32_t*>(&r2);
                    }
                    tmem_st16(ts + c, o);
                }
                l += (la.x + lb.x) + (la.y + lb.y);
                tmem_wait_st();
                tc_before();
                mbar_arrive(bar(kPFull + w));
                ++n_s;
            }
            if (!ok) break;
            // ---- end of the segment -----------------------------------------------------------------------
            if (mine > 0) {
                ok = warp_wait(kOFull + w, n_s - 1);
                if (!ok) break;
                tc_after();
            }
            float mo = m, lo_sum = l, f0 = 1.f, f1 = 0.f;   // joined maximum and sum; factors of accumulator 0 / 1
            bool has1 = false;
            int c_lo = 0, c_hi = kHeadDim;                   // dims this thread writes
            uint32_t acc0 = to, acc1 = to;
            if (!two) {                              // both groups hold part of the same rows: join, half the dims each
                ml[w * kRows + row] = make_float2(m, l);
                tc_before();
                mbar_arrive(bar(kXchg));
                ok = warp_wait(kXchg, n_x++);
                if (!ok) break;
                tc_after();
                const float2 a0 = ml[row], a1 = ml[kRows + row];
                mo = fmaxf(a0.x, a1.x);
                f0 = a0.x == -INFINITY ? 0.f : exp2f(a0.x - mo);
                f1 = a1.x == -INFINITY ? 0.f : exp2f(a1.x - mo);
                lo_sum = a0.y * f0 + a1.y * f1;
                has1 = tiles > 1;
                acc0 = lane_base + 256;
                acc1 = lane_base + 384;
                c_lo = 64 * w;
                c_hi = c_lo + 64;
            }
            const size_t out_row = (size_t)seq * a.Hq + head;
            float fo = 1.f, fown = 0.f;
            const float* own = nullptr;
            float* dst;
            if (s.slot < 0) {
                const Join j = join(mo, lo_sum, BIAS ? bias_shift(a, s.len, seq, head) : 0.f, a.own_lse != nullptr,
                                    a.own_lse ? a.own_lse[out_row] : 0.f);
                fo = j.fo;
                fown = j.fown;
                if (a.own_out && fown != 0.f) own = a.own_out + out_row * kHeadDim;
                dst = a.out + out_row * kHeadDim;
                if (live && a.lse && c_lo == 0) a.lse[out_row] = j.lse;
            } else {
                const size_t slot = (size_t)s.slot * a.slot_rows + (two ? w * a.seqs * a.Gq : 0) + row;
                dst = a.part_o + slot * kHeadDim;
                if (live && c_lo == 0) a.part_ml[slot] = make_float2(mo, lo_sum);
            }
#pragma unroll 1
            for (int c = c_lo; c < c_hi; c += 16) {
                uint32_t r0[16], r1[16];
                tmem_ld16(acc0 + c, r0);
                if (has1) tmem_ld16(acc1 + c, r1);
                tmem_wait_ld();
                if (live) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] = f0 != 0.f ? __uint_as_float(r0[i + e]) * f0 : 0.f;
                            if (has1 && f1 != 0.f) v[e] = fmaf(__uint_as_float(r1[i + e]), f1, v[e]);
                            v[e] = fo != 0.f ? v[e] * fo : 0.f;
                        }
                        float4 v4 = make_float4(v[0], v[1], v[2], v[3]);
                        if (own) {
                            const float4 w4 = *reinterpret_cast<const float4*>(own + c + i);
                            v4.x = fmaf(w4.x, fown, v4.x); v4.y = fmaf(w4.y, fown, v4.y);
                            v4.z = fmaf(w4.z, fown, v4.z); v4.w = fmaf(w4.w, fown, v4.w);
                        }
                        *reinterpret_cast<float4*>(dst + c + i) = v4;
                    }
                }
            }
            if (!two) {                              // the other group's accumulator and the exchange are free again
                tc_before();
                mbar_arrive(bar(kXchg));
                ok = warp_wait(kXchg, n_x++);
                tc_after();
            }
        }
        if (!ok) give_up();
    } else if (warp >= 12) {
        // ---- value tiles: packed groups -> swizzled rows ---------------------------------------------------
        // Warps 12, 13 build the even tiles of 64 tokens and 14, 15 the odd ones, 32 tokens each.  A lane owns one
        // 16-byte column of every other token; a kept group is one asynchronous 16-byte copy, a dropped one a
        // zero-filled copy that reads nothing.  The copies of a warp's next tile are under way before the last
        // one's are waited for, unless its stage is still being read.
        const int pair = (warp - 12) >> 1, tok0 = (warp & 1) * 32, oct = lane & 15, grp = oct / OPG, sub = oct % OPG;
        const uint32_t below = (1u << grp) - 1u;
        int vc = 0;                                  // tiles of 64 tokens so far, both pairs'
        int pending = -1;                            // stage whose copies are not waited for yet
        bool ok = true;
        auto publish = [&]() {                       // this warp's copies into `pending` have landed
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kVFull + pending));
            pending = -1;
        };
        while (ok && walk.next(a, s)) {
            const size_t problem = (size_t)s.g * a.Hkv + s.hk;
            const uint16_t* mask_row = a.v_mask + problem * a.T;
            const uint32_t* offs = a.v_offs + problem * (a.T + 1);
            const uint4* packed = a.v_packed + problem * a.cap_groups * OPG;
            const int64_t limit = a.cap_groups;
            const int n_half = 2 * (s.tile1 - s.tile0), first_tok = s.tile0 * kTok + tok0;
            auto fetch = [&](int h, uint32_t& m, uint32_t& first) {        // this lane's token mask, the warp's first group
                const int t = first_tok + h * kVTok;
                m = h < n_half && t + lane < s.len ? mask_row[t + lane] : 0u;
                first = h < n_half && t < s.len ? offs[t] : 0u;
            };
            uint32_t m_next, first_next;
            fetch(pair, m_next, first_next);         // a segment is an even number of tiles of 64 tokens
            for (int h = pair; h < n_half; h += 2) {
                const uint32_t m = m_next & ((1u << S) - 1u), first = first_next;
                fetch(h + 2, m_next, first_next);
                const uint32_t cnt = __popc(m);
                const uint32_t pre = warp_incl_scan(cnt, lane) - cnt;
                const int j = vc + h, st = j % kVStages;
                if (j >= kVStages) {
                    const uint32_t par = (uint32_t)(j / kVStages - 1) & 1u;
                    int free = 0;
                    if (lane == 0) free = mbar_try_wait(bar(kVEmpty + st), par);
                    if (!__shfl_sync(0xFFFFFFFFu, free, 0)) {
                        if (pending >= 0) { cp_async_wait<0>(); publish(); }
                        ok = warp_wait(kVEmpty + st, par);
                        if (!ok) break;
                    }
                }
                const uint32_t dst = base + kOffV + st * kVTile + (uint32_t)(oct >> 3) * kVHalf;
#pragma unroll 4
                for (int i = 0; i < 16; ++i) {
                    const int tok = 2 * i + (lane >> 4);
                    const uint32_t mt = __shfl_sync(0xFFFFFFFFu, m, tok), pt = __shfl_sync(0xFFFFFFFFu, pre, tok);
                    const int64_t at = (int64_t)first + pt + __popc(mt & below);
                    const bool kept = ((mt >> grp) & 1u) && at < limit;
                    cp_async16_zfill(dst + (uint32_t)(tok0 + tok) * 128u + (uint32_t)(((oct & 7) ^ (tok & 7)) * 16),
                                     kept ? packed + at * OPG + sub : packed, kept ? 16 : 0);
                }
                cp_async_commit();
                if (pending >= 0) { cp_async_wait<1>(); publish(); }
                pending = st;
            }
            vc += n_half;
        }
        cp_async_wait<0>();
        if (ok && pending >= 0) publish();
        if (!ok) give_up();
    }
    tc_before();
    __syncthreads();
    if (warp == 1) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Joins the partials of units that more than one CTA worked on, and answers the rows whose prefix is empty.
// One warp per (row, query head), a lane four channels; partials in CTA order.
__global__ void __launch_bounds__(256)
prefix_merge_kernel(const PrefixArgs a, int n_cta) {
    const long long task = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (task >= (long long)a.n_rows * a.Hq || a.base[a.G + 1] != 0) return;
    const int seq = (int)(task / a.Hq), head = (int)(task - (long long)seq * a.Hq);
    if (seq < a.row_start[0] || seq >= a.row_start[a.G]) return;
    int g = 0, g_hi = a.G;                           // last prefix that starts at or before the row
    while (g_hi - g > 1) {
        const int mid = (g + g_hi) >> 1;
        if (a.row_start[mid] <= seq) g = mid; else g_hi = mid;
    }
    const Group grp = load_group(a, g);
    const int hk = head / a.Gq, in_group = seq - grp.row0, blk = in_group / (2 * a.seqs);
    const int row = (in_group - blk * 2 * a.seqs) * a.Gq + head % a.Gq;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (grp.tiles > 0) {
        const long long total = a.base[a.G];
        const long long x0 = a.base[g] + ((long long)hk * grp.blocks + blk) * grp.tiles, x1 = x0 + grp.tiles;
        const long long c0 = ((x0 + 1) * n_cta + total - 1) / total - 1, c1 = (x1 * n_cta + total - 1) / total - 1;
        if (c0 == c1) return;                        // a whole unit: done where it was computed
        // a range that begins inside the unit used its first slot; with fewer tiles than CTAs some ranges are empty
        auto slot_of = [&](long long c) -> long long {
            const long long lo = total * c / n_cta, hi = total * (c + 1) / n_cta;
            return lo < hi ? (2 * c + (lo >= x0 ? 0 : 1)) * a.slot_rows + row : -1;
        };
        for (long long c = c0; c <= c1; ++c) {
            const long long slot = slot_of(c);
            if (slot >= 0) m = fmaxf(m, a.part_ml[slot].x);
        }
        for (long long c = c0; c <= c1; ++c) {
            const long long slot = slot_of(c);
            if (slot < 0) continue;
            const float2 p = a.part_ml[slot];
            if (p.x == -INFINITY) continue;
            const float f = exp2f(p.x - m);
            const float4 v = reinterpret_cast<const float4*>(a.part_o + slot * kHeadDim)[lane];
            l = fmaf(p.y, f, l);
            o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
        }
    }
    const size_t out_row = (size_t)seq * a.Hq + head;
    const Join j = join(m, l, bias_shift(a, grp.len, seq, head), a.own_lse != nullptr,
                        a.own_lse ? a.own_lse[out_row] : 0.f);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j.fo != 0.f) v = make_float4(o.x * j.fo, o.y * j.fo, o.z * j.fo, o.w * j.fo);
    if (a.own_out && j.fown != 0.f) {
        const float4 w = reinterpret_cast<const float4*>(a.own_out + out_row * kHeadDim)[lane];
        v.x = fmaf(w.x, j.fown, v.x); v.y = fmaf(w.y, j.fown, v.y); v.z = fmaf(w.z, j.fown, v.z); v.w = fmaf(w.w, j.fown, v.w);
    }
    reinterpret_cast<float4*>(a.out + out_row * kHeadDim)[lane] = v;
    if (a.lse && lane == 0) a.lse[out_row] = j.lse;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// The workspace has to be sized without a device, so the partial slots are counted for this many CTAs.
constexpr int kPlanSms = 148;

int slot_rows(const Geom& g, int n_rows) {
    const long long rows = (long long)n_rows * g.Gq, most = 2LL * (kRows / g.Gq) * g.Gq;
    return (int)(rows < most ? rows : most);
}

}  // namespace

size_t prefix_ws_bytes(const Geom& g, int n_rows) {
    const size_t slots = 2 * (size_t)kPlanSms * slot_rows(g, n_rows);
    return 256 + align256(((size_t)g.B + 2) * 8) + align256(slots * 8) + align256(slots * kHeadDim * 4);
}

cudaError_t launch_prefix_attn(const Geom& g, const void* k, const void* v_packed, const uint16_t* v_mask,
                               const uint32_t* v_offs, int64_t cap_groups, int n_rows, const void* q,
                               const int32_t* row_start, float sm_scale, const ScoreArgs* score, const float* own_out,
                               const float* own_lse, float* out, float* lse, void* ws, cudaStream_t st) {
    char* w = static_cast<char*>(ws);
    PrefixArgs a;
    a.row_start = row_start; a.seq_len = g.seq_len;
    a.v_mask = v_mask; a.v_offs = v_offs; a.v_packed = static_cast<const uint4*>(v_packed);
    a.own_out = own_out; a.own_lse = own_lse; a.out = out; a.lse = lse;
    a.status = reinterpret_cast<int32_t*>(w);
    w += 256;
    a.base = reinterpret_cast<long long*>(w);
    w += align256(((size_t)g.B + 2) * 8);
    a.slot_rows = slot_rows(g, n_rows);
    a.part_ml = reinterpret_cast<float2*>(w);
    w += align256(2 * (size_t)kPlanSms * a.slot_rows * 8);
    a.part_o = reinterpret_cast<float*>(w);
    a.cap_groups = cap_groups;
    a.G = g.B; a.Hq = g.Hq; a.Hkv = g.Hkv; a.Gq = g.Gq; a.T = g.T; a.n_rows = n_rows;
    a.seqs = kRows / g.Gq;
    a.sc = score ? *score : ScoreArgs{};
    a.scale_log2 = sm_scale * kLog2e;
    a.cap_in = a.sc.softcap > 0.f ? sm_scale / a.sc.softcap : 0.f;
    a.cap_log2 = a.sc.softcap * kLog2e;
    int sms = 0;
    cudaError_t e = device_sm_count(&sms);
    if (e != cudaSuccess) return e;
    const int n_cta = sms < kPlanSms ? sms : kPlanSms;

    EncodeTiled enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    CUtensorMap map_q, map_k;
    {
        const cuuint64_t dims[3] = {kHeadDim, (cuuint64_t)g.Hq, (cuuint64_t)n_rows};
        const cuuint64_t strides[2] = {kRowBytes, (cuuint64_t)g.Hq * kRowBytes};
        const cuuint32_t box[3] = {64, (cuuint32_t)g.Gq, (cuuint32_t)a.seqs}, step[3] = {1, 1, 1};
        if (enc(&map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    {
        // a cache without tokens: no tile is ever loaded, the map only has to be a valid one
        const bool none = g.T == 0;
        const cuuint64_t dims[2] = {kHeadDim, none ? (cuuint64_t)n_rows * (cuuint64_t)g.Hq : (cuuint64_t)g.problems * (cuuint64_t)g.T};
        const cuuint64_t strides[1] = {kRowBytes};
        const cuuint32_t box[2] = {64, kTok}, step[2] = {1, 1};
        if (enc(&map_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(none ? q : k), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    e = cudaMemsetAsync(a.status, 0, 4, st);
    if (e != cudaSuccess) return e;
    const bool cap = a.sc.softcap > 0.f, bias = a.sc.slopes || !(sm_scale > 0.f);
#define STC_PREFIX_LAUNCH(S_, C_, B_)                                                                            \
    do {                                                                                                         \
        e = cudaFuncSetAttribute(prefix_attn_kernel<S_, C_, B_>, cudaFuncAttributeMaxDynamicSharedMemorySize,    \
                                 (int)kSmem);                                                                    \
        if (e != cudaSuccess) return e;                                                                          \
        prefix_attn_kernel<S_, C_, B_><<<n_cta, kThreads, kSmem, st>>>(map_q, map_k, a);                         \
    } while (0)
#define STC_PREFIX(S_)                                                                                           \
    case S_:                                                                                                     \
        if (cap && bias) STC_PREFIX_LAUNCH(S_, true, true);                                                      \
        else if (cap) STC_PREFIX_LAUNCH(S_, true, false);                                                        \
        else if (bias) STC_PREFIX_LAUNCH(S_, false, true);                                                       \
        else STC_PREFIX_LAUNCH(S_, false, false);                                                                \
        break;
    switch (g.S) {
        STC_PREFIX(4) STC_PREFIX(8) STC_PREFIX(16)
        default: return cudaErrorInvalidValue;
    }
#undef STC_PREFIX
#undef STC_PREFIX_LAUNCH
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const long long tasks = (long long)n_rows * g.Hq;
    const unsigned grid = (unsigned)((tasks + 7) / 8);
    prefix_merge_kernel<<<grid, 256, 0, st>>>(a, n_cta);
    return cudaGetLastError();
}

}  // namespace stc
