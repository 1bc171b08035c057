// Attention over shared prefixes: the sequences of a batch that continue the same cached prefix attend it
// together, so that the prefix is read once for all of them instead of once per sequence.
//
//   For every prefix g, KV head and query row r = (sequence, query head of that KV head) of the prefix's sequences:
//     s_t = sm_scale * q_r.k_t (+ options of stc_score),  p = softmax over the prefix's tokens of s
//     out_r = sum_t p_t v~_t   (v~: routed values, dropped groups zero),  lse_r = log sum exp s
//   optionally joined with (own_out, own_lse) of the sequence's own tokens by their log-sum-exps.
//
// Rows of one KV head form tiles of 128, tokens tiles of 64; both products run on the 5th-generation tensor
// cores with their accumulators in tensor memory:
//   S[row][token] = Q . K^T     Q, K tiles by TMA (128-byte swizzle), M = 128, N = 64, K = 128
//   O[row][dim]  += P . V~      P from tensor memory, written over S by the softmax; V~ rebuilt from the packed
//                               groups in shared memory, token rows of 128 dims = N-major operand
// P enters as a bf16 high part plus a bf16 residual (two MMAs): the output is fp32, and one bf16 weight alone would
// leave it 2^-8 off; the pair leaves 2^-16.  The tensor core truncates when it adds to an accumulator (measured:
// 4e-8 of its value per product), so an accumulator is emptied into fp32 sums now and then (kFlush).
//
// What bounds it.  Up to 128 rows per KV head the two products of 128 tokens take about 1800 cycles of the tensor pipe
// and their bytes (K 32 KiB, V up to 32 KiB) 2100 to 2800 cycles of an SM's share of HBM; the loop product -> softmax ->
// product of a group takes about 2850 for its 64 of them, so a long prefix runs at 0.6 of the copy rate (131072 tokens, 16 x
// 32/8 heads: 107 us for 405 MB).  Halving the softmax's work or the second product alone gains 5 % each, halving the value
// warps' 1 %: it is the chain, not one of its links.  At 256 rows 64 tokens take 3020 cycles (start and end included), of which
// the products are 1792: 1536 at the pipe's rate, 256 because an S product of N = 64 takes 1.5 times its share.  A work unit is
// at most two row tiles (one pass over K and V for 256 rows); larger batches take more units, whose K and V come from L2
// (32768 tokens, 128 x 32/8 heads: 112 us for 69 GFLOP).  A short call pays 4.5 us to its first scores, 2 us for a segment's end
// and 4 us for the second kernel (272 tokens, 8 x 32 heads: 14.6 us).
//
// A window, positions inside the prefix and documents are masks on the scores: every tile of a prefix is loaded and multiplied,
// whatever its rows see of it (131072 tokens, 16 x 32/8 heads: 105 us; with a window of 4096 100 us; with documents 135 to 138 us,
// each thread then reads its tile's document words and hides scores one by one).
//
// Work split.  Unit = (prefix, KV head, block of up to two row tiles); the token tiles of all units form one flat
// sequence, each as long as it takes (2, 3 or 4 for a tile whose softmax has 32 scores per thread, 64, or 64 in both
// groups), that is cut into equal contiguous ranges, one per CTA (one CTA per SM).  A CTA takes the tiles that begin in its
// range and walks them unit by unit, segment by segment; a segment that is a whole unit is finished in place, another one leaves a partial (max, sum,
// accumulator) which a second small kernel joins in CTA order: no atomics, bitwise repeatable.
//
// Roles (16 warps): warp 0 = TMA producer of Q and K; warps 1, 2 = MMA issuers of the two groups; warp 3 = scheduler
// (walks the segments for all roles, a few ahead); warps 4..7 and
// 8..11 = softmax of the two groups, thread = row; warps 12..15 rebuild the value tiles with 16-byte asynchronous
// copies straight from the packed store into the swizzled tile.  Two row tiles: group w owns row tile w and both see
// every token tile.  One row tile: the groups take the token tiles in turn.  A group has two S buffers: the product for
// its next tile runs while it works on this one, and its softmax waits for nothing else unless the maximum moves.
// Few rows: a row tile is four quarters of 32 lanes (the lanes of one warp), and the softmax of a row is 64 scores of
// one thread, so half-empty tiles would cost as much as full ones.  With at most two quarters of rows the tile holds
// them twice; copy i weighs columns [32 i, 32 i + 32) and writes zeros for the others, so each thread has 32 scores.
// At the end of a segment the groups join their accumulators (each reads both, for half of the channels); copies are joined
// like the partials of different CTAs.
//
// The running maximum only moves when a tile exceeds it by more than 2^8, so the accumulator in tensor memory is
// rescaled a few times per segment and not per tile; weights are then at most 2^8, far from fp32's limits.
//
// The token tiles of a segment are taken from the last to the first: with a distance bias the largest scores come
// first and the maximum hardly moves afterwards.
//
// Every wait is bounded (about a second); one that expires raises a CTA-wide flag and STC_ERR_TIMEOUT in the
// status word, the roles leave, the producer waits (bounded) for its copies, tensor memory is freed.
#include <type_traits>

#include "umma.cuh"

namespace stc {
namespace {

constexpr int kRows = 128;                        // rows per tile = tensor-memory lanes
constexpr int kTok = 64;                          // tokens per tile
constexpr int kThreads = 512;
constexpr int kKStages = 6, kVStages = 4;
// Tiles an accumulator takes before it is emptied, eight products each.  A product truncates the accumulator by 4e-8, so 32 tiles
// leave up to 5e-6 of it and 16 half of that.  With one row tile a group sees every other tile and the weights' own error (up to
// 2^-16 each, 1.2e-6 to 2e-6 of a result) is the larger part; emptying every 16 would cost 7 % there.  With two row tiles accumulators
// see twice the tiles: 16 cost 7 % (32768 tokens, 128 sequences of 32/8 heads: 103 -> 111 us) and leave 3.2e-6 instead of 4.9e-6,
// the plain fp32 form 2.3e-6.
constexpr int kFlush = 32, kFlushTwo = 16;
__device__ __forceinline__ bool empties(int n, bool two) { return n > 0 && (two ? n % kFlushTwo : n % kFlush) == 0; }
constexpr int kSegs = 8;                          // segments the scheduler may be ahead
constexpr uint32_t kQHalf = kRows * 128;          // 64 channels of a row tile: 128 rows of 128 bytes
constexpr uint32_t kQTile = 2 * kQHalf;           // 32 KiB
constexpr uint32_t kHalf = kTok * 128;            // 64 channels of a token tile
constexpr uint32_t kTile = 2 * kHalf;             // 16 KiB
constexpr uint32_t kOffK = 2 * kQTile, kOffV = kOffK + kKStages * kTile, kOffCtl = kOffV + kVStages * kTile;
constexpr uint32_t kCtlMl = 1024;                 // [2 groups][128 lanes] maximum and sum, exchanged at a segment's end
constexpr uint32_t kCtlBytes = kCtlMl + 2 * kRows * 8;
constexpr uint32_t kSmem = kOffCtl + kCtlBytes;
static_assert(kSmem <= 232448, "shared memory of a block");
constexpr unsigned long long kWaitNs = 1000000000ull;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;                     // log2 units the maximum may be exceeded by

// barriers, in 8-byte words of the control block; [2] = per group, empties [stage][group], S / P / O [group][buffer].
// A waiter may be two products behind (its group has two buffers), which one barrier's parity could not tell from none:
// hence one O barrier per buffer, whose earlier use the waiter always knows to be through.
enum { kQFull, kQEmpty, kKFull = kQEmpty + 2, kKEmpty = kKFull + kKStages, kVFull = kKEmpty + 2 * kKStages,
       kVEmpty = kVFull + kVStages, kSFull = kVEmpty + 2 * kVStages, kPFull = kSFull + 4, kOFull = kPFull + 4,
       kXchg = kOFull + 4, kSegFull, kSegEmpty = kSegFull + kSegs, kBars = kSegEmpty + kSegs };
static_assert(kBars * 8 <= 512, "control block");
constexpr uint32_t kCtlTmem = 512, kCtlAbort = 516, kCtlSegs = 544;    // tensor-memory address, abort flag, kSegs x 32 bytes
constexpr int kSegReaders = 15;                   // warps that follow the segments: all but the scheduler

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
    int32_t* cta_status;         // [grid], one word per CTA
    int32_t* status;             // the call's status word, written by the second kernel
    long long* base;             // [G + 3]: where each prefix begins in the flat sequence; [G] = its length; [G + 1] = CTAs that
                                 // share it; [G + 2] = 1 if row_start is bad
    float4* part_o;              // [3 * grid][2 groups][32 chunks of 4 dims][128 lanes]
    float2* part_ml;             // [3 * grid][2][128]
    float4* flush;               // [grid][2 groups][32][128 rows]: sums of emptied accumulators
    int64_t cap_groups;
    int G, Hq, Hkv, Gq, T, n_rows;
    int quarter;                 // sequences per quarter of a row tile = 32 / Gq
    int seqs;                    // sequences per row tile = 4 * quarter
    int q_box;                   // quarters a load of Q brings: 2 where their rows are contiguous (Gq divides 32), else 1
    float scale_log2, cap_in, cap_log2;
    ScoreArgs sc;
};

// Copies of its rows that the row tile of a segment holds.
__device__ __forceinline__ int copies(const PrefixArgs& a, int n_seq) {
    return n_seq <= 2 * a.quarter ? 2 : 1;
}

struct Group {
    int row0, n_seq, len, tiles, blocks;
    int weight;                  // length of a tile of its first block in the flat sequence
};
__device__ __forceinline__ Group make_group(const PrefixArgs& a, int row0, int row1, int len) {
    Group r;
    r.row0 = row0;
    r.n_seq = row1 - row0;
    r.len = len;
    r.tiles = (len + kTok - 1) / kTok;
    r.blocks = (r.n_seq + 2 * a.seqs - 1) / (2 * a.seqs);
    r.weight = r.n_seq > a.seqs ? 4 : copies(a, r.n_seq) == 2 ? 2 : 3;
    return r;
}
__device__ __forceinline__ Group load_group(const PrefixArgs& a, int g) {
    return make_group(a, a.row_start[g], a.row_start[g + 1], clamp_len(a.seq_len, g, a.T));
}
__device__ __forceinline__ long long group_length(const PrefixArgs& a, const Group& g) {
    return (long long)g.tiles * g.weight * g.blocks * a.Hkv;
}

// One segment: tiles [tile0, tile1) of one unit.
struct Segment {
    int g, hk, row0, n_seq, len, tile0, tile1;
    int slot;                    // partial slot, -1 = the whole unit
};
__device__ __forceinline__ long long div_small(long long x, int d) {        // x >= 0, d > 0
    return (x >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)d) : x / d;
}
// CTA `c` of `n` takes the positions [total * c / n, total * (c + 1) / n) of the flat sequence.
__device__ __forceinline__ long long range_begin(long long total, int c, int n) {
    return total < (1 << 24) ? (long long)((uint32_t)total * (uint32_t)c / (uint32_t)n) : total * c / n;
}
__device__ __forceinline__ int cta_of(long long total, long long x, int n) {
    return total < (1 << 24) ? (int)((((uint32_t)x + 1u) * (uint32_t)n + (uint32_t)total - 1u) / (uint32_t)total) - 1
                             : (int)(((x + 1) * n + total - 1) / total - 1);
}

// Walks the segments of the CTA's range.
struct Walker {
    long long x, x_end, off;     // positions; off = x - begin of group g
    int g;
    Group grp;                   // group g
    __device__ __forceinline__ bool next(const PrefixArgs& a, Segment& s) {
        while (x < x_end) {
            while (off >= group_length(a, grp)) {
                off -= group_length(a, grp);
                grp = load_group(a, ++g);
            }
            const int length = grp.tiles * grp.weight;                     // of a unit (below 2^27)
            const long long unit = div_small(off, length);
            const int from = (int)(off - unit * length), to = (int)min((long long)length, from + (x_end - x));
            x += to - from;
            off += to - from;
            s.tile0 = (int)((uint32_t)(from + grp.weight - 1) / (uint32_t)grp.weight);
            s.tile1 = (int)((uint32_t)(to + grp.weight - 1) / (uint32_t)grp.weight);
            if (s.tile0 >= s.tile1) continue;                              // the rest of a tile that began before the range
            s.hk = (int)div_small(unit, grp.blocks);
            const int blk = (int)(unit - (long long)s.hk * grp.blocks);
            s.g = g;
            s.row0 = grp.row0 + blk * 2 * a.seqs;
            s.n_seq = min(2 * a.seqs, grp.n_seq - blk * 2 * a.seqs);
            s.len = grp.len;
            // a CTA continues at most one unit (slot 0) and leaves at most one that it begins (slot 1)
            s.slot = s.tile1 - s.tile0 == grp.tiles ? -1 : 2 * (int)blockIdx.x + (s.tile0 == 0 ? 1 : 0);
            return true;
        }
        return false;
    }
};

// Joins an attention result (m in log2 units, l, unnormalised o) with the sequence's own (own, own_lse): factors
// for o and own, and the joined lse.  An empty side gets the factor 0 and is not to be multiplied.
struct Join { float fo, fown, lse; };
__device__ __forceinline__ Join join(float m, float l, float shift, bool has_own, float own_lse) {
    const float nan = __int_as_float(0x7FFFFFFF);
    if (l != l || (has_own && own_lse != own_lse)) return Join{nan, nan, nan};      // a NaN among the seen is an answer
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

// Two raw products capped, in log2 units, where they stay below 0.35 of the cap: x scale (1 + u P(u)) with u the square of
// x scale / cap, P of three terms by weighted least squares at Chebyshev nodes (relative error 4.3e-8 of tanh).
constexpr float kCapSmall = 0.35f, kCap1 = -0.33332642912864685f, kCap2 = 0.13299374282360077f, kCap3 = -0.049123503267765045f;
__device__ __forceinline__ float2 cap_small(float2 x, float cap_in, float scale_log2) {
    const float2 z = mul2(x, both(cap_in)), u = mul2(z, z);
    float2 p = fma2(both(kCap3 * scale_log2), u, both(kCap2 * scale_log2));
    p = fma2(p, u, both(kCap1 * scale_log2));
    p = fma2(p, u, both(scale_log2));
    return mul2(x, p);
}
__device__ __forceinline__ float cap_any(float x, float cap_in, float cap_log2) {
    const float z = x * cap_in, lo = tanh_small(z), hi = tanh_large(z);
    return cap_log2 * (fabsf(z) <= kTanhSmall ? lo : hi);
}
// Cap the N scores of a row: far below the cap (the usual case; the warp votes once per tile instead of branching per
// score), and of any size.
template <int N>
__device__ __forceinline__ void cap_scores_low(uint32_t (&r)[N], float cap_in, float scale_log2) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 y = cap_small(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), cap_in, scale_log2);
        r[i] = __float_as_uint(y.x);
        r[i + 1] = __float_as_uint(y.y);
    }
}
template <int N>
__device__ __forceinline__ void cap_scores_any(uint32_t (&r)[N], float cap_in, float cap_log2) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __float_as_uint(cap_any(__uint_as_float(r[i]), cap_in, cap_log2));
}
template <int N>
__device__ __forceinline__ float magnitude(const uint32_t (&r)[N]) {
    float b[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; i += 2)
        b[(i >> 1) & 3] = fmaxf(fmaxf(b[(i >> 1) & 3], fabsf(__uint_as_float(r[i]))), fabsf(__uint_as_float(r[i + 1])));
    return fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]));
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
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctl + kCtlTmem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctl + kCtlAbort);
    float2* const ml = reinterpret_cast<float2*>(ctl + kCtlMl);
    volatile int* const segs = reinterpret_cast<volatile int*>(ctl + kCtlSegs);        // [kSegs][8]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;");

    // ---- set-up: barriers, tensor memory; the scheduler's and the producer's first reads are under way meanwhile ------------
    int first_r0 = 0, first_r1 = 0, first_len = 0;   // scheduler: prefix `lane`
    if (warp == 3 && lane < a.G) {
        first_r0 = a.row_start[lane];
        first_r1 = a.row_start[lane + 1];
        first_len = clamp_len(a.seq_len, lane, a.T);
    }
    if (warp == 0 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &map_k : &map_q) : "memory");
    if (threadIdx.x >= 128 && threadIdx.x < 128 + kBars) {       // one barrier per thread
        const int i = (int)threadIdx.x - 128;
        mbar_init(bars + 8 * i, i >= kPFull && i < kOFull ? kRows : i == kXchg ? 2 * kRows : i >= kVFull && i < kVEmpty ? 2 : i >= kSegEmpty ? kSegReaders : 1);
        fence_mbar_init();
    }
    if (threadIdx.x == 128) *abort_flag = (base & 1023u) != 0 ? (int)STC_ERR_CUDA : 0;      // swizzled tiles need 1024-byte aligned bases
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(bars + kCtlTmem), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_slot;
    Segment s;
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto wait = [&](int i, uint32_t parity) { return mbar_wait_or_abort(bar(i), parity & 1u, abort_flag, kWaitNs); };
    auto warp_wait = [&](int i, uint32_t parity) { return mbar_warp_wait_or_abort(bar(i), parity & 1u, abort_flag, kWaitNs); };
    auto give_up = [&]() { *abort_flag = (int)STC_ERR_TIMEOUT; };
    // The next segment, for a role that is one lane / a whole warp.  False: none left, or given up (`good` cleared).
    int n_seg = 0;
    auto read_segment = [&]() {
        const volatile int* e = segs + (n_seg % kSegs) * 8;
        s = Segment{e[0], e[1], e[2], e[3], e[4], e[5], e[6], e[7]};
    };
    auto next_lane = [&](bool& good) -> bool {
        good = wait(kSegFull + n_seg % kSegs, (uint32_t)(n_seg / kSegs));
        if (!good) return false;
        read_segment();
        mbar_arrive(bar(kSegEmpty + n_seg % kSegs));
        ++n_seg;
        return s.tile1 >= 0;
    };
    auto next_warp = [&](bool& good) -> bool {
        good = warp_wait(kSegFull + n_seg % kSegs, (uint32_t)(n_seg / kSegs));
        if (!good) return false;
        read_segment();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kSegEmpty + n_seg % kSegs));
        ++n_seg;
        return s.tile1 >= 0;
    };

    if (*abort_flag) {
        // nothing was started
    } else if (warp == 0) {
        // ---- producer of Q and K ---------------------------------------------------------------------
        if (lane == 0) {
            int kc = 0, seg = 0;
            uint32_t used[2] = {0u, 0u}, par[2] = {0u, 0u};    // per group, bit = stage: its last tile was read; parity to wait for
            bool ok = true;
            const uint32_t q_bytes = 2u * 128u * (uint32_t)(a.Gq * a.seqs);       // per row tile
            const int loads = 4 / a.q_box, box_seqs = a.q_box * a.quarter;         // per half of a row tile
            while (ok && next_lane(ok)) {
                const bool two = s.n_seq > a.seqs;
                auto bring_q = [&]() -> bool {
                    if (seg > 0 && !(wait(kQEmpty, (uint32_t)(seg - 1)) && wait(kQEmpty + 1, (uint32_t)(seg - 1)))) return false;
                    mbar_expect_tx(bar(kQFull), two ? 2 * q_bytes : q_bytes);
                    const int distinct = loads / copies(a, s.n_seq);
#pragma unroll 1
                    for (int tile = 0; tile < (two ? 2 : 1); ++tile)
#pragma unroll 1
                        for (int i = 0; i < loads; ++i) {
                            const uint32_t dst = base + tile * kQTile + i * (uint32_t)a.q_box * (kQHalf / 4);
                            const int first = s.row0 + tile * a.seqs + (i < distinct ? i : i - distinct) * box_seqs;
                            tma_3d(dst, &map_q, 0, s.hk * a.Gq, first, bar(kQFull));
                            tma_3d(dst + kQHalf, &map_q, 64, s.hk * a.Gq, first, bar(kQFull));
                        }
                    ++seg;
                    return true;
                };
                // the queries behind the first key tile: both are wanted at once, and the keys come from farther away
                bool q_due = true;
                const int row = (s.g * a.Hkv + s.hk) * a.T;
                int st = kc % kKStages;
#pragma unroll 1
                for (int t = s.tile1 - 1; t >= s.tile0; --t, ++kc) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        if (!((used[w] >> st) & 1u)) continue;
                        ok = ok && wait(kKEmpty + 2 * st + w, par[w] >> st);
                        par[w] ^= 1u << st;
                        used[w] &= ~(1u << st);
                    }
                    if (!ok) break;
                    mbar_expect_tx(bar(kKFull + st), kTile);
                    for (int h = 0; h < 2; ++h)
                        tma_2d(base + kOffK + st * kTile + h * kHalf, &map_k, 64 * h, row + t * kTok, bar(kKFull + st));
                    const uint32_t odd = (uint32_t)(s.tile1 - 1 - t) & 1u;
                    if (two || odd == 0) used[0] |= 1u << st;
                    if (two || odd == 1) used[1] |= 1u << st;
                    if (++st == kKStages) st = 0;
                    if (q_due) {
                        q_due = false;
                        ok = bring_q();
                        if (!ok) { ++kc; break; }
                    }
                }
            }
            if (!ok) give_up();
            if (*abort_flag) {                       // copies still in flight get one more bounded wait each
                int none = 0;
                if (seg > 0) mbar_wait_or_abort(bar(kQFull), (uint32_t)(seg - 1) & 1u, &none, kWaitNs);
                for (int i = max(0, kc - kKStages); i < kc; ++i)
                    mbar_wait_or_abort(bar(kKFull + i % kKStages), (uint32_t)(i / kKStages) & 1u, &none, kWaitNs);
            }
        }
    } else if (warp == 1 || warp == 2) {
        // ---- MMA issuer of group w: the warp stays together, an elected lane issues ---------------------------
        constexpr uint32_t id_qk = idesc_bf16(kRows, kTok, false), id_pv = idesc_bf16(kRows, kHeadDim, true);
        const int w = uniform(warp) - 1;
        const uint32_t sm = uniform(base), ts = uniform(tmem) + (uint32_t)w * 128u, to = uniform(tmem) + 256 + (uint32_t)w * 128u;
        uint32_t kc0 = 0, seg = 0;                   // tiles of the segments before; segments before
        uint32_t n_s = 0, n_o = 0;                   // products issued by this group
        bool ok = true;
        while (ok && next_warp(ok)) {
            const int tiles = uniform(s.tile1 - s.tile0);
            const bool two = uniform((int)(s.n_seq > a.seqs)) != 0;       // two row tiles: every token tile goes to both groups
            const int mine = two ? tiles : (tiles + 1 - w) >> 1;
            const uint32_t first = kc0 + (two ? 0 : w), stride = two ? 1 : 2;
            ok = warp_wait(kQFull, seg);
            if (ok && mine == 0 && lane == 0) mbar_arrive(bar(kQEmpty + w));
            const uint32_t q_at = sm + (two ? w * kQTile : 0u);
            // iteration n: O += P V of tile n - 2, whose S buffer then takes S = Q K^T of tile n
#pragma unroll 1
            for (int n = 0; ok && mine > 0 && n < mine + 2; ++n) {
                if (n >= 2) {
                    const uint32_t j = first + (uint32_t)(n - 2) * stride, st = j % kVStages, buf = n_o & 1u;
                    ok = warp_wait(kPFull + 2 * w + buf, n_o >> 1) && warp_wait(kVFull + st, j / kVStages);
                    if (!ok) break;
                    tc_after();
                    const uint64_t dv = smem_desc_128(sm + kOffV + st * kTile, kHalf);
                    const uint32_t p = ts + buf * 64u;
                    const uint32_t more = n > 2 && !empties(n - 2, two);  // else O starts anew
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {        // 16 tokens: 16 rows of 128 bytes; P: 8 columns high, 8 residual
                            tc_mma_ts(to, p + 16 * k, dv + (uint64_t)(k * (2048 >> 4)), id_pv, k ? 1u : more);
                            tc_mma_ts(to, p + 16 * k + 8, dv + (uint64_t)(k * (2048 >> 4)), id_pv, 1);
                        }
                        tc_commit_to(bar(kOFull + 2 * w + buf));
                        tc_commit_to(bar(kVEmpty + 2 * st + w));
                    }
                    __syncwarp();
                    ++n_o;
                }
                if (n < mine) {
                    const uint32_t j = first + (uint32_t)n * stride, st = j % kKStages, buf = n_s & 1u;
                    ok = warp_wait(kKFull + st, j / kKStages);
                    // the buffer holds the P of the group's last but one tile until that product is through
                    if (ok && n_s >= 2) ok = warp_wait(kOFull + 2 * w + buf, (n_s - 2) >> 1);
                    if (!ok) break;
                    tc_after();
                    const uint64_t dq = smem_desc_128(q_at, 16), dk = smem_desc_128(sm + kOffK + st * kTile, 16);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)          // 16 dims = 32 bytes = 2 units; 64 dims = one half tile
                            tc_mma_ss(ts + buf * 64u, dq + (uint64_t)((k >> 2) * (kQHalf >> 4) + (k & 3) * 2),
                                      dk + (uint64_t)((k >> 2) * (kHalf >> 4) + (k & 3) * 2), id_qk, k != 0);
                        tc_commit_to(bar(kSFull + 2 * w + buf));
                        tc_commit_to(bar(kKEmpty + 2 * st + w));
                        if (n == mine - 1) tc_commit_to(bar(kQEmpty + w));
                    }
                    __syncwarp();
                    ++n_s;
                }
            }
            kc0 += (uint32_t)tiles;
            ++seg;
        }
        if (!ok) give_up();
    } else if (warp == 3) {
        // ---- scheduler: the flat sequence by prefix sums over the prefixes, this CTA's range, its segments ----------------------
        // (32 prefixes at a time; straight through for up to 32, since this stands before everything else)
        Group grp = {};                              // of prefix `lane`
        bool bad = false;
        if (lane < a.G) {
            bad = first_r0 < 0 || first_r1 < first_r0 || first_r1 > a.n_rows;
            if (!bad) grp = make_group(a, first_r0, first_r1, first_len);
        }
        auto sums = [&](long long n) {               // inclusive over the lanes
            if (a.G == 1) return __shfl_sync(0xFFFFFFFFu, n, 0);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long o = __shfl_up_sync(0xFFFFFFFFu, n, d);
                if (lane >= d) n += o;
            }
            return n;
        };
        long long mine = group_length(a, grp), end = sums(mine), total = __shfl_sync(0xFFFFFFFFu, end, 31);
        int weight = __reduce_max_sync(0xFFFFFFFFu, mine > 0 ? grp.weight : 0);
        auto some = [&](const Group& g) { return g.tiles > 0 ? (int)min((long long)g.blocks * a.Hkv, 1LL << 20) : 0; };
        const int units = __reduce_add_sync(0xFFFFFFFFu, some(grp));
        const int longest = __reduce_max_sync(0xFFFFFFFFu, grp.tiles * grp.weight);
        const bool alike = a.G <= 32 && __all_sync(0xFFFFFFFFu, grp.tiles == 0 || grp.tiles * grp.weight == longest);
        if (blockIdx.x == 0 && lane < a.G) a.base[lane] = end - mine;
        for (int g0 = 32; g0 < a.G; g0 += 32) {
            Group more = {};
            if (g0 + lane < a.G) {
                const int r0 = a.row_start[g0 + lane], r1 = a.row_start[g0 + lane + 1];
                if (r0 < 0 || r1 < r0 || r1 > a.n_rows) bad = true;
                else more = load_group(a, g0 + lane);
            }
            const long long n = group_length(a, more), e = total + sums(n);
            if (blockIdx.x == 0 && g0 + lane < a.G) a.base[g0 + lane] = e - n;
            total = __shfl_sync(0xFFFFFFFFu, e, 31);
            weight = max(weight, __reduce_max_sync(0xFFFFFFFFu, n > 0 ? more.weight : 0));
        }
        bad = __any_sync(0xFFFFFFFFu, bad);
        if (bad) total = 0;
        // with fewer tiles than CTAs the rest stay idle: every range holds the beginning of a tile
        const int cta = (int)blockIdx.x;
        int n_cta = total > 0 ? (int)min(div_small(total, weight), (long long)gridDim.x) : 0;
        if (alike && units > 0 && units < n_cta) {
            // Units of one length: the same number of CTAs for each, so that units end where ranges end, if the CTAs that this
            // leaves idle cost the others less than three tiles, about what a second segment costs a CTA.
            const int even = n_cta / units * units;
            if (total / even - total / n_cta < 3 * weight) n_cta = even;
        }
        Walker walk;
        walk.x = walk.x_end = walk.off = 0;
        walk.g = 0;
        if (cta < n_cta) {
            walk.x = range_begin(total, cta, n_cta);
            walk.x_end = range_begin(total, cta + 1, n_cta);
            // the prefix that holds x
            long long before = 0;
            int g0 = 0;
            for (;;) {
                const uint32_t who = __ballot_sync(0xFFFFFFFFu, end - mine <= walk.x && walk.x < end);
                if (who) {
                    const int from = __ffs(who) - 1;
                    walk.off = walk.x - __shfl_sync(0xFFFFFFFFu, end - mine, from);
                    walk.g = g0 + from;
                    walk.grp = Group{__shfl_sync(0xFFFFFFFFu, grp.row0, from), __shfl_sync(0xFFFFFFFFu, grp.n_seq, from),
                                     __shfl_sync(0xFFFFFFFFu, grp.len, from), __shfl_sync(0xFFFFFFFFu, grp.tiles, from),
                                     __shfl_sync(0xFFFFFFFFu, grp.blocks, from), __shfl_sync(0xFFFFFFFFu, grp.weight, from)};
                    break;
                }
                before = __shfl_sync(0xFFFFFFFFu, end, 31);
                g0 += 32;                            // (x < total: there is a next 32)
                grp = Group{};
                if (g0 + lane < a.G) grp = load_group(a, g0 + lane);
                mine = group_length(a, grp);
                end = before + sums(mine);
            }
        }
        if (lane == 0) {
            bool ok = true, more = true;
            for (int i = 0; ok && more; ++i) {
                more = walk.next(a, s);
                if (i >= kSegs) ok = wait(kSegEmpty + i % kSegs, (uint32_t)(i / kSegs - 1));
                if (!ok) break;
                volatile int* e = segs + (i % kSegs) * 8;
                e[0] = s.g; e[1] = s.hk; e[2] = s.row0; e[3] = s.n_seq; e[4] = s.len; e[5] = s.tile0;
                e[6] = more ? s.tile1 : -1;
                e[7] = s.slot;
                mbar_arrive(bar(kSegFull + i % kSegs));
            }
            if (!ok) give_up();
            if (cta == 0) { a.base[a.G] = total; a.base[a.G + 1] = n_cta; a.base[a.G + 2] = bad; }
        }
    } else if (warp >= 4 && warp < 12) {
        // ---- softmax: thread = row of the tile's lanes --------------------------------------------------------
        const int w = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t to = lane_base + 256 + w * 128;
        float4* const my_flush = a.flush + ((size_t)blockIdx.x * 2 + w) * 32 * kRows + row;
        uint32_t n_s = 0, n_x = 0;                   // tiles of this group; uses of the exchange barrier
        bool ok = true;

        // One segment with 64 / COLS copies of the rows; this thread weighs COLS of a tile's 64 scores.
        auto segment = [&](auto cols) {
            constexpr int COLS = decltype(cols)::value, REP = kTok / COLS;
            const int tiles = s.tile1 - s.tile0;
            const bool two = s.n_seq > a.seqs;
            const int mine = two ? tiles : (tiles + 1 - w) >> 1, stride = two ? 1 : 2, last = s.tile1 - 1 - (two ? 0 : w);
            // this thread's row: sequence, head, copy
            const int copy = quarter / (4 / REP), c0 = copy * COLS;
            const int in_quarter = lane / a.Gq, seq_i = (two ? w * a.seqs : 0) + (quarter % (4 / REP)) * a.quarter + in_quarter;
            const bool live = in_quarter < a.quarter && seq_i < s.n_seq;
            const bool warp_live = __any_sync(0xFFFFFFFFu, live);
            const int seq = s.row0 + (live ? seq_i : 0), head = s.hk * a.Gq + lane % a.Gq;
            int lo = 0, hi = s.len, my_doc = 0;
            float slope2 = 0.f;
            if (a.sc.q_pos) visible_range(s.len, a.sc.q_pos[seq], a.sc.window, lo, hi);
            if (BIAS && a.sc.slopes) slope2 = a.sc.slopes[head] * kLog2e;
            const int32_t* doc = a.sc.tok_doc ? a.sc.tok_doc + (size_t)s.g * a.T : nullptr;
            if (doc) my_doc = a.sc.q_doc[seq];
            // `v` for the tokens t .. t + COLS - 1 that the row does not see
            auto hide = [&](uint32_t (&r)[COLS], int t, float v) {
#pragma unroll
                for (int i = 0; i < COLS; ++i)
                    if (t + i < lo || t + i >= hi) r[i] = __float_as_uint(v);
                if (doc) {
#pragma unroll
                    for (int i = 0; i < COLS; ++i) {
                        const int d = __ldg(doc + min(t + i, a.T - 1));
                        if (d >= 0 && d != my_doc) r[i] = __float_as_uint(v);
                    }
                }
            };
            const int first_flush = two ? kFlushTwo : kFlush;
            float m = -INFINITY, l = 0.f, m_flush = -INFINITY;
#pragma unroll 1
            for (int n = 0; n < mine; ++n) {
                const uint32_t buf = n_s & 1u, ts = lane_base + w * 128 + buf * 64;
                if (!warp_live) {                    // a quarter without rows: its P may be anything
                    ok = warp_wait(kSFull + 2 * w + buf, n_s >> 1);
                    if (!ok) return;
                    mbar_arrive(bar(kPFull + 2 * w + buf));
                    ++n_s;
                    continue;
                }
                const bool empty_now = empties(n, two);
                const float m_acc = m;               // maximum the accumulator was built with
                ok = warp_wait(kSFull + 2 * w + buf, n_s >> 1);
                if (!ok) return;
                tc_after();
                const int t0 = (last - n * stride) * kTok + c0;
                uint32_t r[COLS];
                tmem_ld16<0>(ts + c0, r);
                if constexpr (COLS > 16) tmem_ld16<16>(ts + c0 + 16, r);
                if constexpr (COLS > 32) {
                    tmem_ld16<32>(ts + c0 + 32, r);
                    tmem_ld16<48>(ts + c0 + 48, r);
                }
                tmem_wait_ld();
                // does every row of the warp see all the tokens?
                auto all_seen = [&]() { return !doc && __all_sync(0xFFFFFFFFu, lo <= t0 && hi >= t0 + COLS); };
                // scores in log2 units where they are not the raw products times a positive scale
                if constexpr (CAP) {
                    // Tokens that are not seen, and lanes without a row, hold whatever was in memory and have no say in how
                    // the others are capped.  If everything is small, so is what is seen; else it is asked by itself (looking
                    // at seen tokens only from the start costs 4 % of 131072 tokens, 18 % with a window).
                    auto small = [&]() { return __all_sync(0xFFFFFFFFu, (live ? magnitude(r) : 0.f) * fabsf(a.cap_in) <= kCapSmall); };
                    if (__builtin_expect(small(), 1)) {
                        cap_scores_low(r, a.cap_in, a.scale_log2);
                    } else {
                        bool low = false;
                        if (!all_seen()) {
                            hide(r, t0, 0.f);
                            low = small();
                        }
                        if (low) cap_scores_low(r, a.cap_in, a.scale_log2);
                        else cap_scores_any(r, a.cap_in, a.cap_log2);
                    }
                }
                if constexpr (BIAS) {
                    const float far = (float)(t0 - (hi - 1));
#pragma unroll
                    for (int i = 0; i < COLS; i += 2) {
                        float2 x = make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                        if constexpr (!CAP) x = mul2(x, both(a.scale_log2));
                        x = fma2(both(slope2), add2(both(far), make_float2((float)i, (float)(i + 1))), x);
                        r[i] = __float_as_uint(x.x);
                        r[i + 1] = __float_as_uint(x.y);
                    }
                }
                if (!all_seen()) hide(r, t0, -INFINITY);
                float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < COLS; i += 2)
                    t4[(i >> 1) & 3] = fmaxf(fmaxf(t4[(i >> 1) & 3], __uint_as_float(r[i])), __uint_as_float(r[i + 1]));
                float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
                if constexpr (!CAP && !BIAS) top *= a.scale_log2;     // (-inf stays -inf: the scale is positive)
                // move the maximum only if it is exceeded by much; the accumulator follows
                const bool move = top > m + kSlack || (m == -INFINITY && top > -INFINITY);
                if (__any_sync(0xFFFFFFFFu, move)) {
                    const float to_m = move ? top : m;
                    const float f = (m == -INFINITY) ? 0.f : ex2(m - to_m);
                    l *= f;
                    if (n > 0 && !empty_now) {
                        ok = warp_wait(kOFull + 2 * w + ((n_s - 1) & 1u), (n_s - 1) >> 1);
                        if (!ok) return;
                        tc_after();
#pragma unroll 1
                        for (int c = 0; c < kHeadDim; c += 16) {
                            uint32_t q[16];
                            tmem_ld16(to + c, q);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                q[i] = move ? __float_as_uint(__uint_as_float(q[i]) * f) : q[i];
                            tmem_st16(to + c, q);
                        }
                    }
                    m = to_m;
                }
                // weights, their sum, and P over S: per 16 tokens 8 columns of bf16 pairs high, 8 residual
                const float ref = m == -INFINITY ? 0.f : m;
                float2 la = make_float2(0.f, 0.f), lb = la;
#pragma unroll
                for (int c = 0; c < COLS; c += 16) {
                    uint32_t o[16];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float2 p = make_float2(__uint_as_float(r[c + 2 * i]), __uint_as_float(r[c + 2 * i + 1]));
                        if constexpr (CAP || BIAS) p = add2(p, both(-ref));
                        else p = fma2(p, both(a.scale_log2), both(-ref));
                        p.x = ex2(p.x);
                        p.y = ex2(p.y);
                        if (i & 1) lb = add2(lb, p); else la = add2(la, p);
                        const __nv_bfloat162 h2 = __floats2bfloat162_rn(p.x, p.y);
                        o[i] = *reinterpret_cast<const uint32_t*>(&h2);
                        const float2 d = fma2(make_float2(bf16lo(o[i]), bf16hi(o[i])), both(-1.f), p);
                        const __nv_bfloat162 r2 = __floats2bfloat162_rn(d.x, d.y);
                        o[8 + i] = *reinterpret_cast<const uint32_t*>(&r2);
                    }
                    tmem_st16(ts + c0 + c, o);
                }
                if constexpr (REP > 1) {             // the columns of the other copies
                    uint32_t zero[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll
                    for (int c = 0; c < kTok - COLS; c += 16) tmem_st16(ts + ((c0 + COLS + c) & (kTok - 1)), zero);
                }
                l += (la.x + lb.x) + (la.y + lb.y);
                // The accumulator is emptied into fp32 sums and the issuer starts it anew.  Here the product it
                // waits for is long through, and the product of the next scores runs meanwhile.
                if (empty_now) {
                    ok = warp_wait(kOFull + 2 * w + ((n_s - 1) & 1u), (n_s - 1) >> 1);
                    if (!ok) return;
                    tc_after();
                    const float keep = m_flush == -INFINITY ? 0.f : ex2(m_flush - m_acc);
                    const bool grow = n > first_flush && __all_sync(0xFFFFFFFFu, keep == 1.f);   // nothing to read back
#pragma unroll 1
                    for (int c = 0; c < kHeadDim; c += 32) {
                        float4 old[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            old[i] = n > first_flush && !grow ? __ldcg(my_flush + (size_t)(c / 4 + i) * kRows) : make_float4(0.f, 0.f, 0.f, 0.f);
                        uint32_t q[32];
                        tmem_ld16<0>(to + c, q);
                        tmem_ld16<16>(to + c + 16, q);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float4* dst = my_flush + (size_t)(c / 4 + i) * kRows;
                            const float4 v = make_float4(
                                fmaf(old[i].x, keep, __uint_as_float(q[4 * i])), fmaf(old[i].y, keep, __uint_as_float(q[4 * i + 1])),
                                fmaf(old[i].z, keep, __uint_as_float(q[4 * i + 2])), fmaf(old[i].w, keep, __uint_as_float(q[4 * i + 3])));
                            if (grow) red_add4(dst, v.x, v.y, v.z, v.w);
                            else __stcg(dst, v);
                        }
                    }
                    m_flush = m_acc;
                }
                tmem_wait_st();
                tc_before();
                mbar_arrive(bar(kPFull + 2 * w + buf));
                ++n_s;
            }
            // ---- end of the segment -----------------------------------------------------------------------------
            const bool whole = s.slot < 0;
            const size_t out_row = (size_t)seq * a.Hq + head;
            const float own_l = whole && a.own_lse && live ? a.own_lse[out_row] : -INFINITY;
            if (mine > 0 && warp_live) {
                ok = warp_wait(kOFull + 2 * w + ((n_s - 1) & 1u), (n_s - 1) >> 1);
                if (!ok) return;
                tc_after();
                if (mine > first_flush) {                 // take back what the accumulator was emptied of
                    const float keep = m_flush == -INFINITY ? 0.f : ex2(m_flush - m);
#pragma unroll 1
                    for (int c = 0; c < kHeadDim; c += 64) {
                        float4 old[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) old[i] = __ldcg(my_flush + (size_t)(c / 4 + i) * kRows);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t q[16];
                            tmem_ld16(to + c + 16 * k, q);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float4 o = old[4 * k + i];
                                q[4 * i] = __float_as_uint(fmaf(o.x, keep, __uint_as_float(q[4 * i])));
                                q[4 * i + 1] = __float_as_uint(fmaf(o.y, keep, __uint_as_float(q[4 * i + 1])));
                                q[4 * i + 2] = __float_as_uint(fmaf(o.z, keep, __uint_as_float(q[4 * i + 2])));
                                q[4 * i + 3] = __float_as_uint(fmaf(o.w, keep, __uint_as_float(q[4 * i + 3])));
                            }
                            tmem_st16(to + c + 16 * k, q);
                        }
                    }
                    tmem_wait_st();
                }
            }
            // one row tile: both groups hold part of its rows; each joins them for half of the channels
            float f0 = 1.f, f1 = 0.f;
            uint32_t acc0 = to, acc1 = to;
            int c_lo = 0, c_hi = kHeadDim;
            if (!two) {
                ml[w * kRows + row] = make_float2(m, l);
                tc_before();
                mbar_arrive(bar(kXchg));
                ok = warp_wait(kXchg, n_x++);
                if (!ok) return;
                tc_after();
                const float2 a0 = ml[row], a1 = ml[kRows + row];
                m = fmaxf(a0.x, a1.x);
                f0 = a0.x == -INFINITY ? 0.f : ex2(a0.x - m);
                f1 = a1.x == -INFINITY ? 0.f : ex2(a1.x - m);
                l = a0.y * f0 + a1.y * f1;
                acc0 = lane_base + 256;
                acc1 = lane_base + 384;
                c_lo = 64 * w;
                c_hi = c_lo + 64;
            }
            const bool part = !whole || REP > 1;     // one of several parts of the row: as it stands; else the row's output
            const size_t slot = ((size_t)(whole ? 2 * (int)gridDim.x + (int)blockIdx.x : s.slot) * 2 + (two ? w : 0));
            const Join j = part ? Join{1.f, 0.f, 0.f}
                                : join(m, l, BIAS ? bias_shift(a, s.len, seq, head) : 0.f, a.own_lse != nullptr, own_l);
            if (c_lo == 0) {
                if (part) __stcg(a.part_ml + slot * kRows + row, make_float2(m, l));
                else if (live && a.lse) a.lse[out_row] = j.lse;
            }
            if (warp_live) {
                const bool add_own = !part && live && a.own_out && j.fown != 0.f, both_acc = f1 != 0.f;
                const float4* own = reinterpret_cast<const float4*>(a.own_out) + out_row * 32;
                float4* dst = part ? a.part_o + slot * 32 * kRows + row : reinterpret_cast<float4*>(a.out) + out_row * 32;
                const int step = part ? kRows : 1;
#pragma unroll 1
                for (int c = c_lo; c < c_hi; c += 16) {
                    float4 mix[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) mix[i] = add_own ? own[c / 4 + i] : make_float4(0.f, 0.f, 0.f, 0.f);
                    uint32_t q[16], q1[16];
                    tmem_ld16(acc0 + c, q);
                    tmem_ld16(acc1 + c, q1);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {        // (a factor 0 stands for "nothing seen", whatever was summed)
                            const float x = f0 != 0.f ? __uint_as_float(q[4 * i + e]) * f0 : 0.f;
                            v[e] = both_acc ? fmaf(__uint_as_float(q1[4 * i + e]), f1, x) : x;
                            v[e] = j.fo != 0.f ? v[e] * j.fo : 0.f;
                        }
                        if (live || part)
                            dst[(size_t)(c / 4 + i) * step] =
                                make_float4(fmaf(mix[i].x, j.fown, v[0]), fmaf(mix[i].y, j.fown, v[1]),
                                            fmaf(mix[i].z, j.fown, v[2]), fmaf(mix[i].w, j.fown, v[3]));
                    }
                }
                tc_before();
            }
            if (two) return;
            if constexpr (REP > 1) {
                // a whole unit whose tile held its rows twice: the four threads of a row join the copies, 32 channels each
                if (whole) {
                    __threadfence();
                    mbar_arrive(bar(kXchg));
                    ok = warp_wait(kXchg, n_x++);
                    if (!ok) return;
                    const int lane0 = (quarter % (4 / REP)) * 32 + lane, d0 = (w * REP + copy) * (32 / (2 * REP));
                    if (live) {
                        const float2 p0 = __ldcg(a.part_ml + slot * kRows + lane0), p1 = __ldcg(a.part_ml + slot * kRows + lane0 + kRows / 2);
                        const float top = fmaxf(p0.x, p1.x);
                        const float e0 = p0.x == -INFINITY ? 0.f : ex2(p0.x - top), e1 = p1.x == -INFINITY ? 0.f : ex2(p1.x - top);
                        const Join jj = join(top, p0.y * e0 + p1.y * e1, BIAS ? bias_shift(a, s.len, seq, head) : 0.f,
                                             a.own_lse != nullptr, own_l);
                        const float g0 = e0 * jj.fo, g1 = e1 * jj.fo;
                        const float4* src = a.part_o + (slot * 32 + d0) * kRows + lane0;
                        const float4* own = reinterpret_cast<const float4*>(a.own_out) + out_row * 32 + d0;
                        float4* dst = reinterpret_cast<float4*>(a.out) + out_row * 32 + d0;
                        const bool add_own = a.own_out && jj.fown != 0.f;
#pragma unroll 4
                        for (int i = 0; i < 32 / (2 * REP); ++i) {
                            const float4 x = g0 != 0.f ? __ldcg(src + i * kRows) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const float4 y = g1 != 0.f ? __ldcg(src + i * kRows + kRows / 2) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const float4 z = add_own ? own[i] : make_float4(0.f, 0.f, 0.f, 0.f);
                            dst[i] = make_float4(fmaf(x.x, g0, fmaf(y.x, g1, z.x * jj.fown)), fmaf(x.y, g0, fmaf(y.y, g1, z.y * jj.fown)),
                                                 fmaf(x.z, g0, fmaf(y.z, g1, z.z * jj.fown)), fmaf(x.w, g0, fmaf(y.w, g1, z.w * jj.fown)));
                        }
                        if (a.lse && d0 == 0) a.lse[out_row] = jj.lse;
                    }
                }
            }
            mbar_arrive(bar(kXchg));                 // the accumulators, the exchange and the scratch slot are free again
            ok = warp_wait(kXchg, n_x++);
            tc_after();
        };
        while (ok && next_warp(ok)) {
            const int n_copies = copies(a, s.n_seq);
            if (n_copies == 1) segment(std::integral_constant<int, 64>{});
            else segment(std::integral_constant<int, 32>{});
        }
        if (!ok) give_up();
    } else if (warp >= 12) {
        // ---- value tiles: packed groups -> swizzled rows ---------------------------------------------------
        // Warps 12, 13 build the even tiles and 14, 15 the odd ones (counted over the CTA), 32 tokens each.  LPT
        // neighbouring lanes copy 16-byte chunks of one token (a whole group of 32 or 64 bytes; two groups of 16), so a
        // token's mask stays with its lanes and the place of a kept group is a running count.  A kept group is one
        // asynchronous 16-byte copy per chunk, a dropped one a zero-filled copy that reads nothing.  The copies of a
        // warp's next tile are under way before the last one's are waited for, unless its stage is still being read.
        constexpr int LPT = OPG < 2 ? 2 : OPG, GPL = LPT / OPG;           // lanes per token, groups they span
        const int pair = (warp - 12) >> 1, tok0 = (warp & 1) * 32, sub = lane % LPT;
        uint32_t used[2] = {0u, 0u}, par[2] = {0u, 0u};    // as the producer's, for the value stages
        int vc = 0;                                  // tiles of the segments before
        int pending = -1;                            // stage whose copies are not waited for yet
        bool ok = true;
        auto publish = [&]() {                       // this warp's copies into `pending` have landed
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kVFull + pending));
            pending = -1;
        };
        while (ok && next_warp(ok)) {
            const bool two = s.n_seq > a.seqs;
            const size_t problem = (size_t)s.g * a.Hkv + s.hk;
            const uint16_t* mask_row = a.v_mask + problem * a.T;
            const uint32_t* offs = a.v_offs + problem * (a.T + 1);
            const uint4* packed = a.v_packed + problem * a.cap_groups * OPG;
            const int64_t limit = a.cap_groups;
            const int tiles = s.tile1 - s.tile0, last_tok = (s.tile1 - 1) * kTok + tok0;
            auto fetch = [&](int h, uint32_t& m, uint32_t& first) {        // this lane's token mask, the warp's first group
                const int t = last_tok - h * kTok;
                m = h < tiles && t + lane < s.len ? mask_row[t + lane] : 0u;
                first = h < tiles && t < s.len ? offs[t] : 0u;
            };
            const int h0 = (vc + pair) & 1;          // the pair's first tile of the segment
            uint32_t m_next, first_next;
            fetch(h0, m_next, first_next);
#pragma unroll 1
            for (int h = h0; h < tiles; h += 2) {
                const uint32_t m = m_next & ((1u << S) - 1u), first = first_next;
                fetch(h + 2, m_next, first_next);
                // per token: groups of the warp's tokens before it << 16 | its mask
                const uint32_t cnt = __popc(m), tok_word = (warp_incl_scan(cnt, lane) - cnt) << 16 | m;
                const int st = (vc + h) % kVStages;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (!((used[w] >> st) & 1u)) continue;
                    const uint32_t p = (par[w] >> st) & 1u;
                    par[w] ^= 1u << st;
                    used[w] &= ~(1u << st);
                    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar(kVEmpty + 2 * st + w), p))) continue;
                    if (pending >= 0) { cp_async_wait<0>(); publish(); }
                    ok = ok && warp_wait(kVEmpty + 2 * st + w, p);
                }
                if (!ok) break;
                if (two || !(h & 1)) used[0] |= 1u << st;
                if (two || (h & 1)) used[1] |= 1u << st;
                const int64_t room = limit - (int64_t)first;
                const uint32_t most = room <= 0 ? 0u : room > 1024 ? 1024u : (uint32_t)room;   // groups left in the store
                const uint4* src = packed + (int64_t)first * OPG + sub % OPG;
#pragma unroll 1
                for (int pass = 0; pass < LPT; ++pass) {
                    const int tok = pass * (32 / LPT) + lane / LPT;      // of the warp's 32
                    const uint32_t tw = __shfl_sync(0xFFFFFFFFu, tok_word, tok);
                    uint32_t at = tw >> 16;          // place of the next kept group of the token
                    const uint32_t row = base + kOffV + st * kTile + (uint32_t)(tok0 + tok) * 128u, swz = (uint32_t)(tok & 7);
#pragma unroll
                    for (int k = 0; k < 16 / LPT; ++k) {
                        const uint32_t oct = (uint32_t)(k * LPT + sub);  // chunk of the row: half oct >> 3, swizzled by the token
                        uint32_t mine_at = at;
                        bool kept;
                        if constexpr (GPL == 1) {
                            kept = (tw >> k) & 1u;
                            at += kept;
                        } else {
                            kept = (tw >> (2 * k + sub)) & 1u;
                            if (sub) mine_at += (tw >> (2 * k)) & 1u;
                            at += ((tw >> (2 * k)) & 1u) + ((tw >> (2 * k + 1)) & 1u);
                        }
                        kept = kept && mine_at < most;
                        cp_async16_zfill(row + (oct >> 3) * kHalf + (((oct & 7u) ^ swz) << 4), kept ? src + mine_at * OPG : packed,
                                         kept ? 16 : 0);
                    }
                }
                cp_async_commit();
                if (pending >= 0) { cp_async_wait<1>(); publish(); }
                pending = st;
            }
            vc += tiles;
        }
        cp_async_wait<0>();
        if (ok && pending >= 0) publish();
        if (!ok) give_up();
    }
    tc_before();
    __syncthreads();
    if (threadIdx.x == 0) a.cta_status[blockIdx.x] = *abort_flag;
    if (warp == 1) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Joins the partials of units that more than one CTA worked on, answers the rows whose prefix is empty, and gathers the
// CTAs' status.  A thread owns four channels of one row (row = sequence * Gq + head within the KV head); a warp eight
// consecutive rows by four such chunks (8 rows x 16 bytes are mostly one 128-byte line of a partial).  SPLIT = 1: the
// eight warps take the row's 32 chunks and each thread all partials; SPLIT = 8: the warps share the partials of four
// chunks, for calls with so few KV heads that a row has dozens of partials.  Eight loads in flight, a fixed order.
template <int SPLIT>
__global__ void __launch_bounds__(256)
prefix_merge_kernel(const PrefixArgs a, int grid, int chunks) {
    __shared__ float4 sh_o[SPLIT][32];
    __shared__ float2 sh_ml[SPLIT][32];
    // Launched while the first kernel still runs: what the call was given is read before the wait (what came before the
    // first kernel is complete), the first kernel's results after it.
    const int lane = threadIdx.x & 31;
    // lane = prefix (more than 32: searched below)
    const bool few = a.G <= 32;
    int my_r0 = 0x7FFFFFFF, my_r1 = 0, my_len = 0;
    if (few && lane < a.G) {
        my_r0 = a.row_start[lane];
        my_r1 = a.row_start[lane + 1];
        my_len = clamp_len(a.seq_len, lane, a.T);
    }
    const int row_begin = a.row_start[0], row_end = a.row_start[a.G];
    const int hk = blockIdx.x / chunks, warp = threadIdx.x >> 5, part = SPLIT == 1 ? 0 : warp;
    const uint32_t flat = (uint32_t)(blockIdx.x - hk * chunks) * 8u + (uint32_t)(lane >> 2);     // below 2^31 + 8
    const int d4 = (SPLIT == 1 ? warp : (int)blockIdx.y) * 4 + (lane & 3);
    const int seq = (int)(flat / (uint32_t)a.Gq), in_head = (int)(flat - (uint32_t)seq * (uint32_t)a.Gq), head = hk * a.Gq + in_head;
    bool mine = seq < a.n_rows && seq >= row_begin && seq < row_end;
    float m = -INFINITY, l = 0.f, shift = 0.f, own_l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f), own = o;
    const size_t out_row = (size_t)seq * a.Hq + head;
    if (mine && a.own_lse) {
        own_l = a.own_lse[out_row];
        own = reinterpret_cast<const float4*>(a.own_out + out_row * kHeadDim)[d4];
    }
    // last prefix that starts at or before the row (row_start that does not fit gives some prefix, and nothing is written)
    int g = 0;
    Group grp = {};
    if (few) {
        for (int i = 1; i < a.G; ++i)
            if (__shfl_sync(0xFFFFFFFFu, my_r0, i) <= seq) g = i;
        grp = make_group(a, __shfl_sync(0xFFFFFFFFu, my_r0, g), __shfl_sync(0xFFFFFFFFu, my_r1, g), __shfl_sync(0xFFFFFFFFu, my_len, g));
    } else if (mine) {
        int g_hi = a.G;
        while (g_hi - g > 1) {
            const int mid = (g + g_hi) >> 1;
            if (a.row_start[mid] <= seq) g = mid; else g_hi = mid;
        }
        grp = load_group(a, g);
    }
    if (mine) shift = bias_shift(a, grp.len, seq, head);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long base_g = a.base[g], total = a.base[a.G], n_cta = a.base[a.G + 1];
    const bool bad = a.base[a.G + 2] != 0;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 32) {
        int st = 0;
        for (int c = threadIdx.x; c < grid; c += 32) st = max(st, a.cta_status[c]);
        st = __reduce_max_sync(0xFFFFFFFFu, st);
        if (threadIdx.x == 0) *a.status = bad ? (int)STC_ERR_INVALID_ARG : st;
    }
    if (bad) mine = false;
    if (mine) {
        const int in_group = seq - grp.row0, blk = in_group / (2 * a.seqs), in_blk = in_group - blk * 2 * a.seqs;
        const int n_seq = min(2 * a.seqs, grp.n_seq - blk * 2 * a.seqs);
        const bool two = n_seq > a.seqs;
        // where the row's parts stand in a slot: row tile, lane of the first copy, log2 of the copies
        const int tile = two ? in_blk / a.seqs : 0, in_tile = in_blk - tile * a.seqs, qr = in_tile / a.quarter;
        const int row = qr * 32 + (in_tile - qr * a.quarter) * a.Gq + in_head;
        const int lg_copies = copies(a, n_seq) >> 1;         // (two row tiles: one copy)
        int c0 = 0, n_parts = 0;
        if (grp.tiles > 0) {                         // CTAs that the unit's first and last tile begin in
            const long long x0 = base_g + ((long long)hk * grp.blocks + blk) * grp.tiles * grp.weight;
            c0 = cta_of(total, x0, (int)n_cta);
            const int c1 = cta_of(total, x0 + (long long)(grp.tiles - 1) * grp.weight, (int)n_cta);
            mine = c0 != c1;                         // a whole unit was finished where it was computed
            if (mine) n_parts = (c1 - c0 + 1) << lg_copies;
        }
#pragma unroll 1
        for (int e0 = part; e0 < n_parts; e0 += 8 * SPLIT) {
            float2 p[8];
            float4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = min(e0 + SPLIT * i, n_parts - 1), c = e >> lg_copies, at = row + (e - (c << lg_copies)) * (kRows / 2);
                const size_t slot = (2 * (size_t)(c0 + c) + (c == 0 ? 1 : 0)) * 2 + tile;
                p[i] = __ldcg(a.part_ml + slot * kRows + at);
                v[i] = __ldcg(a.part_o + (slot * 32 + d4) * kRows + at);
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (e0 + SPLIT * i >= n_parts) p[i].x = -INFINITY;
                top = fmaxf(top, p[i].x);
            }
            const float fm = m == -INFINITY ? 0.f : ex2(m - top);
            l *= fm; o.x *= fm; o.y *= fm; o.z *= fm; o.w *= fm;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (p[i].x == -INFINITY) {           // (its sums may never have been written; a sum of weights is 0 or NaN)
                    if (e0 + SPLIT * i < n_parts) l += p[i].y;
                    continue;
                }
                const float f = ex2(p[i].x - top);
                l = fmaf(p[i].y, f, l);
                o.x = fmaf(v[i].x, f, o.x); o.y = fmaf(v[i].y, f, o.y); o.z = fmaf(v[i].z, f, o.z); o.w = fmaf(v[i].w, f, o.w);
            }
            m = top;
        }
    }
    if constexpr (SPLIT > 1) {
        sh_o[part][lane] = o;
        sh_ml[part][lane] = make_float2(m, l);
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int i = 1; i < SPLIT; ++i) {
            const float2 p = sh_ml[i][lane];
            const float4 v = sh_o[i][lane];
            if (p.x == -INFINITY) {
                l += p.y;
                continue;
            }
            const float top = fmaxf(m, p.x), fm = m == -INFINITY ? 0.f : ex2(m - top), fp = ex2(p.x - top);
            l = fmaf(p.y, fp, l * fm);
            o.x = fmaf(v.x, fp, o.x * fm); o.y = fmaf(v.y, fp, o.y * fm);
            o.z = fmaf(v.z, fp, o.z * fm); o.w = fmaf(v.w, fp, o.w * fm);
            m = top;
        }
    }
    if (!mine) return;
    const Join j = join(m, l, shift, a.own_lse != nullptr, own_l);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j.fo != 0.f) v = make_float4(o.x * j.fo, o.y * j.fo, o.z * j.fo, o.w * j.fo);
    if (j.fown != 0.f) {
        v.x = fmaf(own.x, j.fown, v.x); v.y = fmaf(own.y, j.fown, v.y);
        v.z = fmaf(own.z, j.fown, v.z); v.w = fmaf(own.w, j.fown, v.w);
    }
    reinterpret_cast<float4*>(a.out + out_row * kHeadDim)[d4] = v;
    if (a.lse && d4 == 0) a.lse[out_row] = j.lse;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// The workspace has to be sized without a device, so the partial slots are counted for this many CTAs.
constexpr int kPlanSms = 148;

constexpr size_t kSlots = 3 * (size_t)kPlanSms * 2;          // first and last partial and a scratch slot, two groups

}  // namespace

size_t prefix_ws_bytes(const Geom& g) {
    return 256 + align256(kPlanSms * 4) + align256(((size_t)g.B + 3) * 8) + kSlots * kRows * 8 + kSlots * kRows * kHeadDim * 4 +
           2 * (size_t)kPlanSms * kRows * kHeadDim * 4;
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
    a.cta_status = reinterpret_cast<int32_t*>(w);
    w += align256(kPlanSms * 4);
    a.base = reinterpret_cast<long long*>(w);
    w += align256(((size_t)g.B + 3) * 8);
    a.part_ml = reinterpret_cast<float2*>(w);
    w += kSlots * kRows * 8;
    a.part_o = reinterpret_cast<float4*>(w);
    w += kSlots * kRows * kHeadDim * 4;
    a.flush = reinterpret_cast<float4*>(w);
    a.cap_groups = cap_groups;
    a.G = g.B; a.Hq = g.Hq; a.Hkv = g.Hkv; a.Gq = g.Gq; a.T = g.T; a.n_rows = n_rows;
    a.quarter = 32 / g.Gq;
    a.seqs = 4 * a.quarter;
    a.q_box = 32 % g.Gq == 0 ? 2 : 1;
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
        const cuuint32_t box[3] = {64, (cuuint32_t)g.Gq, (cuuint32_t)(a.q_box * a.quarter)}, step[3] = {1, 1, 1};
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
    const int chunks = (int)(((long long)n_rows * g.Gq + 7) / 8);    // times Hkv: below 2^31, as n_rows * Hq is
    // about how many parts a row has: CTAs per unit (if the prefixes are alike) times copies
    const bool split = (n_cta / g.problems + 1) * (n_rows <= 2 * a.quarter ? 2 : 1) > 24;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(chunks * g.Hkv), split ? 8 : 1);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute early;                       // its blocks wait in place instead of behind a launch
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    return split ? cudaLaunchKernelEx(&cfg, prefix_merge_kernel<8>, a, n_cta, chunks)
                 : cudaLaunchKernelEx(&cfg, prefix_merge_kernel<1>, a, n_cta, chunks);
}

}  // namespace stc
