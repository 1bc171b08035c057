// Attention for trees of drafted tokens over a routed cache.
//
//   Row r = (node i, query head) of a (sequence, KV head):  softmax over the valid tokens of the listed pages and the nodes N_i
//   (node i and its ancestors) of s = sm_scale * q.k (+ options of stc_score),  out = sum p v~,  lse = log sum exp s.
//
// Rows (32, 64 or 128: whole nodes with their query heads) are the lanes of tensor memory, 128 tokens (8 pages, or the tree itself) a tile:
//   S[row][token] = Q . K^T       Q, K tiles by TMA (128-byte swizzle), M = 128, N = 128, K = 128
//   O[row][dim]  += P . V~        P from tensor memory, written over S by the softmax; V~ rebuilt from the packed groups
//                                 in shared memory, token rows of 128 dims = N-major operand
// Fewer than 128 rows are loaded several times.  The products cost the same, every copy of a row has all its scores; a copy weighs its share
// of the tile's tokens, writes zeros for the others, and the copies' outputs add up at the end.  So the exponentials of a tile, 1024
// cycles of an SM with 128 rows, go with the rows.
// (Tried first: tokens as lanes and rows as columns, which leaves no lane idle.  Weights then pass through shared memory, sums take a
// register per row, maxima need the other warps, and the unrolled columns do not fit the instruction cache: 3200 cycles per tile
// with 16 rows, 5000 with 128; in this form 2600 and 3100.)
// P enters as a bf16 high part plus a bf16 residual (two MMAs): the output is fp32, and one bf16 weight alone would leave it 2^-8 off;
// the pair leaves 2^-16.
//
// Work split.  Unit = (sequence, KV head, block of nodes); its tiles are eight listed pages each and, last, the tree.  The tiles
// of all units form one flat sequence that is cut into equal contiguous ranges, one per CTA (one CTA per SM).  A unit within
// a range is finished in place; of others each CTA leaves (max, sum, accumulator), which a second kernel joins in CTA order:
// no atomics, the same bits every time.  (Joining in the CTA that is through last, with a counter per unit: 1x8 heads 19 -> 25 us, 8x28/4
// 78 -> 89: cold instructions and dependent loads at the end of every segment.)
//
// Roles (16 warps): 0 = TMA producer of Q and K, which also tells which tokens of a tile there are; 1 = issuer of S, 2 = issuer of O;
// 3 = scheduler, and the ancestors of a tree's nodes as bit masks (pointer doubling); 4..7 and 8..11 = softmax, two warps for each 32
// lanes, which have 64 tokens of a tile and later 64 channels of the output each and tell each other their maxima; 12..15 rebuild the value
// tiles with 16-byte asynchronous copies straight from the packed store into the swizzled tile, 32 tokens of every tile each.
// Three score buffers of 128 columns and O fill the tensor memory.
//
// The running maximum only moves when a tile exceeds it by more than 2^24, so the accumulator in tensor memory is rescaled a few times
// per segment and not per tile.  The tensor core truncates when it adds to an accumulator (4e-8 of its value per product, 16
// products per tile), so an accumulator is emptied every kFlush tiles into fp32 sums, which the softmax warps hold in registers (184 a
// thread, the other warps 72).  A unit's tree comes first, then its pages from the last to the first: with a distance bias the
// largest scores come first.
//
// What bounds it (16x32/8 heads, 256 listed pages; measured by leaving parts out): with 64 nodes (two blocks, 127 us) the softmax, 102
// without it, and a little the value copies, 123 without them; with 16 nodes and documents (74 us) not the softmax (75 without it), but the
// way of a tile from its page ids over TMA, S, softmax and O, two tiles of K and three of S deep; half of its pages are hidden and go the
// same way.  8x28/4 chain, cap and window (72 us): 62 without the softmax, 66 without the value copies.  Three K stages, keys prefetched
// into L2, one copy per page instead of two, the next tile's maximum before the weights of this one: no gain.
//
// Every wait is bounded (about a second); one that expires raises a CTA-wide flag and STC_ERR_TIMEOUT in the status word, the
// roles leave, the producer waits (bounded) for its copies, tensor memory is freed.
#include <type_traits>

#include "cap.cuh"

namespace stc {
namespace {

constexpr int kTok = 128;                         // tokens per tile = tensor-memory columns of its scores
constexpr int kTilePages = kTok / kPage;
constexpr int kThreads = 512;
constexpr int kSegs = 2;                          // segments the scheduler may be ahead
constexpr int kSegReaders = 15;                   // warps that follow the segments: all but the scheduler
constexpr uint32_t kHalf = kTok * 128;            // 64 channels of a token tile: 128 rows of 128 bytes
constexpr uint32_t kTile = 2 * kHalf;             // 32 KiB
constexpr uint32_t kSlot = kTile / 2;             // values of 64 tokens: two halves of 64 channels
constexpr int kRows = 128;                        // tensor-memory lanes
constexpr int kFlush = 4;                         // tiles that an accumulator takes: 64 products, at most 2.6e-6 of it
constexpr int kBufs = 3;                          // score buffers: 128 columns each, and 128 for O
constexpr unsigned long long kWaitNs = 1000000000ull;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 24.f;                    // log2 units a maximum may be exceeded by: weights up to 2^24 are as exact as others
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72;           // of the 128 per thread of the launch; 168, 176, 184: 8x28/4 chain 73.9, 73.2, 71.8 us
static_assert(256 * kSoftmaxRegs + 256 * kOtherRegs <= 128 * kThreads, "registers of a block");
constexpr int kKStages = 2, kVSlots = 6;          // K tiles; half V tiles

// barriers, in 8-byte words of the control block; S, P, O per score buffer
enum { kQFull, kQEmpty, kKFull, kKEmpty = kKFull + kKStages, kVFull = kKEmpty + kKStages, kVEmpty = kVFull + kVSlots,
       kSFull = kVEmpty + kVSlots, kPFull = kSFull + kBufs, kOFull = kPFull + kBufs, kPair = kOFull + kBufs, kTabFull = kPair + 4,
       kTabEmpty, kSegFull, kSegEmpty = kSegFull + kSegs, kBars = kSegEmpty + kSegs };
constexpr int kRing = 6;                          // tiles whose valid tokens are kept: K stages, score buffers and one more
constexpr uint32_t kQHalf = kRows * 128;
constexpr uint32_t kOffK = 2 * kQHalf, kOffV = kOffK + kKStages * kTile, kOffCtl = kOffV + kVSlots * kSlot;
constexpr uint32_t kCtlTmem = 304, kCtlAbort = 308, kCtlSegs = 320, kCtlValid = kCtlSegs + kSegs * 48,            // [ring][4 words]
                   kCtlIds = kCtlValid + kRing * 16, kCtlPos = kCtlIds + kRing * 32,                              // [ring][8 pages], [128]
                   kCtlKin = (kCtlPos + 512 + 15) / 16 * 16,                                                      // [128 nodes][4 words]
                   kCtlMl = kCtlKin + STC_TREE_MAX_NODES * 16, kCtlBytes = kCtlMl + 2 * kRows * 8;                // [2][2 groups][128]
constexpr uint32_t kSmem = kOffCtl + kCtlBytes;
static_assert(kBars * 8 <= kCtlTmem && kSmem <= 232448, "shared memory of a block");

struct TreeArgs {
    const int32_t* seq_len;
    const int32_t* n_nodes;
    const int32_t* parent;       // or nullptr: a chain
    const int32_t* page_ids;     // or nullptr: all pages
    const int32_t* n_pages;
    const uint16_t* v_mask;
    const uint32_t* v_offs;
    const uint4* v_packed;
    const uint4* v_new;
    float* out;
    float* lse;                  // or nullptr
    int32_t* status;             // [B]
    int32_t* word;               // the call's status word
    int32_t* cta_status;         // [grid]
    int4* split;                 // [grid] the unit that a CTA begins and leaves to others: problem (-1: none), block, last CTA, nodes
    float2* part_ml;             // [2 * grid][128 lanes]
    float4* part_o;              // [3 * grid][32][128 lanes]: first and last partial of a CTA, and a place to add copies up
    int64_t cap_groups;
    int B, Hq, Hkv, Gq, S, T, n_cap, max_pages, problems;
    int rows;                    // rows of a block: 32, 64 or 128
    int block_nodes;             // nodes of a block = rows / Gq
    uint32_t gq_inv;             // row / Gq = row * gq_inv >> 16 for rows below 128
    float scale_log2, cap_in, cap_log2;
    uint32_t window;             // tokens a row sees, 0xFFFFFFFF without a window
    ScoreArgs sc;
};

__device__ __forceinline__ int nodes_of(const TreeArgs& a, int b) {
    return a.n_nodes ? min(max(a.n_nodes[b], 0), a.n_cap) : a.n_cap;
}
// Pages that a problem attends: `list` of them, from `first` on where there is no list (nothing before it is in the window).
__device__ __forceinline__ void pages_of(const TreeArgs& a, int problem, int len, int& list, int& first) {
    first = 0;
    if (a.page_ids) {
        list = min(max(a.n_pages[problem], 0), a.max_pages);
        return;
    }
    if (a.sc.window > 0 && !a.sc.q_pos && len >= a.sc.window) first = (len - a.sc.window + 1) / kPage;
    list = (len + kPage - 1) / kPage - first;
}
struct Unit { int tiles, blocks; };              // tiles of a unit of the problem (the tree's among them), units
__device__ __forceinline__ Unit unit_of(const TreeArgs& a, int nodes, int list) {
    return Unit{1 + (list + kTilePages - 1) / kTilePages, (nodes + a.block_nodes - 1) / a.block_nodes};
}
__device__ __forceinline__ int problem_length(const TreeArgs& a, int problem) {
    const int b = problem / a.Hkv, nodes = nodes_of(a, b);
    int list, first;
    pages_of(a, problem, clamp_len(a.seq_len, b, a.T), list, first);
    const Unit u = unit_of(a, nodes, list);
    return u.tiles * u.blocks;
}
// The flat sequence is cut into `n` ranges of `each` tiles, the first `more` of them one longer.
struct Cut {
    int n, each, more;
    __device__ __forceinline__ Cut(int total, int grid) {
        n = min(total, grid);
        each = n > 0 ? (int)((uint32_t)total / (uint32_t)n) : 0;
        more = total - each * n;
    }
    __device__ __forceinline__ int begin(int c) const { return c * each + min(c, more); }
    __device__ __forceinline__ int owner(int x) const {                       // of position x
        const int longer = more * (each + 1);
        return x < longer ? (int)((uint32_t)x / (uint32_t)(each + 1)) : more + (int)((uint32_t)(x - longer) / (uint32_t)each);
    }
};

// One segment: tiles [tile0, tile1) of one unit.
struct Segment {
    int b, hk, node0, nodes, len, list, first, tile0, tile1;
    int slot;                    // partial slot, -1 = the whole unit
};

// Bounded wait of a converged warp for a barrier's phase; false once it expired or another role has given up.  One copy of
// the instructions that ask (a kernel with fifty waits is bound by fetching its own code otherwise), and the clock, which is read faster
// than the timer; its limit is a second at the highest clock.
__device__ __forceinline__ bool warp_wait_clocked(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
    const long long t0 = clock64();
#pragma unroll 1
    for (;;) {
        if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
        if (__any_sync(0xFFFFFFFFu, *abort_flag != 0 || clock64() - t0 > 2000000000ll)) return false;
    }
}
// Asynchronous 16-byte copy global -> shared; zeros, and nothing is read, where `take` is 0.
__device__ __forceinline__ void cp_async16_if(uint32_t dst, const void* src, uint32_t take) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.u32 p, %2, 0;\n\tcp.async.cg.shared.global [%0], [%1], 16, p;\n\t}"
                 ::"r"(dst), "l"(src), "r"(take) : "memory");
}
// MASK: a window, documents or positions that are given; SCORE: cap, slopes, or a scale that is not positive (with MASK).
// R rows of a block; the lanes hold 128 / R copies of them.  APART: a window and given positions, whose windows may lie apart (a variant
// of its own: with the look-up in all of them 16x32/8 heads, 16 nodes, documents took 78 us, now 73, the 8x28/4 chain 78, now 70).
template <int R, bool MASK, bool SCORE, bool APART>
__global__ void __launch_bounds__(kThreads, 1)
tree_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_new, const TreeArgs a) {
    static_assert(MASK || !(SCORE || APART), "SCORE and APART need the positions");
    constexpr int kCopies = kRows / R, kCols = R / 2;         // tokens of a tile that a thread weighs
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const uint32_t bars = base + kOffCtl;
    unsigned char* const ctl = smem + kOffCtl;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctl + kCtlTmem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(ctl + kCtlAbort);
    volatile int* segs = reinterpret_cast<volatile int*>(ctl + kCtlSegs);                   // [kSegs][12]
    uint32_t* const kin = reinterpret_cast<uint32_t*>(ctl + kCtlKin);
    int* const node_pos = reinterpret_cast<int*>(ctl + kCtlPos);
    float* const told = reinterpret_cast<float*>(ctl + kCtlMl);
    volatile uint32_t* const valid_tokens = reinterpret_cast<volatile uint32_t*>(ctl + kCtlValid);
    volatile int* const tile_pages = reinterpret_cast<volatile int*>(ctl + kCtlIds);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;");

    // ---- set-up: barriers, tensor memory, and where this CTA's range begins -----------------------------------------------
    if (warp == 0 && lane < 3)
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &map_q : lane == 1 ? &map_k : &map_new) : "memory");
    if (threadIdx.x >= 64 && threadIdx.x < 64 + kBars) {
        const int i = (int)threadIdx.x - 64;
        mbar_init(bars + 8 * i, i >= kVFull && i < kVEmpty ? 2 : i >= kPFull && i < kOFull ? 8
                                : i >= kPair && i < kTabFull ? 2 * kCopies : i == kTabEmpty ? 8
                                : i >= kSegEmpty ? kSegReaders : 1);
        fence_mbar_init();
    }
    if (threadIdx.x == 4) *abort_flag = (base & 1023u) != 0 ? (int)STC_ERR_CUDA : 0;        // swizzled tiles need 1024-byte aligned bases
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(bars + kCtlTmem), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // thread = `per` problems; prefix sums over the block
    const int per = (a.problems + kThreads - 1) / kThreads;
    const int p_lo = min((int)threadIdx.x * per, a.problems), p_hi = min(p_lo + per, a.problems);
    int mine = 0;
#pragma unroll 1
    for (int p = p_lo; p < p_hi; ++p) mine += problem_length(a, p);
    const int incl = (int)warp_incl_scan((uint32_t)mine, lane);
    volatile int* const sums = reinterpret_cast<volatile int*>(kin);      // [16] of the warps, then problem and offset of the range
    if (lane == 31) sums[warp] = incl;
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_slot;
    int total, x_begin = 0, x_end = 0;
    {
        const int of_warp = lane < kThreads / 32 ? sums[lane] : 0;
        const int upto = (int)warp_incl_scan((uint32_t)of_warp, lane);
        total = __shfl_sync(0xFFFFFFFFu, upto, 31);
        const int before = __shfl_sync(0xFFFFFFFFu, upto - of_warp, warp) + incl - mine;
        const Cut cut(total, (int)gridDim.x);
        if ((int)blockIdx.x < cut.n) {
            x_begin = cut.begin((int)blockIdx.x);
            x_end = cut.begin((int)blockIdx.x + 1);
        }
        const bool holds = x_begin < x_end && before <= x_begin && x_begin < before + mine;
        if (holds) {
            int at = before;
#pragma unroll 1
            for (int p = p_lo; p < p_hi; ++p) {
                const int n = per > 1 ? problem_length(a, p) : mine;
                if (at <= x_begin && x_begin < at + n) {
                    sums[16] = p;
                    sums[17] = x_begin - at;
                }
                at += n;
            }
        }
    }
    __syncthreads();
    const int p_first = sums[16], x_first = sums[17];
    __syncthreads();                                 // (the ancestors' table takes their place)
    if (threadIdx.x == 96) a.split[blockIdx.x] = make_int4(-1, 0, 0, 0);         // (the scheduler's)

    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto warp_wait = [&](int i, uint32_t phase) { return warp_wait_clocked(bar(i), phase & 1u, abort_flag); };
    auto give_up = [&]() { atomicCAS(const_cast<int*>(abort_flag), 0, (int)STC_ERR_TIMEOUT); };
    Segment s;
    int n_seg = 0;
    // the next segment, for a whole warp; false at the end
    auto next = [&](bool& good) -> bool {
        good = warp_wait(kSegFull + n_seg % kSegs, (uint32_t)(n_seg / kSegs));
        if (!good) return false;
        volatile int* e = segs + (n_seg % kSegs) * 12;
        s.b = e[0]; s.hk = e[1]; s.node0 = e[2]; s.nodes = e[3]; s.len = e[4]; s.list = e[5]; s.first = e[6];
        s.tile0 = e[7]; s.tile1 = e[8]; s.slot = e[9];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kSegEmpty + n_seg % kSegs));
        ++n_seg;
        return s.tile1 >= 0;
    };
    // the tree is the last tile of a unit, and the first that is taken; before it stand eight listed pages each
    auto is_tree = [&](int t) { return t * kTilePages >= s.list; };
    // entry j of the segment's page list as it stands there, to be asked for ahead of its use; -1 outside the list
    auto listed = [&](int j) {
        if (j < 0 || j >= s.list) return -1;
        return a.page_ids ? __ldg(a.page_ids + (size_t)(s.b * a.Hkv + s.hk) * a.max_pages + j) : s.first + j;
    };
    auto is_page = [&](int id) { return id >= 0 && id < (s.len + kPage - 1) / kPage; };

    // the softmax warps hold 64 channels of their rows besides a tile's scores; the registers are moved within each role, where ptxas
    // sees how many there are
    auto fewer_registers = [] { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs)); };
    if (*abort_flag) {
        // nothing was started
    } else if (warp < 4) {
        fewer_registers();
        if (warp == 0) {
            // ---- producer of Q and K ---------------------------------------------------------------------------
            int kc = 0, seg = 0, ring = 0;
            uint32_t st = 0, phase = 1;                  // K stage, and the phase in which it is empty (of the second round on)
            bool ok = true;
            const uint32_t q_bytes = 2u * 128u * (uint32_t)(a.Gq * a.block_nodes * kCopies);
            while (ok && next(ok)) {
                const int problem = s.b * a.Hkv + s.hk;
                const int32_t* const doc_row = MASK && a.sc.tok_doc ? a.sc.tok_doc + (size_t)s.b * a.T : nullptr;
                const int q_doc = doc_row ? a.sc.q_doc[s.b] : 0;
                // pages of a tile in lanes 0 .. 7, asked for two tiles ahead; documents of its tokens (32 c + lane) one tile ahead
                auto ask = [&](int t) { return lane < kTilePages && t >= s.tile0 ? listed(t * kTilePages + lane) : -1; };
                int doc[4];
                auto ask_docs = [&](int pages) {
                    if (MASK && doc_row) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int page = __shfl_sync(0xFFFFFFFFu, pages, 2 * c + (lane >> 4)), t = page * kPage + (lane & 15);
                            doc[c] = is_page(page) && t < s.len ? __ldg(doc_row + t) : -1;
                        }
                    }
                };
                int id = ask(s.tile1 - 1), id_next = ask(s.tile1 - 2);
                ask_docs(id);
                bool q_due = true;
#pragma unroll 1
                for (int t = s.tile1 - 1; t >= s.tile0; --t) {
                    // tokens of the tile that there are: 16 bits per page, a word per softmax warp of a group
                    const bool tree = is_tree(t);
                    const int here = !tree ? (is_page(id) ? min(kPage, s.len - id * kPage) : 0) : min(max(s.nodes - lane * kPage, 0), kPage);
                    uint32_t word = (1u << here) - 1u;
                    word = (word | __shfl_down_sync(0xFFFFFFFFu, word, 1) << 16);                // (lanes 0, 2, 4, 6)
                    word = __shfl_sync(0xFFFFFFFFu, word, 2 * lane & 7);
                    if (MASK && doc_row && !tree) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t same = __ballot_sync(0xFFFFFFFFu, doc[c] < 0 || doc[c] == q_doc);
                            if (lane == c) word &= same;
                        }
                    }
                    if (kc >= kKStages) ok = warp_wait(kKEmpty + st, phase);
                    if (!ok) break;
                    if (lane < 4) valid_tokens[ring * 4 + lane] = word;
                    if (MASK && lane < kTilePages) tile_pages[ring * kTilePages + lane] = id;
                    if (++ring == kRing) ring = 0;
                    __syncwarp();
                    const uint32_t full = bar(kKFull + st), dst = base + kOffK + st * kTile;
                    if (tree || !a.page_ids) {           // consecutive rows: two copies of 64 channels
                        if (elect_one()) {
                            const CUtensorMap* map = tree ? &map_new : &map_k;
                            const int y = tree ? problem * a.n_cap : problem * a.T + (s.first + t * kTilePages) * kPage;
                            mbar_expect_tx(full, (uint32_t)(tree ? a.n_cap : kTok) * kRowBytes);
                            tma_2d(dst, map, 0, y, full);
                            tma_2d(dst + kHalf, map, 64, y, full);
                        }
                    } else {                             // two copies per page.  (From eight lanes at once they take 1300 cycles.)
                        const uint32_t pages = __ballot_sync(0xFFFFFFFFu, is_page(id));
                        if (elect_one()) mbar_expect_tx(full, (uint32_t)__popc(pages) * kPage * kRowBytes);
                        __syncwarp();
#pragma unroll
                        for (int p = 0; p < kTilePages; ++p) {
                            const int y = problem * a.T + __shfl_sync(0xFFFFFFFFu, id, p) * kPage;
                            if (((pages >> p) & 1u) && elect_one()) {
                                tma_2d(dst + p * kPage * 128, &map_k, 0, y, full);
                                tma_2d(dst + kHalf + p * kPage * 128, &map_k, 64, y, full);
                            }
                        }
                    }
                    __syncwarp();
                    ++kc;
                    if (++st == (uint32_t)kKStages) { st = 0; phase ^= 1u; }
                    id = id_next;
                    id_next = ask(t - 2);
                    ask_docs(id);
                    if (q_due) {                         // the queries behind the first keys, which come from farther away
                        q_due = false;
                        if (seg > 0) ok = warp_wait(kQEmpty, (uint32_t)(seg - 1));
                        if (!ok) break;
                        if (lane == 0) {
                            mbar_expect_tx(bar(kQFull), q_bytes);
#pragma unroll
                            for (int i = 0; i < kCopies; ++i) {
                                tma_3d(base + i * R * 128, &map_q, 0, s.hk * a.Gq, s.b * a.n_cap + s.node0, bar(kQFull));
                                tma_3d(base + kQHalf + i * R * 128, &map_q, 64, s.hk * a.Gq, s.b * a.n_cap + s.node0, bar(kQFull));
                            }
                        }
                        __syncwarp();
                        ++seg;
                    }
                }
            }
            if (!ok) give_up();
            if (*abort_flag) {                           // copies still in flight get one more bounded wait each
                int none = 0;
                if (seg > 0) mbar_wait_or_abort(bar(kQFull), (uint32_t)(seg - 1) & 1u, &none, kWaitNs);
                for (int i = max(0, kc - kKStages); i < kc; ++i)
                    mbar_wait_or_abort(bar(kKFull + i % kKStages), (uint32_t)(i / kKStages) & 1u, &none, kWaitNs);
            }
        } else if (warp == 1) {
            // ---- issuer of S = Q K^T: the warp stays together, an elected lane issues ----------------------------------------
            constexpr uint32_t id_s = idesc_bf16(kRows, kTok, false);
            const uint32_t sm = uniform(base), ts = uniform(tmem);
            const uint64_t dq = smem_desc_128(sm, 16), dk0 = smem_desc_128(sm + kOffK, 16);
            uint32_t st = 0, phase = 0, seg = 0, buf = 0, turn = 0;      // K stage and its phase; segments; score buffer, its uses so far
            bool ok = true;
            while (ok && next(ok)) {
                const int tiles = (int)__reduce_max_sync(0xFFFFFFFFu, (uint32_t)(s.tile1 - s.tile0));
                ok = warp_wait(kQFull, seg);
#pragma unroll 1
                for (int n = 0; ok && n < tiles; ++n) {
                    // the buffer holds the weights of an earlier tile until their product is through
                    ok = warp_wait(kKFull + st, phase) && (turn == 0 || warp_wait(kOFull + buf, turn - 1u));
                    if (!ok) break;
                    tc_after();
                    const uint64_t dk = dk0 + (uint64_t)(st * (kTile >> 4));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)      // 16 dims = 32 bytes = 2 units; 64 dims = one half tile
                            tc_mma_ss(ts + buf * kTok, dq + (uint64_t)((k >> 2) * (kQHalf >> 4) + (k & 3) * 2),
                                      dk + (uint64_t)((k >> 2) * (kHalf >> 4) + (k & 3) * 2), id_s, k != 0);
                        tc_commit_to(bar(kSFull + buf));
                        tc_commit_to(bar(kKEmpty + st));
                        if (n == tiles - 1) tc_commit_to(bar(kQEmpty));
                    }
                    __syncwarp();
                    if (++buf == (uint32_t)kBufs) { buf = 0; ++turn; }
                    if (++st == (uint32_t)kKStages) { st = 0; phase ^= 1u; }
                }
                ++seg;
            }
            if (!ok) give_up();
        } else if (warp == 2) {
            // ---- issuer of O += P V~ ----------------------------------------------------------------------------------------
            constexpr uint32_t id_o = idesc_bf16(kRows, kHeadDim, true);
            const uint32_t sm = uniform(base), ts = uniform(tmem), to = ts + kBufs * kTok;
            const uint64_t dv0 = smem_desc_128(sm + kOffV, kSlot / 2);
            uint32_t slot = 0, phase = 0, buf = 0, turn = 0;
            bool ok = true;
            while (ok && next(ok)) {
                const int tiles = (int)__reduce_max_sync(0xFFFFFFFFu, (uint32_t)(s.tile1 - s.tile0));
#pragma unroll 1
                for (int n = 0; ok && n < tiles; ++n) {
                    const uint32_t next_slot = slot + 1u;                        // (a tile's slots are neighbours)
                    ok = warp_wait(kVFull + slot, phase) && warp_wait(kVFull + next_slot, phase) && warp_wait(kPFull + buf, turn);
                    if (!ok) break;
                    tc_after();
                    const uint64_t dv = dv0 + (uint64_t)(slot * (kSlot >> 4));
                    const uint32_t p = ts + buf * kTok, more = (uint32_t)(n % kFlush != 0);               // else O starts anew
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {    // 16 tokens: 16 rows of 128 bytes; P: 8 columns high, 8 residual
                            const uint64_t d = dv + (uint64_t)((k >> 2) * (kSlot >> 4) + (k & 3) * (2048 >> 4));
                            tc_mma_ts(to, p + 16 * k, d, id_o, k ? 1u : more);
                            tc_mma_ts(to, p + 16 * k + 8, d, id_o, 1);
                        }
                        tc_commit_to(bar(kOFull + buf));
                        tc_commit_to(bar(kVEmpty + slot));
                        tc_commit_to(bar(kVEmpty + next_slot));
                    }
                    __syncwarp();
                    if (++buf == (uint32_t)kBufs) { buf = 0; ++turn; }
                    slot += 2;
                    if (slot == (uint32_t)kVSlots) { slot = 0; phase ^= 1u; }
                }
            }
            if (!ok) give_up();
        } else if (warp == 3) {
            // ---- scheduler: walks the CTA's range, segment by segment; and, behind each, the ancestors of its nodes as bit masks
            bool ok = true;
            int x = x_begin, p = p_first, off = x_first;
            uint32_t made = 0;                           // tables
#pragma unroll 1
            for (int i = 0; ok; ++i) {
                Segment g = {};
                g.tile1 = -1;
#pragma unroll 1
                while (x < x_end) {
                    g.b = (int)((uint32_t)p / (uint32_t)a.Hkv);
                    g.hk = p - g.b * a.Hkv;
                    g.len = clamp_len(a.seq_len, g.b, a.T);
                    g.nodes = nodes_of(a, g.b);
                    pages_of(a, p, g.len, g.list, g.first);
                    const Unit u = unit_of(a, g.nodes, g.list);
                    if (off >= u.tiles * u.blocks) {
                        off -= u.tiles * u.blocks;
                        ++p;
                        continue;
                    }
                    const int blk = (int)((uint32_t)off / (uint32_t)u.tiles);
                    g.tile0 = off - blk * u.tiles;
                    g.tile1 = min(u.tiles, g.tile0 + (x_end - x));
                    g.node0 = blk * a.block_nodes;
                    // a CTA continues at most one unit (slot 0) and leaves at most one that it begins (slot 1)
                    g.slot = g.tile1 - g.tile0 == u.tiles ? -1 : 2 * (int)blockIdx.x + (g.tile0 == 0 ? 1 : 0);
                    if (lane == 0 && g.slot > 0 && (g.slot & 1))
                        a.split[blockIdx.x] = make_int4(p, blk, Cut(total, (int)gridDim.x).owner(x + u.tiles - 1), g.nodes);
                    x += g.tile1 - g.tile0;
                    off += g.tile1 - g.tile0;
                    break;
                }
                if (i >= kSegs) ok = warp_wait(kSegEmpty + i % kSegs, (uint32_t)(i / kSegs - 1));
                if (!ok) break;
                if (lane == 0) {
                    volatile int* e = segs + (i % kSegs) * 12;
                    e[0] = g.b; e[1] = g.hk; e[2] = g.node0; e[3] = g.nodes; e[4] = g.len; e[5] = g.list; e[6] = g.first;
                    e[7] = g.tile0; e[8] = g.tile1; e[9] = g.slot;
                    mbar_arrive(bar(kSegFull + i % kSegs));
                }
                __syncwarp();
                if (g.tile1 < 0) break;
                if (!MASK && (g.tile1 - 1) * kTilePages < g.list) continue;      // nobody asks for the tree
                int up[4];
                uint32_t m[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int node = k * 32 + lane;
                    up[k] = -1;
                    if (node < g.nodes) {
                        up[k] = a.parent ? a.parent[(size_t)g.b * a.n_cap + node] : node - 1;
                        if (up[k] < 0 || up[k] >= node) up[k] = -1;
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) m[k][w] = w == k ? 1u << lane : 0u;
                }
                if (made > 0) ok = warp_wait(kTabEmpty, made - 1);
                if (!ok) break;
                // each node's mask holds the node and its ancestors up to the one `up` points at, twice as many each time
                uint4* const table = reinterpret_cast<uint4*>(kin);
#pragma unroll 1
                for (;;) {
                    bool going = false;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        table[k * 32 + lane] = make_uint4(m[k][0], m[k][1], m[k][2], m[k][3]);
                        going |= up[k] >= 0;
                    }
                    __syncwarp();
                    if (!__any_sync(0xFFFFFFFFu, going)) break;
                    int next_up[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        // the node that `up` points at: its mask, and where its pointer goes (held by its lane)
                        const uint4 t = table[max(up[k], 0)];
                        int to[4];
#pragma unroll
                        for (int w = 0; w < 4; ++w) to[w] = __shfl_sync(0xFFFFFFFFu, up[w], max(up[k], 0) & 31);
                        const int which = max(up[k], 0) >> 5;
                        next_up[k] = up[k] < 0 ? -1 : which == 0 ? to[0] : which == 1 ? to[1] : which == 2 ? to[2] : to[3];
                        if (up[k] >= 0) { m[k][0] |= t.x; m[k][1] |= t.y; m[k][2] |= t.z; m[k][3] |= t.w; }
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 4; ++k) up[k] = next_up[k];
                }
                if constexpr (MASK) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int node = k * 32 + lane;
                        const int depth = __popc(m[k][0]) + __popc(m[k][1]) + __popc(m[k][2]) + __popc(m[k][3]) - 1;
                        node_pos[node] = a.sc.q_pos && node < g.nodes ? a.sc.q_pos[(size_t)g.b * a.n_cap + node] : g.len + depth;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kTabFull));
                ++made;
            }
            if (!ok) give_up();
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ---- softmax: thread = a row and kCols of a tile's 128 tokens: a lane has 64 of them in each of its two warps, a copy its
        // part of those and zeros elsewhere -----------------------------------------------------------------------------
        constexpr int kStep = kCols < 32 ? kCols : 32;           // of them at a time
        constexpr bool kHeld = kCols == kStep;                   // a tile's scores stay in registers from the maximum to the weights
        const int grp = (warp - 4) >> 2, quarter = warp & 3, place = quarter * 32 + lane, row = place % R, copy = place / R;
        const int half = 64 * grp, c0 = half + copy * kCols;     // first token; half: first channel of those that this warp looks after
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), to = lanes + kBufs * kTok;
        uint32_t buf = 0, turn = 0, last_buf = 0, last_turn = 0, ring = 0;   // score buffer and its uses so far, of the tile before too
        uint32_t pairs = 0, tabs = 0;
        bool ok = true;
        // what the warps that share rows tell each other, a number per row
        constexpr int kTold = 2 * kCopies;
        auto exchange = [&](float mine, float (&all)[kTold]) {
            float* const board = told + (pairs & 1u) * 2 * kRows;
            board[(grp * kCopies + copy) * R + row] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kPair + quarter % (R / 32)));
            if (!warp_wait(kPair + quarter % (R / 32), pairs++)) return false;
#pragma unroll
            for (int i = 0; i < kTold; ++i) all[i] = board[i * R + row];
            return true;
        };
        auto step = [&]() {
            last_buf = buf; last_turn = turn;
            if (++buf == (uint32_t)kBufs) { buf = 0; ++turn; }
            if (++ring == (uint32_t)kRing) ring = 0;
        };

        auto segment = [&]() {
            const int live = min(a.block_nodes, s.nodes - s.node0) * a.Gq;    // rows of the block
            const bool mine = row < live, warp_live = quarter * 32 % R < live;
            const int tiles = s.tile1 - s.tile0;
            const bool tables = MASK || is_tree(s.tile1 - 1);
            const uint32_t in_block = ((uint32_t)row * a.gq_inv) >> 16;
            const int node = min(s.node0 + (int)in_block, STC_TREE_MAX_NODES - 1), h = row - (int)in_block * a.Gq;
            int p = 0;
            float slope2 = 0.f;
            if (MASK) {
                ok = warp_wait(kTabFull, tabs);
                if (!ok) return;
                p = node_pos[node];
                if (SCORE && a.sc.slopes && mine) slope2 = a.sc.slopes[s.hk * a.Gq + h] * kLog2e;
            }
            float m = -INFINITY, l = 0.f, m_sums = -INFINITY;
            float sums[64];                          // the channels of half: sums of emptied accumulators, relative to m_sums
#pragma unroll
            for (int i = 0; i < 64; ++i) sums[i] = 0.f;
#pragma unroll 1
            for (int n = 0; n < tiles; ++n, step()) {
                const int t = s.tile1 - 1 - n;
                ok = warp_wait(kSFull + buf, turn);
                if (!ok) return;
                if (!warp_live) {                    // a quarter without rows: its P may be anything
                    if (lane == 0) mbar_arrive(bar(kPFull + buf));
                    continue;
                }
                const uint32_t ts = lanes + buf * kTok + c0, word0 = (uint32_t)c0 >> 5, shift = (uint32_t)c0 & 31u;
                auto last_product = [&]() {          // the product of the tile before is through
                    const bool good = warp_wait(kOFull + last_buf, last_turn);
                    tc_after();
                    return good;
                };
                tc_after();
                // tokens that the row sees: those that there are, in the tree its ancestors, and the window's
                constexpr int kWords = kCols == 64 ? 2 : 1;
                uint32_t see[kWords];
#pragma unroll
                for (int i = 0; i < kWords; ++i) see[i] = valid_tokens[ring * 4 + word0 + i] >> shift;
                const bool tree = is_tree(t);
                if (tree) {
                    if (!MASK) {
                        ok = warp_wait(kTabFull, tabs);
                        if (!ok) return;
                    }
#pragma unroll
                    for (int i = 0; i < kWords; ++i) see[i] &= kin[node * 4 + word0 + i] >> shift;
                }
                if constexpr (MASK) {
                    if (tree) {
#pragma unroll 1
                        for (int i = 0; i < min(kCols, s.nodes - c0); ++i) {
                            const int at_i = node_pos[c0 + i];
                            if (at_i > p || (uint32_t)p - (uint32_t)at_i >= a.window) {
                                if (i < 32) see[0] &= ~(1u << i);
                                else see[kWords - 1] &= ~(1u << (i - 32));
                            }
                        }
                    } else if (a.sc.q_pos || a.sc.window > 0) {
#pragma unroll
                        for (int i = 0; i < kCols / kPage; ++i) {             // of a page's 16 tokens the bits [lo, hi)
                            const int t0 = tile_pages[ring * kTilePages + c0 / kPage + i] * kPage;
                            const long long ahead = (long long)p - t0;        // distance of its first token
                            const int hi = (int)min(max(ahead + 1, 0LL), 16LL), lo = (int)min(max(ahead + 1 - (long long)a.window, 0LL), 16LL);
                            const uint32_t bits = ((1u << hi) - 1u) & ~((1u << lo) - 1u);
                            see[i >> 1] &= i & 1 ? bits << 16 | 0xFFFFu : bits | 0xFFFF0000u;
                        }
                    }
                }
                constexpr uint32_t kAll = kCols >= 32 ? 0xFFFFFFFFu : (1u << kCols % 32) - 1u;       // the tokens of a word
                const bool open = __all_sync(0xFFFFFFFFu, !mine || (see[0] & see[kWords - 1] & kAll) == kAll);
                const bool empty_now = n > 0 && n % kFlush == 0;
                const float m_acc = m;               // maximum the accumulator was built with
                // maximum of the tile; scores that are not raw products times a positive scale, or hidden, are written back (where a
                // thread has up to 32 they stay in its registers instead: 8x28/4 heads, 5 nodes, capped, 78 -> 73 us)
                float top = -INFINITY;
                uint32_t r[kStep];
#pragma unroll 1
                for (int c = 0; c < kCols; c += kStep) {
                    tmem_ld16<0>(ts + c, r);
                    if constexpr (kStep > 16) tmem_ld16<16>(ts + c + 16, r);
                    tmem_wait_ld();
                    const uint32_t bits = c ? see[kWords - 1] : see[0];
                    if constexpr (SCORE) {
                        if (a.cap_in != 0.f) {
                            // (what a row does not see, and lanes without a row, have no say in how the others are capped)
                            const bool all = __all_sync(0xFFFFFFFFu, (bits & kAll) == kAll || !mine);
                            if (all && __all_sync(0xFFFFFFFFu, (mine ? magnitude(r) : 0.f) * fabsf(a.cap_in) <= kCapSmall))
                                cap_scores_low(r, a.cap_in, a.scale_log2);
                            else
                                cap_scores_any(r, a.cap_in, a.cap_log2);
                        } else {
#pragma unroll
                            for (int i = 0; i < kStep; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * a.scale_log2);
                        }
                        if (a.sc.slopes) {
                            if (tree) {
#pragma unroll
                                for (int i = 0; i < kStep; ++i)
                                    r[i] = __float_as_uint(fmaf(slope2, (float)(node_pos[c0 + c + i] - p), __uint_as_float(r[i])));
                            } else {
#pragma unroll
                                for (int e = 0; e < kStep / kPage; ++e) {
                                    const float far = (float)(tile_pages[ring * kTilePages + (c0 + c) / kPage + e] * kPage - p);
#pragma unroll
                                    for (int i = 0; i < 16; i += 2) {
                                        const float2 x = fma2(both(slope2), add2(both(far), make_float2((float)i, (float)(i + 1))),
                                                              make_float2(__uint_as_float(r[16 * e + i]), __uint_as_float(r[16 * e + i + 1])));
                                        r[16 * e + i] = __float_as_uint(x.x);
                                        r[16 * e + i + 1] = __float_as_uint(x.y);
                                    }
                                }
                            }
                        }
                    }
                    if (!open) {
#pragma unroll
                        for (int i = 0; i < kStep; ++i)
                            if (!((bits >> i) & 1u)) r[i] = __float_as_uint(-INFINITY);
                    }
                    float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < kStep; i += 2)
                        t4[(i >> 1) & 3] = fmaxf(fmaxf(t4[(i >> 1) & 3], __uint_as_float(r[i])), __uint_as_float(r[i + 1]));
                    __syncwarp();
                    top = fmaxf(top, fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
                    if (!kHeld && (SCORE || !open)) {
#pragma unroll
                        for (int e = 0; e < kStep; e += 16) {
                            uint32_t o[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = r[e + i];
                            tmem_st16(ts + c + e, o);
                        }
                    }
                }
                if (!kHeld && (SCORE || !open)) tmem_wait_st();
                if (!SCORE) top *= a.scale_log2;     // (-inf stays -inf: the scale is positive)
                float all_tops[kTold];
                ok = exchange(top, all_tops);
                if (!ok) return;
#pragma unroll
                for (int i = 0; i < kTold; ++i) top = fmaxf(top, all_tops[i]);
                // move the maximum only if it is exceeded by much; the accumulator follows (half of its channels here, half there)
                const bool move = mine && (top > m + kSlack || (m == -INFINITY && top > -INFINITY));
                if (__any_sync(0xFFFFFFFFu, move)) {
                    const float to_m = move ? top : m, f = m == -INFINITY ? 0.f : ex2(m - to_m);
                    l *= f;
                    if (n > 0 && !empty_now) {
                        ok = last_product();
                        if (!ok) return;
#pragma unroll 1
                        for (int c = half; c < half + 64; c += 16) {
                            uint32_t q[16];
                            tmem_ld16(to + c, q);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) q[i] = move ? __float_as_uint(__uint_as_float(q[i]) * f) : q[i];
                            tmem_st16(to + c, q);
                        }
                    }
                    m = to_m;
                }
                // the accumulator is emptied into the sums; the issuer starts it anew
                if (empty_now) {
                    ok = last_product();
                    if (!ok) return;
                    const float keep = m_sums == -INFINITY ? 0.f : ex2(m_sums - m_acc);
#pragma unroll
                    for (int c = 0; c < 64; c += 16) {
                        uint32_t q[16];
                        tmem_ld16(to + half + c, q);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sums[c + i] = fmaf(sums[c + i], keep, __uint_as_float(q[i]));
                    }
                    m_sums = m_acc;
                }
                // weights, their sum, and P over S: per 16 tokens 8 columns of bf16 pairs high, 8 residual
                const float ref = m == -INFINITY ? 0.f : m;
                float2 la = make_float2(0.f, 0.f), lb = la;
#pragma unroll 1
                for (int c = 0; c < kCols; c += kStep) {
                    if constexpr (!kHeld) {
                        tmem_ld16<0>(ts + c, r);
                        if constexpr (kStep > 16) tmem_ld16<16>(ts + c + 16, r);
                        tmem_wait_ld();
                    }
#pragma unroll
                    for (int e = 0; e < kStep; e += 16) {
                        uint32_t o[16];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float2 x = make_float2(__uint_as_float(r[e + 2 * i]), __uint_as_float(r[e + 2 * i + 1]));
                            if constexpr (SCORE) x = add2(x, both(-ref));
                            else x = fma2(x, both(a.scale_log2), both(-ref));
                            x.x = ex2(x.x);
                            x.y = ex2(x.y);
                            if (i & 1) lb = add2(lb, x); else la = add2(la, x);
                            const __nv_bfloat162 h2 = __floats2bfloat162_rn(x.x, x.y);
                            o[i] = *reinterpret_cast<const uint32_t*>(&h2);
                            const float2 d = fma2(make_float2(bf16lo(o[i]), bf16hi(o[i])), both(-1.f), x);
                            const __nv_bfloat162 r2 = __floats2bfloat162_rn(d.x, d.y);
                            o[8 + i] = *reinterpret_cast<const uint32_t*>(&r2);
                        }
                        tmem_st16(ts + c + e, o);
                    }
                }
                if constexpr (kCopies > 1) {         // the tokens of the other copies
                    uint32_t zero[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll
                    for (int c = kCols; c < 64; c += 16) tmem_st16(lanes + buf * kTok + half + ((copy * kCols + c) & 63), zero);
                }
                l += (la.x + lb.x) + (la.y + lb.y);
                tmem_wait_st();
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kPFull + buf));
            }
            // ---- end of the segment: each warp of a quarter writes half of its rows' channels --------------------------------
            ok = warp_wait(kOFull + last_buf, last_turn);
            if (!ok) return;
            tc_after();
            if (warp_live) {
                float told_sums[kTold];
                ok = exchange(l, told_sums);
                if (!ok) return;
                l = 0.f;
#pragma unroll
                for (int i = 0; i < kTold; ++i) l += told_sums[i];
                const bool whole = s.slot < 0;
                const size_t at = ((size_t)s.b * a.n_cap + node) * a.Hq + s.hk * a.Gq + h;
                if (grp == 0 && copy == 0 && mine) {
                    if (!whole) a.part_ml[(size_t)s.slot * kRows + row] = make_float2(m, l);
                    else if (a.lse) a.lse[at] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                }
                __syncwarp();
                const float f = !whole ? 1.f : l != 0.f ? 1.f / l : 0.f;     // (0: nothing seen, whatever was summed)
                const float keep = f * (m_sums == -INFINITY ? 0.f : ex2(m_sums - m));
                // the copies of a row are added up where their CTA finishes it, or by the second kernel
                const bool aside = whole && copy > 0;
                float4* const to_lane = a.part_o + (size_t)(whole ? 2 * (int)gridDim.x + (int)blockIdx.x : s.slot) * 32 * kRows + row;
                float4* const to_row = reinterpret_cast<float4*>(a.out + at * kHeadDim);
#pragma unroll 1
                for (int pass = 0; pass < (kCopies > 1 && whole ? 2 : 1); ++pass) {
                    if (pass == (kCopies > 1 && whole && !aside ? 1 : 0)) {
#pragma unroll
                        for (int c = 0; c < 64; c += 16) {
                            uint32_t q[16];
                            __syncwarp();
                            tmem_ld16(to + half + c, q);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int at4 = half / 4 + c / 4 + i;
                                auto sum = [&](int e) { return fmaf(__uint_as_float(q[4 * i + e]), f, sums[c + 4 * i + e] * keep); };
                                float4 v = make_float4(sum(0), sum(1), sum(2), sum(3));
                                if (kCopies > 1 && whole && !aside) {
#pragma unroll
                                    for (int k = 1; k < kCopies; ++k) {
                                        const float4 w = __ldcg(to_lane + (size_t)at4 * kRows + k * R);
                                        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
                                    }
                                }
                                if (f == 0.f) v = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (mine) __stcg(whole && !aside ? to_row + at4 : to_lane + (size_t)at4 * kRows + copy * R, v);
                            }
                        }
                    }
                    if (kCopies > 1 && whole) {      // the other copies' parts are there; later, they may be written anew
                        __threadfence();
                        ok = exchange(0.f, told_sums);
                        if (!ok) return;
                    }
                }
                tc_before();
            }
            if (tables) {
                ++tabs;
                if (lane == 0) mbar_arrive(bar(kTabEmpty));
            }
        };
        while (ok && next(ok)) segment();
        if (!ok) give_up();
    } else {
        fewer_registers();
        // ---- value tiles: packed groups -> swizzled rows -------------------------------------------------------
        // A warp takes 32 tokens (two pages) of every tile.  LPT neighbouring lanes copy 16-byte chunks of one token (a whole group of
        // 32 or 64 bytes; two groups of 16), so a token's mask stays with its lanes and the place of a kept group is a
        // running count.  A kept group is one asynchronous 16-byte copy per chunk, a dropped one a copy that writes zeros and
        // reads nothing.  The copies of a warp's next tile are under way before the last one's are waited for, unless its slot is
        // still being read.  Page ids are asked for two tiles ahead, masks and offsets one.
        const int tok0 = (warp - 12) * 32, half = (warp - 12) >> 1;
        int vc = 0, pending = -1;                    // tiles so far; slot whose copies are not waited for yet
        bool ok = true;
        auto publish = [&]() {                       // this warp's copies into `pending` have landed
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kVFull + pending));
            pending = -1;
        };
        const int opg = kOctets / a.S;               // 16-byte chunks of a group
        const uint32_t all_groups = (1u << a.S) - 1u, limit = (uint32_t)min(a.cap_groups, (int64_t)0xFFFFFFFF);   // (of the store)
        while (ok && next(ok)) {
            const size_t problem = (size_t)s.b * a.Hkv + s.hk;
            const uint16_t* mask_row = a.v_mask + problem * a.T;
            const uint32_t* offs = a.v_offs + problem * (a.T + 1);
            const uint4* packed = a.v_packed + problem * a.cap_groups * opg;
            const uint4* fresh = a.v_new + problem * a.n_cap * kOctets;
            // tokens that no row of the sequence sees are left out: they may hold anything.  All that are seen lie in [lo_all, hi_all);
            // with given positions farther apart than the window there may be others between them, and each token is looked up
            // (16x32/8 heads, 256 listed pages, window 64: 16 nodes 71 -> 77 us, 4x32/8 with 128 nodes 90 -> 138)
            int lo_all = 0, hi_all = s.len, q_doc = 0;
            bool gaps = false;
            if constexpr (MASK) {
                if (a.sc.q_pos) {
                    int least = 0x7FFFFFFF, most = -1;
#pragma unroll 1
                    for (int i = lane; i < s.nodes; i += 32) {
                        const int p = a.sc.q_pos[(size_t)s.b * a.n_cap + i];
                        least = min(least, p);
                        most = max(most, p);
                    }
                    least = __reduce_min_sync(0xFFFFFFFFu, least);
                    most = __reduce_max_sync(0xFFFFFFFFu, most);
                    if (a.sc.window > 0 && least >= a.sc.window) lo_all = least - a.sc.window + 1;
                    if (most < s.len) hi_all = most + 1;
                    gaps = (long long)most - least > a.sc.window;
                } else if (a.sc.window > 0 && s.len >= a.sc.window) {
                    lo_all = s.len - a.sc.window + 1;
                }
                if (a.sc.tok_doc) q_doc = a.sc.q_doc[s.b];
            }
            auto seen_by_a_node = [&](int at) {
                const int32_t* const pos = a.sc.q_pos + (size_t)s.b * a.n_cap;
                bool seen = false;
#pragma unroll 4
                for (int i = 0; i < s.nodes; ++i) {
                    const int p = __ldg(pos + i);
                    seen |= at <= p && (uint32_t)p - (uint32_t)at < a.window;
                }
                return seen;
            };
            // of this lane's token: its mask, its page's first group, its document; -1 or the token
            auto ask_page = [&](int t) { return t >= s.tile0 ? listed(t * kTilePages + (tok0 + lane) / kPage) : -1; };
            auto ask_mask = [&](int id, uint32_t& m, uint32_t& first, int& doc) {
                m = first = 0;
                doc = -1;
                if (!is_page(id)) return -1;
                const int at = id * kPage + (lane & 15);
                first = offs[id * kPage];
                if (at >= s.len) return -1;
                m = mask_row[at];
                if (MASK && a.sc.tok_doc) doc = __ldg(a.sc.tok_doc + (size_t)s.b * a.T + at);
                return at;
            };
            uint32_t m_next, first_next;
            int doc_next, at_next = ask_mask(ask_page(s.tile1 - 1), m_next, first_next, doc_next);
            int id_next = ask_page(s.tile1 - 2);
#pragma unroll 1
            for (int t = s.tile1 - 1; t >= s.tile0; --t, ++vc) {
                const uint32_t every = m_next & all_groups, first = first_next;
                uint32_t m = every;
                if (MASK && (at_next < lo_all || at_next >= hi_all || (doc_next >= 0 && doc_next != q_doc))) m = 0;
                if (APART && gaps && !seen_by_a_node(at_next)) m = 0;
                at_next = ask_mask(id_next, m_next, first_next, doc_next);
                id_next = ask_page(t - 2);
                const int v = 2 * vc + half, slot = v % kVSlots;
                if (v >= kVSlots &&
                    !__all_sync(0xFFFFFFFFu, mbar_try_wait(bar(kVEmpty + slot), (uint32_t)(v / kVSlots - 1) & 1u))) {
                    if (pending >= 0) { cp_async_wait<0>(); publish(); }
                    ok = warp_wait(kVEmpty + slot, (uint32_t)(v / kVSlots - 1));
                    if (!ok) break;
                }
                const uint32_t rows = base + kOffV + slot * kSlot + (uint32_t)(tok0 & 63) * 128u;     // of the warp's tokens
                if (is_tree(t)) {                    // the tree's own values, full width
#pragma unroll 4
                    for (int i = lane; i < 32 * kOctets; i += 32) {
                        const int tok = i >> 4;
                        const uint32_t oct = (uint32_t)i & 15u;
                        const bool there = tok0 + tok < s.nodes;
                        cp_async16_if(rows + (oct >> 3) * (kSlot / 2) + (uint32_t)tok * 128u + (((oct & 7u) ^ ((uint32_t)tok & 7u)) << 4),
                                      there ? fresh + (size_t)(tok0 + tok) * kOctets + oct : fresh, there);
                    }
                } else {
                    // place of the token's first group: its page's, and the groups of the page's tokens before it
                    const uint32_t cnt = __popc(every), incl = warp_incl_scan(cnt, lane), page0 = __shfl_sync(0xFFFFFFFFu, incl, 15);
                    const uint32_t place = first + incl - cnt - (lane >= 16 ? page0 : 0u);
                    // groups behind the end of the store are not followed
                    const uint32_t held = place < limit ? limit - place : 0u;
                    while (__popc(m) > held) m &= ~(0x80000000u >> __clz(m));
                    auto copy = [&](auto groups) {
                        constexpr int S = decltype(groups)::value, OPG = kOctets / S, LPT = OPG < 2 ? 2 : OPG, GPL = LPT / OPG;
                        const int sub = lane % LPT;
#pragma unroll 1
                        for (int pass = 0; pass < LPT; ++pass) {
                            const int tok = pass * (32 / LPT) + lane / LPT;       // of the 32
                            uint32_t left = __shfl_sync(0xFFFFFFFFu, m, tok);     // groups from this lane's next one on
                            const uint32_t at = __shfl_sync(0xFFFFFFFFu, place, tok);
                            const uint4* src = packed + (size_t)at * OPG + sub % OPG;
                            if constexpr (GPL > 1) {
                                src += sub ? left & 1u : 0u;
                                left >>= sub;
                            }
                            // chunk oct of the row: half oct >> 3, place (oct & 7) ^ (tok & 7); oct = k LPT + sub
                            const uint32_t row = rows + (uint32_t)tok * 128u + (((uint32_t)(tok & 7) ^ (uint32_t)sub) << 4);
#pragma unroll
                            for (int k = 0; k < 16 / LPT; ++k) {
                                cp_async16_if(((row ^ (uint32_t)(((k * LPT) & 7) << 4))) + ((k * LPT) >> 3) * (kSlot / 2), src, left & 1u);
                                src += (GPL > 1 ? __popc(left & 3u) : (int)(left & 1u)) * OPG;
                                left >>= GPL;
                            }
                        }
                    };
                    if (a.S == 8) copy(std::integral_constant<int, 8>{});
                    else if (a.S == 16) copy(std::integral_constant<int, 16>{});
                    else copy(std::integral_constant<int, 4>{});
                }
                cp_async_commit();
                if (pending >= 0) { cp_async_wait<1>(); publish(); }
                pending = slot;
            }
            cp_async_wait<0>();                      // (the next segment may only come when this one is done)
            if (ok && pending >= 0) publish();
        }
        cp_async_wait<0>();
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

// Joins the partials of units that more than one CTA worked on, in CTA order: blockIdx.x = the CTA that begins the unit, blockIdx.y =
// 8 rows of it; behind them blocks that check the trees and gather the CTAs' status.  Few dependent loads on purpose: nothing
// hides this kernel's latency (with the units looked up by problem it took 24 us at 16x32/8 heads and 64 nodes).
__global__ void __launch_bounds__(256, 4)
tree_join_kernel(const TreeArgs a, int grid) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x >= grid) {
        if (blockIdx.y > 0) return;
        const int b = ((int)blockIdx.x - grid) * 8 + warp;
        if (b < a.B) {
            const int nodes = nodes_of(a, b);
            bool bad = false;
#pragma unroll 1
            for (int i = lane; i < nodes && a.parent; i += 32) {
                const int up = a.parent[(size_t)b * a.n_cap + i];
                bad |= up < -1 || up >= i;
            }
            bad = __any_sync(0xFFFFFFFFu, bad);
            if (lane == 0) a.status[b] = bad ? STC_ERR_INVALID_ARG : STC_OK;
        }
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (b == 0) {
            int st = 0;
#pragma unroll 1
            for (int c = lane; c < grid; c += 32) st = max(st, __ldcg(a.cta_status + c));
            st = __reduce_max_sync(0xFFFFFFFFu, st);
            if (lane == 0) *a.word = st;
        }
        return;
    }
    // warp = 8 rows and 4 chunks of 4 channels: the partials are read in 128 bytes, the rows written in 64
    const int in_block = (int)blockIdx.y * 8 + (lane & 7), chunk = warp * 4 + (lane >> 3);
    const int node_in = (int)(((uint32_t)in_block * a.gq_inv) >> 16), h = in_block - node_in * a.Gq;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 split = __ldcg(a.split + blockIdx.x);
    const int node = split.y * a.block_nodes + node_in, c0 = (int)blockIdx.x, c1 = split.z;
    if (split.x < 0 || node_in >= a.block_nodes || node >= split.w) return;
    const int b = (int)((uint32_t)split.x / (uint32_t)a.Hkv), hk = split.x - b * a.Hkv;
    const size_t row = ((size_t)b * a.n_cap + node) * a.Hq + hk * a.Gq + h;
    constexpr int kAtOnce = 4;                       // loads in flight
    const int copies_log2 = __ffs(kRows / a.rows) - 1, parts = (c1 - c0 + 1) << copies_log2;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int first = 0; first < parts; first += kAtOnce) {
        float2 p[kAtOnce];
        float4 v[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int e = c0 + ((first + i) >> copies_log2), copy = (first + i) & ((1 << copies_log2) - 1);
            const size_t at = (size_t)(2 * e + (e == c0 ? 1 : 0));
            p[i] = make_float2(-INFINITY, 0.f);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (first + i >= parts) continue;
            p[i] = __ldcg(a.part_ml + at * kRows + in_block);
            if (copy) p[i].y = 0.f;                  // the row's sum is told once
            v[i] = __ldcg(a.part_o + (at * 32 + chunk) * kRows + copy * a.rows + in_block);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, p[i].x);
        const float fm = m == -INFINITY ? 0.f : ex2(m - top);
        l *= fm; o.x *= fm; o.y *= fm; o.z *= fm; o.w *= fm;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (p[i].x == -INFINITY) {               // nothing seen: its sum is 0, or NaN
                l += p[i].y;
                continue;
            }
            const float f = ex2(p[i].x - top);
            l = fmaf(p[i].y, f, l);
            o.x = fmaf(v[i].x, f, o.x); o.y = fmaf(v[i].y, f, o.y); o.z = fmaf(v[i].z, f, o.z); o.w = fmaf(v[i].w, f, o.w);
        }
        m = top;
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    if (inv != 0.f) r = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    reinterpret_cast<float4*>(a.out)[row * 32 + chunk] = r;
    if (a.lse && chunk == 0) a.lse[row] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// The workspace has to be sized without a device, so the partial slots are counted for this many CTAs.
constexpr int kPlanSms = 148;

template <int R, bool MASK, bool SCORE, bool APART>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& fresh, const TreeArgs& a, int n_cta, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(tree_attn_kernel<R, MASK, SCORE, APART>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    cudaFuncAttributes f;                            // (a launch with fewer registers would wait for them without end)
    e = cudaFuncGetAttributes(&f, tree_attn_kernel<R, MASK, SCORE, APART>);
    if (e != cudaSuccess) return e;
    if (f.numRegs * kThreads < 256 * kSoftmaxRegs + 256 * kOtherRegs) return cudaErrorInvalidConfiguration;
    tree_attn_kernel<R, MASK, SCORE, APART><<<n_cta, kThreads, kSmem, st>>>(q, k, fresh, a);
    return cudaGetLastError();
}

template <int R>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& fresh, const TreeArgs& a, int n_cta, bool masked, bool scored,
                   cudaStream_t st) {
    if (a.sc.q_pos && a.sc.window > 0)
        return scored ? launch<R, true, true, true>(q, k, fresh, a, n_cta, st) : launch<R, true, false, true>(q, k, fresh, a, n_cta, st);
    return scored ? launch<R, true, true, false>(q, k, fresh, a, n_cta, st)
           : masked ? launch<R, true, false, false>(q, k, fresh, a, n_cta, st) : launch<R, false, false, false>(q, k, fresh, a, n_cta, st);
}

}  // namespace

size_t tree_attn_ws_bytes() {
    return 256 + align256(kPlanSms * 4) + align256(kPlanSms * 16) + 2 * (size_t)kPlanSms * kRows * 8 +
           3 * (size_t)kPlanSms * kRows * kHeadDim * 4;
}

cudaError_t launch_tree_attn(const Geom& g, const stc_cache& cache, const stc_tree& tree, const void* q, const int32_t* page_ids,
                             const int32_t* n_pages, int max_pages, float sm_scale, const ScoreArgs& score, float* out, float* lse,
                             int32_t* status, void* ws, cudaStream_t st) {
    const bool scored = score.softcap > 0.f || score.slopes || !(sm_scale > 0.f);
    const bool masked = scored || score.window > 0 || score.q_pos || score.tok_doc;
    TreeArgs a;
    a.seq_len = g.seq_len; a.n_nodes = tree.n_nodes; a.parent = tree.parent; a.page_ids = page_ids; a.n_pages = n_pages;
    a.v_mask = cache.v_mask; a.v_offs = cache.v_offs; a.v_packed = static_cast<const uint4*>(cache.v_packed);
    a.v_new = static_cast<const uint4*>(tree.v);
    a.out = out; a.lse = lse; a.status = status;
    char* w = static_cast<char*>(ws);
    a.word = reinterpret_cast<int32_t*>(w);
    w += 256;
    a.cta_status = reinterpret_cast<int32_t*>(w);
    w += align256(kPlanSms * 4);
    a.split = reinterpret_cast<int4*>(w);
    w += align256(kPlanSms * 16);
    a.part_ml = reinterpret_cast<float2*>(w);
    w += 2 * (size_t)kPlanSms * kRows * 8;
    a.part_o = reinterpret_cast<float4*>(w);
    a.cap_groups = cache.cap_groups;
    a.B = g.B; a.Hq = g.Hq; a.Hkv = g.Hkv; a.Gq = g.Gq; a.S = g.S; a.T = g.T; a.n_cap = tree.n_cap;
    a.max_pages = max_pages; a.problems = g.problems;
    // The fewest rows that hold a whole tree, copied over the other lanes: the time of a tile goes with the tokens that a thread weighs.  The
    // copies of a row have to be added up at the end, by the second kernel copies * CTAs per unit parts of a row, so they pay from some
    // tiles per CTA on that grow with the parts.  Measured with 1 to 16 sequences of 4 or 8 KV heads, 2 to 48 tiles per CTA; with 5, 9, 18,
    // 37 and 74 parts they pay from 7, 6, 11, 16, 30 tiles on without options, 6, 4, 9, 12, 21 with masks, 3, 2, 3, 6, 10 with a cap, 5, 3,
    // 7, 8, 15 with slopes.  1x32/8 heads, 16 nodes (37 parts), no options: 6 tiles per CTA 31 us without copies and 35 with them, 28 tiles
    // 68 and 62; 8x28/4, 5 nodes, cap (9 parts): 2 tiles 27 and 27, 24 tiles 91 and 66.
    int sms = 0;
    cudaError_t e = device_sm_count(&sms);
    if (e != cudaSuccess) return e;
    const int n_cta = sms < kPlanSms ? sms : kPlanSms;
    const int64_t most_tiles = (int64_t)g.problems * ((page_ids ? max_pages : g.P) / kTilePages + 1);
    a.rows = 32;
    while (a.rows < kRows && a.rows / g.Gq < tree.n_cap) a.rows *= 2;
    const double parts = (double)(kRows / a.rows) * n_cta / g.problems;
    if ((double)most_tiles <= n_cta * (scored ? 1.5 + parts / 7 : masked ? 3.5 + parts / 4 : 4 + parts / 3)) a.rows = kRows;
    a.block_nodes = a.rows / g.Gq;
    a.gq_inv = (65536u + (uint32_t)g.Gq - 1u) / (uint32_t)g.Gq;
    a.sc = score;
    a.scale_log2 = sm_scale * kLog2e;
    a.cap_in = score.softcap > 0.f ? sm_scale / score.softcap : 0.f;
    a.cap_log2 = score.softcap * kLog2e;
    a.window = score.window > 0 ? (uint32_t)score.window : 0xFFFFFFFFu;

    EncodeTiled enc = tensor_map_encoder();
    if (!enc) return cudaErrorNotSupported;
    CUtensorMap map_q, map_k, map_new;
    {
        const cuuint64_t dims[3] = {kHeadDim, (cuuint64_t)g.Hq, (cuuint64_t)g.B * (cuuint64_t)tree.n_cap};
        const cuuint64_t strides[2] = {kRowBytes, (cuuint64_t)g.Hq * kRowBytes};
        const cuuint32_t box[3] = {64, (cuuint32_t)g.Gq, (cuuint32_t)a.block_nodes}, step[3] = {1, 1, 1};
        if (enc(&map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    auto rows_map = [&](CUtensorMap* map, const void* p, long long rows, int at_once) {
        const cuuint64_t dims[2] = {kHeadDim, (cuuint64_t)rows};
        const cuuint64_t strides[1] = {kRowBytes};
        const cuuint32_t box[2] = {64, (cuuint32_t)at_once}, step[2] = {1, 1};
        return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    const long long new_rows = (long long)g.problems * tree.n_cap;
    // (a cache without tokens: no page is ever loaded, the map only has to be a valid one)
    const int at_once = page_ids ? kPage : kTok;     // rows of a copy of K
    if (!rows_map(&map_new, tree.k, new_rows, tree.n_cap) ||
        !(g.T > 0 ? rows_map(&map_k, cache.k, (long long)g.problems * g.T, at_once) : rows_map(&map_k, tree.k, new_rows, at_once)))
        return cudaErrorInvalidValue;
    e = a.rows == 32 ? launch<32>(map_q, map_k, map_new, a, n_cta, masked, scored, st)
        : a.rows == 64 ? launch<64>(map_q, map_k, map_new, a, n_cta, masked, scored, st)
                       : launch<128>(map_q, map_k, map_new, a, n_cta, masked, scored, st);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n_cta + (g.B + 7) / 8), (unsigned)(a.rows / 8));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute early;                       // its blocks wait in place instead of behind a launch
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, tree_join_kernel, a, n_cta);
}

}  // namespace stc
