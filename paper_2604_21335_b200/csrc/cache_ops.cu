// Copying whole cached sequences and closing the gaps that dropped pages leave.  No arithmetic but prefix sums: both calls move
// bytes (one read of each source, one write of each destination): 16 copies of two prompts of 16384 tokens 180 us, 4.6 TB/s; 16x8 lists
// of 256 pages into another cache 91 us, 4.9 TB/s, in place 138 us, where a plain copy reaches 6.6.  The copies write 4.1 TB/s, which is
// not the most that the chip writes: a kernel that only stores, in the same order, reaches 6.0 to 6.8.  (A list of destinations in shared
// memory in place of two dependent reads per copy: 188 us.)
#include <cooperative_groups.h>

#include "common.cuh"

namespace stc {
namespace {

namespace cg = cooperative_groups;

// A cache as the kernels see it.
struct View {
    uint4* k;
    uint4* kmin;                 // or nullptr
    uint4* kmax;
    uint4* v_packed;
    uint16_t* v_mask;
    uint32_t* v_offs;
    int64_t cap_groups;
    int T, P;
};

__device__ __forceinline__ uint4 ld16(const uint4* p) {      // coherent: the cache may be read and written by one call
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// ---- fork ---------------------------------------------------------------------------------------------------------

constexpr int kCheckThreads = 1024;

// Which pairs are copied: a pair's dst_row is its own and, within one cache, no pair's src_row.  One block; the lists pass
// through shared memory, each thread compares its pair with all of them.
__global__ void __launch_bounds__(kCheckThreads)
fork_check_kernel(int n_pairs, const int32_t* __restrict__ src_row, const int32_t* __restrict__ dst_row,
                  const int32_t* __restrict__ seq_len, int src_B, int dst_B, int Hkv, int S, bool same, View src, View dst,
                  int32_t* __restrict__ new_len, int64_t* __restrict__ total_groups, int32_t* __restrict__ status) {
    __shared__ int sh_src[kCheckThreads], sh_dst[kCheckThreads];
    for (int i0 = 0; i0 < n_pairs; i0 += kCheckThreads) {
        const int i = i0 + threadIdx.x;
        int s = -1, d = -1, len = 0;
        bool bad = true;
        if (i < n_pairs) {
            s = src_row[i];
            d = dst_row[i];
            bad = s < 0 || s >= src_B || d < 0 || d >= dst_B;
            if (!bad) {
                len = clamp_len(seq_len, s, src.T);
                bad = len > dst.T;
            }
        }
        for (int j0 = 0; j0 < n_pairs; j0 += kCheckThreads) {
            __syncthreads();
            if (j0 + (int)threadIdx.x < n_pairs) {
                sh_src[threadIdx.x] = src_row[j0 + threadIdx.x];
                sh_dst[threadIdx.x] = dst_row[j0 + threadIdx.x];
            }
            __syncthreads();
            const int m = min(kCheckThreads, n_pairs - j0);
            for (int j = 0; j < m; ++j) {
                if (sh_dst[j] == d && j0 + j < i) bad = true;
                if (same && s != d && sh_src[j] == d) bad = true;
            }
        }
        if (i < n_pairs) {
            if (!bad) new_len[d] = len;
            for (int h = 0; h < Hkv; ++h) {
                const int64_t total = bad ? 0 : (int64_t)src.v_offs[((size_t)s * Hkv + h) * (src.T + 1) + len];
                if (!bad) total_groups[(size_t)d * Hkv + h] = total;
                status[(size_t)i * Hkv + h] = bad ? STC_ERR_INVALID_ARG
                                              : total > min(dst.cap_groups, src.cap_groups) ? STC_ERR_CAPACITY : STC_OK;
            }
        }
    }
}

constexpr int kForkThreads = 256, kForkTok = 64, kForkRun = 16;

// One CTA moves pieces of 64 tokens of (source, KV head): read once into registers, written to the row of every pair of a run of
// pairs with that source.  The CTAs of the run's other pairs leave.  A run ends at every 16th pair of the list: the CTAs of a call are
// divided by its pairs, and a thousand copies of one prompt would be left with a handful of them (1024 x 2048 tokens of one head: 3.3 ms,
// now 0.30, with as many sources 0.33).  Read again for every 16 copies, a source adds at most a sixteenth of what is written.
template <int S>
__global__ void __launch_bounds__(kForkThreads)
fork_copy_kernel(int n_pairs, const int32_t* __restrict__ src_row, const int32_t* __restrict__ dst_row,
                 const int32_t* __restrict__ seq_len, int Hkv, bool same, View src, View dst, const int32_t* __restrict__ status) {
    constexpr int OPG = kOctets / S, kRegs = kForkTok * kOctets / kForkThreads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int first = blockIdx.z, h = blockIdx.y, s = src_row[first], tid = threadIdx.x;
    if (first % kForkRun != 0 && src_row[first - 1] == s) return;
    // the run may begin with pairs that are left out
    bool any = false;
    int end = first;
    const int most = min(n_pairs, (first / kForkRun + 1) * kForkRun);
    for (; end < most && src_row[end] == s; ++end)
        any |= status[(size_t)end * Hkv + h] != STC_ERR_INVALID_ARG && !(same && dst_row[end] == s);
    if (!any) return;
    const size_t from = (size_t)s * Hkv + h;
    const int len = clamp_len(seq_len, s, src.T);
    const uint32_t* offs = src.v_offs + from * (src.T + 1);
    const uint4* ks = src.k + from * src.T * kOctets;
    const uint4* vs = src.v_packed + from * src.cap_groups * OPG;
    // (a sequence of no tokens still has its first offset)
    for (int piece = blockIdx.x; piece == 0 || piece * kForkTok < len; piece += gridDim.x) {
        const int t0 = piece * kForkTok, n = min(kForkTok, len - t0), pages = (n + kPage - 1) / kPage;
        const int64_t g0 = offs[t0], g1 = min((int64_t)offs[t0 + n], src.cap_groups);
        const int chunks = (int)max((int64_t)0, min(g1 - g0, (int64_t)kForkTok * S)) * OPG;
        uint4 key[kRegs], val[kRegs], lo, hi;
        uint32_t word = 0, off = 0;
#pragma unroll
        for (int i = 0; i < kRegs; ++i) {
            const int c = tid + i * kForkThreads;
            if (c < n * kOctets) key[i] = ld16(ks + (size_t)t0 * kOctets + c);
        }
#pragma unroll
        for (int i = 0; i < kRegs; ++i) {
            const int c = tid + i * kForkThreads;
            if (c < chunks) val[i] = ld16(vs + g0 * OPG + c);
        }
        const size_t meta = (size_t)(t0 / kPage) * kOctets + tid;
        const bool has_meta = dst.kmin && tid < pages * kOctets;
        if (has_meta) {
            lo = ld16(src.kmin + from * src.P * kOctets + meta);
            hi = ld16(src.kmax + from * src.P * kOctets + meta);
        }
        if (tid < n) word = src.v_mask[from * src.T + t0 + tid];
        if (tid <= n) off = offs[t0 + tid];
        for (int i = first; i < end; ++i) {
            const int d = dst_row[i];
            if (status[(size_t)i * Hkv + h] == STC_ERR_INVALID_ARG || (same && d == s)) continue;
            const size_t to = (size_t)d * Hkv + h;
            uint4* kd = dst.k + (to * dst.T + t0) * kOctets;
            uint4* vd = dst.v_packed + (to * dst.cap_groups + g0) * OPG;
            const int64_t room = (dst.cap_groups - g0) * OPG;
#pragma unroll
            for (int e = 0; e < kRegs; ++e) {
                const int c = tid + e * kForkThreads;
                if (c < n * kOctets) kd[c] = key[e];
                if (c < chunks && c < room) vd[c] = val[e];
            }
            if (has_meta) {
                dst.kmin[to * dst.P * kOctets + meta] = lo;
                dst.kmax[to * dst.P * kOctets + meta] = hi;
            }
            if (tid < n) dst.v_mask[to * dst.T + t0 + tid] = (uint16_t)word;
            if (tid <= n) dst.v_offs[to * (dst.T + 1) + t0 + tid] = off;
        }
        if (len == 0) break;
    }
}

// ---- compaction ---------------------------------------------------------------------------------------------------

constexpr int kCompactThreads = 256, kCompactCtas = 8, kCompactPages = 4;    // pages a CTA moves per round

// For a cluster per (sequence, KV head): tokens that are kept, or -1, with its status, if a list of the sequence is not as it has to be.
// Every CTA checks a share of all lists of the sequence: every head drops the same number of tokens or nothing is moved.
__device__ __forceinline__ int kept_tokens(int problem, int len, int n, int Hkv, const int32_t* __restrict__ page_ids,
                                           const int32_t* __restrict__ n_pages, int max_pages, int dst_T,
                                           int32_t* __restrict__ new_len, int32_t* __restrict__ status) {
    __shared__ int sh_bad[kCompactCtas];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x, b = problem / Hkv;
    const int pages = (len + kPage - 1) / kPage, rest = pages * kPage - len;
    bool bad = n < 0 || n > max_pages || n > pages;
    bool ends = false;                                                       // the last page is listed
    if (!bad && n > 0) ends = page_ids[(size_t)b * Hkv * max_pages + n - 1] == pages - 1;
    const int kept = bad ? 0 : n * kPage - (ends ? rest : 0);
    bad = bad || kept > dst_T;
    for (int h = tid; h < Hkv && !bad; h += kCompactThreads) bad = n_pages[(size_t)b * Hkv + h] != n;
    bad = __syncthreads_or(bad);
    if (!bad) {
        // entry i of all lists at once: i = e mod n of list e / n
        for (int64_t e = rank * kCompactThreads + tid; e < (int64_t)n * Hkv; e += kCompactCtas * kCompactThreads) {
            const int h = (int)(e / n), i = (int)(e - (int64_t)h * n);
            const int32_t* list = page_ids + ((size_t)b * Hkv + h) * max_pages;
            const int p = list[i];
            bad |= p < 0 || p >= pages || (i > 0 && list[i - 1] >= p);
            if (i == n - 1 && rest > 0) bad |= (p == pages - 1) != ends;
        }
    }
    bad = __syncthreads_or(bad);
    cluster.sync();
    if (tid < kCompactCtas) *cluster.map_shared_rank(&sh_bad[rank], tid) = bad;
    cluster.sync();
#pragma unroll
    for (int i = 0; i < kCompactCtas; ++i) bad |= sh_bad[i] != 0;
    if (rank == 0 && tid == 0) {
        if (problem == b * Hkv) new_len[b] = bad ? len : kept;
        if (bad) status[problem] = STC_ERR_INVALID_ARG;
    }
    return bad ? -1 : kept;
}

// Between two caches the pages are independent once their new offsets are known: a CTA takes a share of the list, the CTAs meet
// once to tell each other the groups of their shares, and every warp moves pages by itself.
template <int S>
__global__ void __launch_bounds__(kCompactThreads, 3)
compact_apart_kernel(const int32_t* __restrict__ seq_len, int Hkv, const int32_t* __restrict__ page_ids,
                     const int32_t* __restrict__ n_pages, int max_pages, View src, View dst, int32_t* __restrict__ new_len,
                     int64_t* __restrict__ total_groups, int32_t* __restrict__ status) {
    constexpr int OPG = kOctets / S, kWarps = kCompactThreads / 32, kPer = kPage * kOctets / 64;        // (half a page at a time)
    __shared__ uint32_t sh_count[kCompactCtas], sh_sum[kWarps], sh_first[kCompactThreads], sh_to[kCompactThreads], sh_size[kCompactThreads];
    __shared__ int sh_page[kCompactThreads];
    cg::cluster_group cluster = cg::this_cluster();
    const int problem = blockIdx.x / kCompactCtas, rank = (int)cluster.block_rank(), b = problem / Hkv, tid = threadIdx.x;
    const int len = clamp_len(seq_len, b, src.T), n = n_pages[(size_t)b * Hkv], warp = tid >> 5, lane = tid & 31;
    const int kept = kept_tokens(problem, len, n, Hkv, page_ids, n_pages, max_pages, dst.T, new_len, status);
    if (kept < 0) return;                                                    // (the whole cluster)
    const int32_t* list = page_ids + (size_t)problem * max_pages;
    const uint32_t* offs = src.v_offs + (size_t)problem * (src.T + 1);
    const int share = (n + kCompactCtas - 1) / kCompactCtas, first = min(rank * share, n), last = min(first + share, n);
    // of entry i: its page, where its groups are, how many
    auto entry = [&](int i, int& page, uint32_t& o0) -> uint32_t {
        page = -1;
        o0 = 0;
        if (i >= last) return 0;
        page = list[i];
        const int t0 = page * kPage, tokens = min(kPage, len - t0);
        o0 = offs[t0];
        return min(offs[t0 + tokens] - o0, (uint32_t)(tokens * S));
    };
    // sum over the block of what each thread has, and the sum before it
    auto scan = [&](uint32_t x, uint32_t& total) -> uint32_t {
        const uint32_t incl = warp_incl_scan(x, lane);
        __syncthreads();
        if (lane == 31) sh_sum[warp] = incl;
        __syncthreads();
        uint32_t before = 0;
        total = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            if (i < warp) before += sh_sum[i];
            total += sh_sum[i];
        }
        return before + incl - x;
    };
    int page;
    uint32_t o0, sum = 0, mine;
    const bool once = share <= kCompactThreads;
    uint32_t size = entry(first + tid, page, o0), before = scan(size, mine);
    if (!once) {
        sum = size;
        for (int i = first + kCompactThreads + tid; i < last; i += kCompactThreads) {
            int p;
            uint32_t o;
            sum += entry(i, p, o);
        }
        scan(sum, mine);
    }
    if (tid < kCompactCtas) *cluster.map_shared_rank(&sh_count[rank], tid) = mine;
    cluster.sync();                                                          // (the last write to another CTA is through)
    uint32_t base = 0, all = 0;                                              // (offsets are 32-bit numbers in the cache itself)
#pragma unroll
    for (int c = 0; c < kCompactCtas; ++c) {
        if (c < rank) base += sh_count[c];
        all += sh_count[c];
    }
    const uint4* ks = src.k + (size_t)problem * src.T * kOctets;
    const uint4* vs = src.v_packed + (size_t)problem * src.cap_groups * OPG;
    uint4* kd = dst.k + (size_t)problem * dst.T * kOctets;
    uint4* vd = dst.v_packed + (size_t)problem * dst.cap_groups * OPG;
    for (int i0 = first; i0 < last; i0 += kCompactThreads) {
        if (i0 > first) size = entry(i0 + tid, page, o0);
        uint32_t total;
        if (i0 > first || !once) before = scan(size, total);
        else total = mine;
        __syncthreads();
        sh_page[tid] = page; sh_first[tid] = o0; sh_size[tid] = size; sh_to[tid] = base + before;
        __syncthreads();
        base += total;
        const int m = min(kCompactThreads, last - i0);
#pragma unroll 1
        for (int j = warp; j < m; j += kWarps) {
            const int i = i0 + j, t0 = sh_page[j] * kPage, tokens = min(kPage, len - t0);
            const uint32_t from = sh_first[j], to = sh_to[j];
            const int64_t room = src.cap_groups - (int64_t)from;             // (offsets that do not fit the store are not followed)
            const int chunks = (int)min((int64_t)sh_size[j], max(room, (int64_t)0)) * OPG;
            const int64_t fits = (dst.cap_groups - (int64_t)to) * OPG;
            uint4 meta = {};
            uint32_t word = 0, off = 0;
            if (dst.kmin) meta = ldg_nc16((lane < kOctets ? src.kmin : src.kmax) + ((size_t)problem * src.P + t0 / kPage) * kOctets + (lane & 15));
            if (lane < tokens) {
                word = src.v_mask[(size_t)problem * src.T + t0 + lane];
                off = offs[t0 + lane] - from;
            }
#pragma unroll 1
            for (int at = lane; at < kPage * kOctets; at += 32 * kPer) {
                uint4 key[kPer], val[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (at + e * 32 < tokens * kOctets) key[e] = ldg_nc16(ks + (size_t)t0 * kOctets + at + e * 32);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (at + e * 32 < chunks) val[e] = ldg_nc16(vs + (size_t)from * OPG + at + e * 32);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (at + e * 32 < tokens * kOctets) kd[(size_t)i * kPage * kOctets + at + e * 32] = key[e];
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (at + e * 32 < chunks && at + e * 32 < fits) vd[(size_t)to * OPG + at + e * 32] = val[e];
            }
            if (dst.kmin) ((lane < kOctets ? dst.kmin : dst.kmax) + ((size_t)problem * dst.P + i) * kOctets)[lane & 15] = meta;
            if (lane < tokens) {
                dst.v_mask[(size_t)problem * dst.T + i * kPage + lane] = (uint16_t)word;
                dst.v_offs[(size_t)problem * (dst.T + 1) + i * kPage + lane] = to + off;
            }
        }
    }
    if (rank == 0 && tid == 0) {                                             // (every token wrote where it begins; this is where the last ends)
        dst.v_offs[(size_t)problem * (dst.T + 1) + kept] = all;
        total_groups[problem] = all;
        status[problem] = (int64_t)all > dst.cap_groups ? STC_ERR_CAPACITY : STC_OK;
    }
}

// Within one cache the order matters.
// One cluster per (sequence, KV head) moves 32 listed pages per round.  A round is read into registers, the CTAs meet (which also
// tells each how many groups those before it hold), and the round is written.  In place that order is enough: the
// i-th listed page is at i or above, so what a round writes lies below everything that later rounds read, and everything that
// it overwrites of its own was read before the meeting.  The same holds for the packed groups, whose new offsets
// never exceed the old ones.
template <int S>
__global__ void __launch_bounds__(kCompactThreads)
compact_kernel(const int32_t* __restrict__ seq_len, int Hkv, const int32_t* __restrict__ page_ids,
               const int32_t* __restrict__ n_pages, int max_pages, View src, View dst, int32_t* __restrict__ new_len,
               int64_t* __restrict__ total_groups, int32_t* __restrict__ status) {
    constexpr int OPG = kOctets / S, kPer = kPage * kOctets / 64;            // 64 threads per page, 16-byte pieces of each
    __shared__ uint32_t sh_count[2][kCompactCtas];                           // groups of each CTA's pages, per round parity
    cg::cluster_group cluster = cg::this_cluster();
    const int problem = blockIdx.x / kCompactCtas, rank = (int)cluster.block_rank(), b = problem / Hkv, tid = threadIdx.x;
    const int len = clamp_len(seq_len, b, src.T), n = n_pages[(size_t)b * Hkv];
    const int kept = kept_tokens(problem, len, n, Hkv, page_ids, n_pages, max_pages, dst.T, new_len, status);
    if (kept < 0) return;                                                    // (the whole cluster: nobody writes to a CTA that left)
    const int32_t* list = page_ids + (size_t)problem * max_pages;
    const uint32_t* offs = src.v_offs + (size_t)problem * (src.T + 1);
    const uint16_t* mask = src.v_mask + (size_t)problem * src.T;
    const uint4* ks = src.k + (size_t)problem * src.T * kOctets;
    const uint4* vs = src.v_packed + (size_t)problem * src.cap_groups * OPG;
    uint4* kd = dst.k + (size_t)problem * dst.T * kOctets;
    uint4* vd = dst.v_packed + (size_t)problem * dst.cap_groups * OPG;
    const int in_page = tid & 63, slot = tid >> 6;                           // this thread's page of the CTA's four
    int64_t base = 0;                                                        // groups of the rounds before
    const int rounds = (n + kCompactCtas * kCompactPages - 1) / (kCompactCtas * kCompactPages);
    auto listed = [&](int round) {
        const int i = (round * kCompactCtas + rank) * kCompactPages + slot;
        return i < n ? list[i] : -1;
    };
    int page = listed(0);
    for (int round = 0; round < rounds; ++round) {
        const int i = (round * kCompactCtas + rank) * kCompactPages + slot;
        const int next = round + 1 < rounds ? listed(round + 1) : -1;
        const int t0 = page * kPage, tokens = page < 0 ? 0 : min(kPage, len - t0);
        uint32_t o0 = 0, size = 0;
        if (page >= 0) {
            o0 = offs[t0];
            size = min(offs[t0 + tokens] - o0, (uint32_t)(tokens * S));
        }
        uint4 key[kPer], val[kPer], meta = {};
        uint32_t word = 0, off = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int c = in_page + e * 64;
            if (c < tokens * kOctets) key[e] = ld16(ks + (size_t)t0 * kOctets + c);
        }
        const int64_t room = src.cap_groups - (int64_t)o0;                   // (offsets that do not fit the store are not followed)
        const int chunks = (int)min((int64_t)size, max(room, (int64_t)0)) * OPG;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int c = in_page + e * 64;
            if (c < chunks) val[e] = ld16(vs + (size_t)o0 * OPG + c);
        }
        const bool has_meta = dst.kmin && page >= 0 && in_page < 2 * kOctets;
        if (has_meta)
            meta = ld16((in_page < kOctets ? src.kmin : src.kmax) + ((size_t)problem * src.P + page) * kOctets + (in_page & 15));
        if (in_page < tokens) {
            word = *reinterpret_cast<const volatile uint16_t*>(mask + t0 + in_page);
            off = *reinterpret_cast<const volatile uint32_t*>(offs + t0 + in_page) - o0;
        }
        // groups of the four pages, told to the other CTAs
        uint32_t mine[kCompactPages], before = 0, all = 0;
        {
            __shared__ uint32_t sh_size[2][kCompactPages];
            if (in_page == 0) sh_size[round & 1][slot] = size;
            __syncthreads();
#pragma unroll
            for (int s = 0; s < kCompactPages; ++s) {
                mine[s] = sh_size[round & 1][s];
                if (s < slot) before += mine[s];
                all += mine[s];
            }
        }
        if (tid < kCompactCtas) *cluster.map_shared_rank(&sh_count[round & 1][rank], tid) = all;
        cluster.sync();
        uint32_t total = 0;
#pragma unroll
        for (int c = 0; c < kCompactCtas; ++c) {
            const uint32_t x = sh_count[round & 1][c];
            if (c < rank) before += x;
            total += x;
        }
        const int64_t to = base + before;
        base += total;
        if (page >= 0) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int c = in_page + e * 64;
                if (c < tokens * kOctets) kd[(size_t)i * kPage * kOctets + c] = key[e];
            }
            const int64_t fits = (dst.cap_groups - to) * OPG;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int c = in_page + e * 64;
                if (c < chunks && c < fits) vd[to * OPG + c] = val[e];
            }
            if (has_meta)
                ((in_page < kOctets ? dst.kmin : dst.kmax) + ((size_t)problem * dst.P + i) * kOctets)[in_page & 15] = meta;
            if (in_page < tokens) {
                dst.v_mask[(size_t)problem * dst.T + i * kPage + in_page] = (uint16_t)word;
                dst.v_offs[(size_t)problem * (dst.T + 1) + i * kPage + in_page] = (uint32_t)to + off;
            }
        }
        page = next;
    }
    if (rank == 0 && tid == 0) {                                             // (every token wrote where it begins; this is where the last ends)
        dst.v_offs[(size_t)problem * (dst.T + 1) + kept] = (uint32_t)base;
        total_groups[problem] = base;
        status[problem] = base > dst.cap_groups ? STC_ERR_CAPACITY : STC_OK;
    }
    cluster.sync();                                                          // nobody leaves while another may still write to it
}

View view(const Geom& g, const stc_cache& c) {
    View v;
    v.k = static_cast<uint4*>(const_cast<void*>(c.k));
    v.kmin = static_cast<uint4*>(c.kmin);
    v.kmax = static_cast<uint4*>(c.kmax);
    v.v_packed = static_cast<uint4*>(c.v_packed);
    v.v_mask = c.v_mask;
    v.v_offs = c.v_offs;
    v.cap_groups = c.cap_groups;
    v.T = g.T;
    v.P = g.P;
    return v;
}

}  // namespace

cudaError_t launch_cache_fork(const Geom& gs, const stc_cache& src, const Geom& gd, const stc_cache& dst, int n_pairs,
                              const int32_t* src_row, const int32_t* dst_row, int32_t* new_len, int64_t* total_groups,
                              int32_t* status, cudaStream_t st) {
    const View vs = view(gs, src), vd = view(gd, dst);
    const bool same = src.k == dst.k;
    fork_check_kernel<<<1, kCheckThreads, 0, st>>>(n_pairs, src_row, dst_row, gs.seq_len, gs.B, gd.B, gs.Hkv, gs.S, same, vs, vd,
                                                   new_len, total_groups, status);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    int sms = 0;
    e = device_sm_count(&sms);
    if (e != cudaSuccess) return e;
    // 32 CTAs per SM if every pair has its own source, two at least if runs of 16 share one
    const long long pieces = ((long long)gs.T + kForkTok - 1) / kForkTok, wide = (long long)gs.Hkv * n_pairs;
    long long gx = ((long long)sms * 32 + wide - 1) / wide;
    gx = gx < pieces ? gx : pieces;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(gx < 1 ? 1 : gx), (unsigned)gs.Hkv, (unsigned)n_pairs);
    cfg.blockDim = dim3(kForkThreads);
    cfg.stream = st;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
#define STC_FORK(S_) \
    case S_: return cudaLaunchKernelEx(&cfg, fork_copy_kernel<S_>, n_pairs, src_row, dst_row, gs.seq_len, gs.Hkv, same, vs, vd, \
                                       static_cast<const int32_t*>(status));
    switch (gs.S) {
        STC_FORK(4) STC_FORK(8) STC_FORK(16)
        default: return cudaErrorInvalidValue;
    }
#undef STC_FORK
}

cudaError_t launch_cache_compact(const Geom& gs, const stc_cache& src, const int32_t* page_ids, const int32_t* n_pages,
                                 int max_pages, const Geom& gd, const stc_cache& dst, int32_t* new_len, int64_t* total_groups,
                                 int32_t* status, cudaStream_t st) {
    const View vs = view(gs, src), vd = view(gd, dst);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)gs.problems * kCompactCtas);
    cfg.blockDim = dim3(kCompactThreads);
    cfg.stream = st;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = kCompactCtas;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
    // (between two caches a share of the list per CTA and one meeting; within one, in order, a meeting per 32 pages.  16x8 lists of 256
    // pages: 91 and 138 us)
#define STC_COMPACT(S_) \
    case S_: return cudaLaunchKernelEx(&cfg, src.k == dst.k ? compact_kernel<S_> : compact_apart_kernel<S_>, gs.seq_len, gs.Hkv, page_ids, \
                                       n_pages, max_pages, vs, vd, new_len, total_groups, status);
    switch (gs.S) {
        STC_COMPACT(4) STC_COMPACT(8) STC_COMPACT(16)
        default: return cudaErrorInvalidValue;
    }
#undef STC_COMPACT
}

}  // namespace stc
