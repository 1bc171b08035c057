// Rotary positions on the way into the cache: the new tokens' q, k, v leave the projection token by token
// ([B][n][H][128], any token stride); q is rotated into the layout the attention calls read, k is rotated
// and v copied into the rows of the cache behind each sequence.
//
//   pair i of a token at position p is turned by the angle p * inv_freq[i]:
//   (a, b) -> scale * (a cos - b sin, b cos + a sin)
//
// Angles.  p * inv_freq in fp32 is off by up to 0.004 rad at position 131072.  Here inv_freq / 2 pi is taken
// modulo one turn as a 64-bit fixed-point fraction (from the fp64 table), so that multiplying by the position
// in wrapping integer arithmetic IS the reduction modulo one turn: the angle is good to 2^-33 turns at any
// position below 2^20 (2^-53 of the table times the position), and sincospif gets an argument in [-1, 1).
//
// Work split.  Bandwidth-bound: 512 bytes moved per head row, 256 each way.  A thread owns two 16-byte chunks
// of a row (a "duo": with the half layout chunk d and its partner d + rot/16, else neighbours), so that both
// members of eight pairs meet in one thread; it computes its eight (cos, sin) once and keeps them in registers
// while it walks over the rows of its token, four in flight.  A CTA is 8 duos x 32 (token, row slot) lanes: four
// tokens with eight slots each, or one token with 32 slots where tokens are few, so that every row is in flight at once.
// Measured: 2 x 16384 tokens of 32 + 8 + 8 heads in 124 us = 6.5 TB/s, 1.0 of the measured copy bandwidth; a decode
// step of 16 tokens in 3 us, which is the launch and two round trips to memory (lengths, then rows).
#include "common.cuh"

namespace stc {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = kThreads / 8;             // (token, head slot) lanes of a CTA
constexpr int kRowsInFlight = 4;

struct RopeArgs {
    const double* inv_freq;
    const int32_t* seq_len;
    const int32_t* old_len;
    const int32_t* positions;
    const uint4 *q_in, *k_in, *v_in;             // strides in 16-byte chunks per token
    int64_t q_stride, k_stride, v_stride;
    uint4 *q_out, *k, *v;
    int32_t* status;
    int Hq, Hkv, T, max_new, rot, chunks;        // chunks of tokens per sequence
    float scale;
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

// One duo turned: HALF: x holds the first, y the second members of eight pairs; else x and y hold four whole
// pairs each, one per word.  One rounding to bf16 per output.
template <bool HALF>
__device__ __forceinline__ void turn_duo(uint4& x, uint4& y, const float (&cs)[8], const float (&sn)[8]) {
    uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (HALF) {
            const float a0 = bf16lo(xw[w]), a1 = bf16hi(xw[w]), b0 = bf16lo(yw[w]), b1 = bf16hi(yw[w]);
            const float c0 = cs[2 * w], c1 = cs[2 * w + 1], s0 = sn[2 * w], s1 = sn[2 * w + 1];
            xw[w] = pack2(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
            yw[w] = pack2(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
        } else {
            const float a0 = bf16lo(xw[w]), b0 = bf16hi(xw[w]), a1 = bf16lo(yw[w]), b1 = bf16hi(yw[w]);
            xw[w] = pack2(a0 * cs[w] - b0 * sn[w], b0 * cs[w] + a0 * sn[w]);
            yw[w] = pack2(a1 * cs[4 + w] - b1 * sn[4 + w], b1 * cs[4 + w] + a1 * sn[4 + w]);
        }
    }
    x = make_uint4(xw[0], xw[1], xw[2], xw[3]);
    y = make_uint4(yw[0], yw[1], yw[2], yw[3]);
}

// TOK tokens and kLanes / TOK head slots per CTA.
template <int TOK, bool HALF>
__global__ void __launch_bounds__(kThreads)
rope_write_kernel(const RopeArgs a) {
    constexpr int SLOTS = kLanes / TOK;
    const int b = blockIdx.x / a.chunks, part = blockIdx.x - b * a.chunks;
    const int duo = threadIdx.x & 7, row = threadIdx.x >> 3;
    const int slot = row % SLOTS, i = part * TOK + row / SLOTS;          // i-th new token
    const int nl = clamp_len(a.seq_len, b, a.T), ol = a.old_len[b];
    const bool bad = ol < 0 || ol > nl || nl - ol > a.max_new;
    if (part == 0 && threadIdx.x == 0) a.status[b] = bad ? STC_ERR_INVALID_ARG : STC_OK;
    if (bad || i >= nl - ol) return;
    const int t = ol + i;

    const int duos = a.rot / 16;                                          // rotated duos of a row
    const bool turned = duo < duos;
    const int c0 = (HALF && turned) ? duo : 2 * duo, c1 = (HALF && turned) ? duo + duos : 2 * duo + 1;
    float cs[8], sn[8];
    if (turned) {
        const long long pos = a.positions ? a.positions[(size_t)b * a.max_new + i] : t;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double turns = a.inv_freq[duo * 8 + e] * 0.15915494309189535;      // 1 / 2 pi
            const unsigned long long step = __double2ull_rn((turns - floor(turns)) * 18446744073709551616.0);
            const long long at = (long long)(step * (unsigned long long)pos);        // turns x 2^64, wrapped to +-1/2
            float s, c;
            sincospif((float)at * 1.0842021724855044e-19f, &s, &c);                  // x 2^-63: half turns
            cs[e] = c * a.scale;
            sn[e] = s * a.scale;
        }
    }

    // rows of this lane: slot, slot + SLOTS, ... of the token's q rows, then k, then v; all parts together, so that a short
    // call has every row of the token in flight at once
    const size_t token = (size_t)b * a.max_new + i;
    const int nq = a.q_in ? a.Hq : 0, nk = nq + (a.k_in ? a.Hkv : 0), nv = nk + (a.v_in ? a.Hkv : 0);
    const int64_t cache_step = (int64_t)a.T * kOctets;                    // from head to head of the cache
    const size_t cache_row = ((size_t)b * a.Hkv * a.T + t) * kOctets;
    const uint4 *q_src = a.q_in + token * a.q_stride, *k_src = a.k_in + token * a.k_stride, *v_src = a.v_in + token * a.v_stride;
#pragma unroll 1
    for (int h0 = slot; h0 < nv; h0 += SLOTS * kRowsInFlight) {
        uint4 x[kRowsInFlight], y[kRowsInFlight];
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int h = h0 + j * SLOTS;
            if (h < nv) {
                const uint4* src = h < nq ? q_src + h * kOctets : h < nk ? k_src + (h - nq) * kOctets : v_src + (h - nk) * kOctets;
                x[j] = src[c0];
                y[j] = src[c1];
            }
        }
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int h = h0 + j * SLOTS;
            if (h < nv) {
                if (h < nk && turned) turn_duo<HALF>(x[j], y[j], cs, sn);
                uint4* dst = h < nq ? a.q_out + (token * a.Hq + h) * kOctets
                                    : h < nk ? a.k + cache_row + (h - nq) * cache_step : a.v + cache_row + (h - nk) * cache_step;
                dst[c0] = x[j];
                dst[c1] = y[j];
            }
        }
    }
}

}  // namespace

cudaError_t launch_rope_write(const Geom& g, const stc_rope& rope, const int32_t* old_len, int max_new,
                              const int32_t* positions, const void* q_in, int64_t q_stride, const void* k_in,
                              int64_t k_stride, const void* v_in, int64_t v_stride, void* q_out, void* k, void* v,
                              int32_t* status, cudaStream_t st) {
    if (g.B == 0 || max_new <= 0) return cudaSuccess;
    RopeArgs a;
    a.inv_freq = rope.inv_freq; a.seq_len = g.seq_len; a.old_len = old_len; a.positions = positions;
    a.q_in = static_cast<const uint4*>(q_in); a.k_in = static_cast<const uint4*>(k_in);
    a.v_in = static_cast<const uint4*>(v_in);
    a.q_stride = q_stride / 8; a.k_stride = k_stride / 8; a.v_stride = v_stride / 8;
    a.q_out = static_cast<uint4*>(q_out); a.k = static_cast<uint4*>(k); a.v = static_cast<uint4*>(v);
    a.status = status;
    a.Hq = g.Hq; a.Hkv = g.Hkv; a.T = g.T; a.max_new = max_new; a.rot = rope.rot_dim; a.scale = rope.scale;
    int sms = 0;
    cudaError_t e = device_sm_count(&sms);
    if (e != cudaSuccess) return e;
    // four tokens per CTA once that still gives every SM one, else one token per CTA (8 x 511 ragged tokens: 10.7 against
    // 16.8 us; 2 x 16384 tokens: 2, 4, 8, 16, 32 tokens per CTA take 143, 124, 124, 127, 131 us)
    // (max_new is a bound and a row stride: no sequence has more than T new tokens, and none of a CTA's token numbers overflows)
    const int most = max_new < g.T ? max_new : g.T;
    const long long tokens = (long long)g.B * most;
    const int tok = tokens >= 4LL * sms ? 4 : 1;
    a.chunks = (most + tok - 1) / tok;
    const long long n_cta = (long long)a.chunks * g.B;
    if (n_cta > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
#define STC_ROPE(TOK_)                                                                                  \
    do {                                                                                                \
        if (rope.interleaved) rope_write_kernel<TOK_, false><<<(unsigned)n_cta, kThreads, 0, st>>>(a);  \
        else rope_write_kernel<TOK_, true><<<(unsigned)n_cta, kThreads, 0, st>>>(a);                    \
    } while (0)
    if (tok == 4) STC_ROPE(4);
    else STC_ROPE(1);
#undef STC_ROPE
    return cudaGetLastError();
}

}  // namespace stc
