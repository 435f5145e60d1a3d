// few.cu -- the whole MoE FFN layer for a few tokens (T <= 64) in one kernel, sm_103a.
//
// With few tokens the layer of Eqs. 1 and 4-7 is a stream of weights: the router, then W1 (and
// W3) and W2 of the experts that some token selects, each byte read once.  One cooperative
// launch, one CTA per SM:
//
//   1. Router logits.  CTA (eb, ds) forms x . W_r for 8 experts and one part of d, in fp32, and
//      the parts' sums of squares of the router columns and of the tokens; grid barrier.
//   2. Selection, one warp per token: keys sigmoid(s) + b from the summed logits, k rounds of
//      arg-max, and a certificate: |error of s| <= n 2^-24 |x| |W_r[:, e]| (n: the length of the
//      summation chains, products of bf16 and fp32 being exact inside an FMA), so a selection
//      whose margin exceeds the key errors is the exact one.  Otherwise the experts near the
//      boundary get 64-bit logits and keys.  Up to FEW_SEL_WARPS tokens every CTA selects for
//      itself (no second barrier); above, the CTAs share the tokens out and meet again.
//   3. Expert products on tcgen05 with the weights as the M operand: D[columns of W, tokens] =
//      W^T . x^T.  W tiles (64 or 128 columns) go from HBM to shared memory by TMA as they lie
//      (MN-major, 128-byte swizzle) and no thread touches them again; the tokens are the N
//      operand, 16 or 32 columns, so the tensor cores do in passing what would otherwise cost an
//      unpack and an FMA per weight and token.  Items (expert, columns) are dealt to the CTAs
//      round-robin.  The weights are marked evict-first in L2: they are read once, and what is
//      read again by the next call (this code, the router's weights) stays.
//   4. Up items apply the activation and store it as two bf16 pieces (hi + lo, 16 bits) so that y
//      is rounded to bf16 once.  Down items (expert, columns, part of K) wait for their expert's up
//      items (a counter), while their weights are already on the way: the weight loads run ahead
//      of the wait by the whole ring.
//   5. Down items leave fp32 partial rows and count them; every warp of the grid sums a share of
//      (token, columns) in slot order once they are complete (no float atomics: results do not
//      depend on timing).
//
// Waits between CTAs rely on co-residency (cooperative launch) and on the item order: every
// CTA takes its up items before its down items and all items before its sums, and up items wait
// for nothing.  All waits have time limits.
//
// What bounds it, measured on one GB300 (against the time of the weights' bytes at the measured
// copy bandwidth of 6.77 TB/s).  Many tokens: the weights' bytes behind a front of 11 to 15 us; 64
// tokens, d 1664, 8 slots, 171 of 256 experts of h 416 touched: 94 us, bytes 72.  One token: a chain of
// dependent steps, each a trip to L2 or HBM (0.7 to 1.5 us): 25 us at d 1536, 8 slots, h 768 (bytes
// 5.6) with the weights in L2 from the call before, 33 with cold ones; of the former about 2 launch, 4
// logits and barrier, 2 selection, 1.2 plan, 5.5 up, 2.4 activation and hand-over, 2.8 down, 3 sum.
// The same layer by the batch path takes 54 to 58 and 65 us.  The code before the first weight
// load is kept short rather than unrolled: run once per call, it is paced by instruction fetches
// (a selection by unrolled counting took 6 us where this one takes 2).
#include <math.h>

#include <atomic>

#include "internal.h"

namespace mv {

namespace {

constexpr int FEW_EPI_WARPS = 8;      // two groups of four (one warp per TMEM lane quadrant)
constexpr int FEW_WARP_W = 8;         // weight loads
constexpr int FEW_WARP_MMA = 9;
constexpr int FEW_WARP_B = 10;        // token / hidden loads: two warps in turn
constexpr int FEW_WARPS = 12;
constexpr int FEW_THREADS = FEW_WARPS * 32;
constexpr int FEW_SEL_WARPS = 8;      // tokens that every CTA selects for itself
constexpr int FEW_TILE_BYTES = 128 * 64 * 2;   // 128 columns x 64 K rows of a weight matrix
constexpr int FEW_TOKEN_BYTES = 2 * 32 * 128;   // token rows of a stage
constexpr int FEW_RT_K = 512;         // rows of W_r staged at a time
constexpr int FEW_RT_XLD = FEW_RT_K + 16;      // row strides of the staged x (bf16; rows 16-byte
constexpr int FEW_RT_WLD = FEW_RT_K + 4;       //   aligned) and W_r^T (fp32)
constexpr int FEW_SMEM_MAX = 232448 - 3072;   // 227 KB less the kernel's static variables
constexpr int FEW_BAR_BYTES = 512, FEW_FLAG_BYTES = 64;   // (multiples of 64)
// Parts of K at most: of a routed and of a shared down item.
constexpr int FEW_MAX_P2 = 4, FEW_MAX_P2S = 8;

__device__ __forceinline__ int up16(int v) { return (v + 15) & ~15; }
// q / d for 0 <= q < 2^24, from an approximate reciprocal: integer division takes some hundred
// cycles, and the way from the router to the first weights is a chain of such small steps.
__device__ __forceinline__ int few_div(int q, int d, float inv) {
    int r = (int)((float)q * inv);
    r += (r + 1) * d <= q ? 1 : 0;
    r -= r * d > q ? 1 : 0;
    return r;
}

// Barrier of one epilogue group's 128 threads.
__device__ __forceinline__ void epi_sync(int group) { asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory"); }
// 32 lanes x 8 consecutive 32-bit columns (thread i: lane base + i).
__device__ __forceinline__ void tmem_ld_32x32b_x8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(taddr)
        : "memory");
}

constexpr unsigned long long FEW_BROKEN = 1ull << 63;   // mark of a count
// Grid barrier on a counter that only grows (64 bits; every launch adds the same multiple of the
// grid's size): one atomic per CTA and no reset, so its cost is two trips to L2.  Gives up
// after the time limit (false, recorded).  The count then need not be a multiple of the grid any
// more, and a later barrier could pass early, so it is marked, and no barrier passes on a marked count:
// neither in this launch nor in a later one, until the workspace is set up again.
__device__ bool few_barrier(DevStatus* st, uint64_t limit_ns) {
    __shared__ int s_ok;
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned long long ticket, now;
        asm volatile("atom.add.acq_rel.gpu.global.u64 %0, [%1], 1;" : "=l"(ticket) : "l"(&st->few_arrivals) : "memory");
        // (a marked ticket waits for nothing)
        const unsigned long long want = ticket < FEW_BROKEN ? (ticket / gridDim.x + 1) * gridDim.x : 0ull;
        const uint64_t t0 = globaltimer_ns();
        now = ticket;
        for (uint32_t i = 1; now < want; ++i) {
            asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(now) : "l"(&st->few_arrivals) : "memory");
            if ((i & 63u) == 0u && now < want && globaltimer_ns() - t0 > limit_ns) {
                atomicOr(&st->few_arrivals, FEW_BROKEN);
                report(st, MOEVIE_ERR_TIMEOUT, SITE_FEW_BARRIER, (int)blockIdx.x, (int)(want - now));
                now = FEW_BROKEN;
            }
        }
        s_ok = now < FEW_BROKEN;
    }
    __syncthreads();
    return s_ok != 0;
}

// ------------------------------------------------------------- 1. logits

// Two fp32 values in one register pair, and a fused multiply-add or a sum of both in one instruction.
__device__ __forceinline__ uint64_t f32x2(float a, float b) {
    return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float both(uint64_t v) {
    return __uint_as_float((uint32_t)v) + __uint_as_float((uint32_t)(v >> 32));
}
// Sums v[0..7] over the 8 lanes that differ in bits 0 to 2: lane l gets that of v[l & 7].
__device__ __forceinline__ float sum8(const float v[8]) {
    const int lane = threadIdx.x & 31;
    float a[4], b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        a[i] = (lane & 4 ? v[i + 4] : v[i]) + __shfl_xor_sync(0xffffffffu, lane & 4 ? v[i] : v[i + 4], 4);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        b[i] = (lane & 2 ? a[i + 2] : a[i]) + __shfl_xor_sync(0xffffffffu, lane & 2 ? a[i] : a[i + 2], 2);
    return (lane & 1 ? b[1] : b[0]) + __shfl_xor_sync(0xffffffffu, lane & 1 ? b[0] : b[1], 1);
}

// part[ds][t][e], wsq[ds][e] and xsq[ds][t] of this CTA's blocks of 8 experts x parts of d.  Up to
// FEW_RT_K rows at a time are staged by cp.async, all copies in flight at once: x as bf16
// [8 TG][FEW_RT_XLD], W_r^T as fp32 [8][FEW_RT_WLD].  A warp sums 8 tokens (group g) over its
// share kp of K; lane (ep, ks): experts ep and ep + 4, four K of every 32.
__device__ void few_logits(const FewArgs& p, uint8_t* smem) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int TG = (p.T + 7) / 8, KP = p.rt_kp;   // KP = FEW_WARPS / TG
    float* ws = reinterpret_cast<float*>(smem);
    float* red = ws + 8 * FEW_RT_WLD;      // [KP][8 TG][8]
    float* redq = red + FEW_WARPS * 64;    // [KP][8]
    float* redx = redq + FEW_WARPS * 8;    // [KP][8 TG]
    __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(redx + FEW_WARPS * 8);
    const int kp = few_div(warp, TG, __fdividef(1.0f, (float)TG)), g = warp - kp * TG, ep = lane >> 3, ks = lane & 7;
    for (int item = blockIdx.x; item < p.rt_eb * p.rt_parts; item += gridDim.x) {
        const int ds = few_div(item, p.rt_eb, __fdividef(1.0f, (float)p.rt_eb)), e0 = (item - ds * p.rt_eb) * 8;
        const int d0 = ds * p.rt_dch, d1 = min(p.d, d0 + p.rt_dch);
        uint64_t tot[2][8] = {}, sq[2] = {};   // sums of the even and of the odd K
        float xq = 0.f;                        // lane l: |x|^2 of token 8 g + (l & 7)
        for (int k0 = d0; k0 < d1; k0 += FEW_RT_K) {
            const int kc = min(FEW_RT_K, d1 - k0), kcp = (kc + 31) & ~31;
            for (int q = threadIdx.x; q < kcp * 8; q += FEW_THREADS) {
                const int r = q >> 3, e = q & 7;
                const bool in = r < kc && e0 + e < p.E;
                const float* src = p.W_r + (in ? (int64_t)(k0 + r) * p.E + e0 + e : 0);
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(
                                 smem_u32(ws + e * FEW_RT_WLD + r)), "l"(src), "r"(in ? 4u : 0u)
                             : "memory");
            }
            for (int t = warp; t < p.T; t += FEW_WARPS)
                for (int c = lane * 8; c < kcp; c += 256)   // kc is a multiple of 8, as d and the parts are
                    cp_async16(smem_u32(xs + t * FEW_RT_XLD + c), c < kc ? p.x + (int64_t)t * p.d + k0 + c : p.x,
                               c < kc ? 16u : 0u);
            cp_async_wait_all();
            __syncthreads();
            if (kp < KP) {
                uint64_t acc[2][8] = {};
                auto products = [&](int it) {   // 32 rows
                    const int k = it * 32 + ks * 4;
                    const ulonglong2 w0 = *reinterpret_cast<const ulonglong2*>(ws + ep * FEW_RT_WLD + k);
                    const ulonglong2 w1 = *reinterpret_cast<const ulonglong2*>(ws + (ep + 4) * FEW_RT_WLD + k);
                    sq[0] = fma2(w0.x, w0.x, fma2(w0.y, w0.y, sq[0]));
                    sq[1] = fma2(w1.x, w1.x, fma2(w1.y, w1.y, sq[1]));
#pragma unroll
                    for (int i = 0; i < 8; ++i) {   // (rows past T hold no token: their sums are dropped)
                        const uint2 xx = *reinterpret_cast<const uint2*>(xs + (8 * g + i) * FEW_RT_XLD + k);
                        const uint64_t x0 = f32x2(__uint_as_float(xx.x << 16), __uint_as_float(xx.x & 0xffff0000u));
                        const uint64_t x1 = f32x2(__uint_as_float(xx.y << 16), __uint_as_float(xx.y & 0xffff0000u));
                        acc[0][i] = fma2(x1, w0.y, fma2(x0, w0.x, acc[0][i]));
                        acc[1][i] = fma2(x1, w1.y, fma2(x0, w1.x, acc[1][i]));
                    }
                };
                int it = kp;
#pragma unroll 1
                for (; it + KP < kcp / 32; it += 2 * KP) {
                    products(it);
                    products(it + KP);
#pragma unroll
                    for (int i = 0; i < 8; ++i)   // short chains: 4 products, then their sums
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            tot[u][i] = add2(tot[u][i], acc[u][i]);
                            acc[u][i] = 0ull;
                        }
                }
                if (it < kcp / 32) products(it);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    tot[0][i] = add2(tot[0][i], acc[0][i]);
                    tot[1][i] = add2(tot[1][i], acc[1][i]);
                }
                if (e0 == 0) {   // squares of x: lanes ep take every fourth of the warp's 32 columns
                    uint64_t x2[8] = {};
#pragma unroll 1
                    for (int xi = kp + KP * ep; xi < kcp / 32; xi += 4 * KP)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint2 xx =
                                *reinterpret_cast<const uint2*>(xs + (8 * g + i) * FEW_RT_XLD + xi * 32 + ks * 4);
                            const uint64_t x0 = f32x2(__uint_as_float(xx.x << 16), __uint_as_float(xx.x & 0xffff0000u));
                            const uint64_t x1 = f32x2(__uint_as_float(xx.y << 16), __uint_as_float(xx.y & 0xffff0000u));
                            x2[i] = fma2(x1, x1, fma2(x0, x0, x2[i]));
                        }
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = both(x2[i]);
                    float q = sum8(v);
                    q += __shfl_xor_sync(0xffffffffu, q, 8);
                    xq += q + __shfl_xor_sync(0xffffffffu, q, 16);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float v[8], q = both(sq[u]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = both(tot[u][i]);
            const float sum = sum8(v);
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
            if (kp < KP) {
                red[(kp * 8 * TG + 8 * g + ks) * 8 + ep + 4 * u] = sum;
                if (g == 0 && ks == 0) redq[kp * 8 + ep + 4 * u] = q;
            }
        }
        if (e0 == 0 && kp < KP && lane < 8) redx[kp * 8 * TG + 8 * g + lane] = xq;
        __syncthreads();
        for (int q = threadIdx.x; q < (p.T + 1) * 8; q += FEW_THREADS) {
            const int t = q >> 3, e = q & 7;
            if (e0 + e >= p.E) continue;
            float s = 0.f;
            if (t < p.T) {
                for (int j = 0; j < KP; ++j) s += red[(j * 8 * TG + t) * 8 + e];
                p.part[((int64_t)ds * p.T + t) * p.E + e0 + e] = s;
                if (q == t * 8 && e0 == 0) {
                    s = 0.f;
                    for (int j = 0; j < KP; ++j) s += redx[j * 8 * TG + t];
                    p.xsq[ds * p.T + t] = s;
                }
            } else {
                for (int j = 0; j < KP; ++j) s += redq[j * 8 + e];
                p.wsq[ds * p.E + e0 + e] = s;
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------- 2. selection

// Order-preserving map of keys to unsigned; NaN before (below) every number, 0: none.
__device__ __forceinline__ uint32_t key_order(float f) {
    if (f != f) return 1u;
    const uint32_t u = __float_as_uint(f + 0.0f);   // -0 -> +0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Sum of up to 8 values `stride` floats apart, all loads in flight at once, added in order.
__device__ __forceinline__ float sum_parts(const float* q, int64_t stride, int n) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? __ldcg(q + j * stride) : 0.f;
    float s = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) s += v[j];
    return s;
}

// Bytes of shared memory per expert (E rounded up to 32) that one token's selection takes:
// bounds of the key (later the 64-bit key), the fp32 key, all as their order; logit; list of experts
// to decide exactly.
constexpr int FEW_SEL_BYTES = 18;

// k rounds of arg-max over a token's keys, by one warp: lane l holds the order of experts l,
// l + 32, ... in registers (NQMAX >= NQ of them).  Lane j < k returns the j-th selected expert.
// lo, hi: the lowest lower bound of a selected key and the highest upper bound of another one.
template <int NQMAX>
__device__ __forceinline__ int few_rounds(int k, int NQ, const uint32_t* ok, const uint32_t* lob, const uint32_t* hib,
                                          uint32_t& lo, uint32_t& hi) {
    const int lane = threadIdx.x & 31;
    uint32_t key[NQMAX];
    int mine = 0;
#pragma unroll
    for (int q = 0; q < NQMAX; ++q) key[q] = q < NQ ? ok[q * 32 + lane] : 0u;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        uint32_t top = 0u;
#pragma unroll
        for (int q = 0; q < NQMAX; ++q) top = max(top, key[q]);
        top = __reduce_max_sync(0xffffffffu, top);
        int e = NQMAX * 32;   // the lowest id with that key
#pragma unroll
        for (int q = NQMAX - 1; q >= 0; --q)
            if (key[q] == top) e = q * 32 + lane;
        e = __reduce_min_sync(0xffffffffu, e);
#pragma unroll
        for (int q = 0; q < NQMAX; ++q)
            if (e == q * 32 + lane) key[q] = 0u;
        if (lane == j) mine = e;
    }
    hi = 0u;
#pragma unroll
    for (int q = 0; q < NQMAX; ++q)
        if (key[q] != 0u) hi = max(hi, hib[q * 32 + lane]);
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lane < k ? lob[mine] : 0xffffffffu);
    return mine;
}

// Places of a token's selected experts (lane j < k holds the j-th; ascending ids) and their gates,
// by one warp; with `mask` also the token's bit in each of those experts' token masks.
__device__ __forceinline__ void few_place(const FewArgs& p, int t, int mine, const float* lg, int32_t* out_idx,
                                          float* out_gate, unsigned long long* mask) {
    const int lane = threadIdx.x & 31;
    const float s = lane < p.k ? __fdividef(1.0f, 1.0f + expf(-lg[mine])) : 0.f;
    const float sum = warp_sum(s);
    int at = t * p.k;
#pragma unroll 1
    for (int j = 0; j < p.k; ++j) at += __shfl_sync(0xffffffffu, mine, j) < mine;
    if (lane < p.k) {
        out_idx[at] = mine;
        out_gate[at] = __fdividef(s, sum);
        if (mask) atomicOr(&mask[mine], 1ull << t);
    }
}

// Selection and gates of the CTA's tokens t0, t0 + step, ... (n <= FEW_SEL_WARPS of them), by all
// threads.  buf: FEW_SEL_BYTES per expert and token.
__device__ void few_select(const FewArgs& p, int t0, int step, int n, uint8_t* buf,
                           int32_t* out_idx, float* out_gate, unsigned long long* mask) {
    __shared__ uint32_t s_sel[FEW_SEL_WARPS][32];
    __shared__ int n_cand[FEW_SEL_WARPS];
    __shared__ double part64[FEW_WARPS][4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, NQ = (p.E + 31) / 32, Ep = NQ * 32;
    auto base = [&](int w) { return buf + (size_t)w * Ep * FEW_SEL_BYTES; };
    auto lob_of = [&](int w) { return reinterpret_cast<uint32_t*>(base(w)); };
    auto hib_of = [&](int w) { return reinterpret_cast<uint32_t*>(base(w) + Ep * 4); };
    auto kd_of = [&](int w) { return reinterpret_cast<double*>(base(w)); };   // in the bounds' place
    auto ok_of = [&](int w) { return reinterpret_cast<uint32_t*>(base(w) + Ep * 8); };
    auto lg_of = [&](int w) { return reinterpret_cast<float*>(base(w) + Ep * 12); };
    auto cand_of = [&](int w) { return reinterpret_cast<uint16_t*>(base(w) + Ep * 16); };
    const float inv_NQ = __fdividef(1.0f, (float)NQ);
    for (int q = warp; q < n * NQ; q += FEW_WARPS) {
        const int w = few_div(q, NQ, inv_NQ), e = (q - w * NQ) * 32 + lane;
        uint32_t o = 0u, ob = 0u, oa = 0u;
        if (e < p.E) {
            const float s = sum_parts(p.part + (int64_t)(t0 + w * step) * p.E + e, (int64_t)p.T * p.E, p.rt_parts);
            const float w2 = sum_parts(p.wsq + e, p.E, p.rt_parts);
            const float x2 = sum_parts(p.xsq + t0 + w * step, p.T, p.rt_parts);
            const float v = __fdividef(1.0f, 1.0f + __expf(-s)) + __ldg(p.b + e);
            // Half-width of the key: a quarter (the sigmoid's largest slope; and some, for the
            // square root) of the logit's error bound, and the fp32 evaluation (fast sigmoid:
            // under 1e-6; the sum's rounding).  A NaN bound bounds nothing.
            float wn, xn;
            asm("sqrt.approx.f32 %0, %1;" : "=f"(wn) : "f"(w2));
            asm("sqrt.approx.f32 %0, %1;" : "=f"(xn) : "f"(x2));
            const float r = 0.2501f * p.rt_err * xn * wn + 2e-6f + 2.4e-7f * fabsf(v), a = v - r, b = v + r;
            o = key_order(v);
            oa = a == a ? key_order(a) : 0u;
            ob = b == b ? key_order(b) : 0xffffffffu;
            lg_of(w)[e] = s;
        }
        ok_of(w)[e] = o;
        lob_of(w)[e] = oa;
        hib_of(w)[e] = ob;
    }
    __syncthreads();
    int unsure = 0;
    if (warp < n) {
        const uint32_t *ok = ok_of(warp), *lob = lob_of(warp), *hib = hib_of(warp);
        uint32_t lo, hi;
        int mine;
        if (NQ <= 2) mine = few_rounds<2>(p.k, NQ, ok, lob, hib, lo, hi);
        else if (NQ <= 8) mine = few_rounds<8>(p.k, NQ, ok, lob, hib, lo, hi);
        else mine = few_rounds<32>(p.k, NQ, ok, lob, hib, lo, hi);
        if (lane == 0) n_cand[warp] = 0;
        if (p.k == p.E || lo > hi) {
            few_place(p, t0 + warp * step, mine, lg_of(warp), out_idx, out_gate, mask);
        } else {
            // The lowest selected key may not be above the highest other one.  An expert whose
            // lower bound is above every other upper bound is in, one whose upper bound is below
            // every selected lower bound is out; the rest get exact keys.
            unsure = 1;
            s_sel[warp][lane] = 0u;
            __syncwarp();
            if (lane < p.k) atomicOr(&s_sel[warp][mine >> 5], 1u << (mine & 31));
            __syncwarp();
            int nc = 0;
            for (int q = 0; q < NQ; ++q) {
                const int e = q * 32 + lane;
                const bool sel = s_sel[warp][q] >> lane & 1u;
                const bool c = e < p.E && (sel ? lob[e] <= hi : hib[e] >= lo);
                const uint32_t m = __ballot_sync(0xffffffffu, c), ms = __ballot_sync(0xffffffffu, sel && !c);
                if (c) cand_of(warp)[nc + __popc(m & ((1u << lane) - 1u))] = (uint16_t)e;
                __syncwarp();
                if (lane == 0) s_sel[warp][q] = ms;
                nc += __popc(m);
            }
            if (lane == 0) n_cand[warp] = nc;
        }
    }
    if (!__syncthreads_or(unsure)) return;
    for (int w = 0; w < n; ++w) {
        const int nc = n_cand[w];
        if (nc == 0) continue;
        // Exact logits, by all threads, four experts at a time: products of bf16 and fp32 are
        // exact in 64 bits, summed in a fixed order.
        const __nv_bfloat16* x = p.x + (int64_t)(t0 + w * step) * p.d;
        for (int c0 = 0; c0 < nc; c0 += 4) {
            double s[4] = {};
            const float* col[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) col[j] = p.W_r + cand_of(w)[min(c0 + j, nc - 1)];
#pragma unroll 4
            for (int i = threadIdx.x; i < p.d; i += FEW_THREADS) {
                const double xv = (double)__bfloat162float(x[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] = fma(xv, (double)__ldg(col[j] + (int64_t)i * p.E), s[j]);
            }
            for (int o = 16; o; o >>= 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] += __shfl_xor_sync(0xffffffffu, s[j], o);
            if (lane < 4) part64[warp][lane] = lane == 0 ? s[0] : lane == 1 ? s[1] : lane == 2 ? s[2] : s[3];
            __syncthreads();
            if (threadIdx.x < 4 && c0 + (int)threadIdx.x < nc) {
                const int e = cand_of(w)[c0 + threadIdx.x];
                double t = 0.0;
                for (int j = 0; j < FEW_WARPS; ++j) t += part64[j][threadIdx.x];
                kd_of(w)[e] = 1.0 / (1.0 + exp(-t)) + (double)__ldg(p.b + e);
            }
            __syncthreads();
        }
        // The places that the sure ones leave go to the largest exact keys (a number before NaN,
        // the lower id of equals).
        int need = p.k;
        for (int q = 0; q < NQ; ++q) need -= __popc(s_sel[w][q]);
        __syncthreads();
        for (int c = threadIdx.x; c < nc; c += FEW_THREADS) {
            const int e = cand_of(w)[c];
            const double v = kd_of(w)[e];
            int ahead = 0;
            for (int j = 0; j < nc; ++j) {
                const int f = cand_of(w)[j];
                const double u = kd_of(w)[f];
                ahead += isnan(v) != isnan(u) ? (isnan(v) ? 1 : 0) : (u > v || (!(v > u) && f < e)) ? 1 : 0;
            }
            if (ahead < need) atomicOr(&s_sel[w][e / 32], 1u << (e & 31));
        }
        __syncthreads();
    }
    if (warp < n && n_cand[warp] > 0) {
        int mine = 0, at = 0;
        for (int q = 0; q < NQ; ++q) {
            const uint32_t m = s_sel[warp][q];
            if (lane >= at && lane < at + __popc(m)) mine = q * 32 + (int)__fns(m, 0, lane - at + 1);
            at += __popc(m);
        }
        few_place(p, t0 + warp * step, mine, lg_of(warp), out_idx, out_gate, mask);
    }
    __syncthreads();
}

// ----------------------------------------------------- 3. work of a call

// An entry is up to nb (16 or 32) tokens of one expert; most experts have one.  More tokens make
// another entry, whose weights then come from L2: with larger N operands the ring would hold fewer
// weights in flight for every expert.
//
// Built by every CTA from the selection; kept in shared memory (128 bytes at most).
struct FewPlan {
    int n_act;              // entries
    int tw, nt, nt_s;       // up items: columns (64 or 128), tiles of h and of h_s
    int tw2, ntd, P2, P2s;  // down items: columns, tiles of d, parts of K (routed, shared)
    int n_up_shared, n_up, n_down_shared, n_items;   // items: up, then down (shared first in each)
    float inv_sh, inv_nt, inv_ntd, inv_P2, inv_P2s;  // reciprocals of the divisors below
};

struct FewItem {
    int up, shared, i;      // i: entry (routed), block of nb tokens (shared)
    int e;
    int n0, tw, kb0, kb1;   // columns; K blocks of 64
    int part;               // down: K part
    int cnt, row0;          // tokens, first row
};

struct FewLists {           // shared memory
    FewPlan* plan;
    uint16_t* act;          // [na] expert of an entry
    uint16_t* off;          // [na] its first row
    uint8_t* cnt;           // [na] its tokens
    uint8_t* row_tok;       // [T k] token of a row
    uint16_t* row_of;       // [T k] row of slot t k + j
    float* gate;            // [T k]
};

__device__ __forceinline__ FewItem few_item(const FewArgs& p, const FewLists& L, int id) {
    const FewPlan& pl = *L.plan;
    FewItem it;
    it.up = id < pl.n_up;
    int q = it.up ? id : id - pl.n_up;
    it.shared = q < (it.up ? pl.n_up_shared : pl.n_down_shared);
    it.part = 0;
    if (it.up) {
        it.tw = pl.tw;
        it.kb0 = 0;
        it.kb1 = p.nkb_d;
        if (!it.shared) q -= pl.n_up_shared;
        const int per = it.shared ? p.n_sh : pl.nt;   // shared: the blocks of a tile side by side
        const int r = few_div(q, per, it.shared ? pl.inv_sh : pl.inv_nt);
        it.i = it.shared ? q - r * per : r;
        it.n0 = (it.shared ? r : q - r * per) * pl.tw;
    } else {
        if (!it.shared) q -= pl.n_down_shared;
        const int P = it.shared ? pl.P2s : pl.P2, nkb = it.shared ? p.nkb_hs : p.nkb_h;
        const int r = few_div(q, P, it.shared ? pl.inv_P2s : pl.inv_P2);
        const int per = it.shared ? p.n_sh : pl.ntd, v = few_div(r, per, it.shared ? pl.inv_sh : pl.inv_ntd);
        it.part = q - r * P;
        it.i = it.shared ? r - v * per : v;
        it.tw = pl.tw2;
        it.n0 = (it.shared ? v : r - v * per) * pl.tw2;
        const float inv = it.shared ? pl.inv_P2s : pl.inv_P2;
        it.kb0 = few_div(it.part * nkb, P, inv);
        it.kb1 = few_div((it.part + 1) * nkb, P, inv);
    }
    it.e = it.shared ? 0 : L.act[it.i];
    it.row0 = it.shared ? it.i * p.nb : L.off[it.i];
    it.cnt = it.shared ? min(p.nb, p.T - it.row0) : L.cnt[it.i];
    return it;
}

// How an item goes through the ring.  A stage holds two halves of 64 columns x 64 K of weights and
// the token blocks that they meet.  128-column items: a K block's columns (SwiGLU: the gate's and
// the up projection's in turn); 64-column ones: the gate's and the up projection's columns of a K
// block (SwiGLU up items), else two K blocks, where both token blocks fit.  (One K block a stage
// left half the ring empty for 64-column items: one token's up items took 217 ns per 8 KB, with
// two 145 ns.)
struct FewSteps {
    int n;               // stages
    int wide, two;       // 128 columns; SwiGLU up item
    int alt, pair;       // wide and two; two K blocks a stage
    int half2, last2;    // the second half is used, in the last stage
};
__device__ __forceinline__ FewSteps few_steps(const FewArgs& p, const FewItem& it) {
    FewSteps r;
    const int nk = it.kb1 - it.kb0;
    r.two = it.up && p.W3;
    r.wide = it.tw == 128;
    r.alt = r.wide & r.two;
    r.pair = !r.wide && !r.two && (it.up ? 2 : 4) * up16(it.cnt) * 128 <= FEW_TOKEN_BYTES;
    r.n = r.pair ? (nk + 1) >> 1 : nk << r.alt;
    r.half2 = r.wide | r.two | r.pair;
    r.last2 = r.pair ? (nk & 1) ^ 1 : r.half2;
    return r;
}

// Estimated time (ns) of `items` items of `blocks` K blocks of `kb` bytes: an SM takes a block
// in kb / 70 GB/s and 0.2 us (its waits and four MMAs) at least, and c CTAs at work share
// 6600 GB/s (measured with tiles streamed by 8 to 152 SMs); the last, partial round of items runs
// at its own c; 400 ns an item besides.
__device__ __forceinline__ float few_time(int items, int blocks, int kb, int ctas) {
    const int rounds = few_div(items, ctas, __fdividef(1.0f, (float)ctas)), rest = items - rounds * ctas;
    const float one = fmaxf((float)kb / 70.0f, 200.0f), all = (float)kb / 6600.0f;
    return rounds * (blocks * fmaxf(one, all * ctas) + 400.0f) +
           (rest > 0 ? blocks * fmaxf(one, all * rest) + 400.0f : 0.0f);
}
// The lane with the smallest time (the lowest of equals).
__device__ __forceinline__ int few_fastest(float t) {
    const uint32_t c = (uint32_t)fminf(t, 1.0e8f) * 32u + (threadIdx.x & 31);
    return (int)(__reduce_min_sync(0xffffffffu, c) & 31u);
}

// Expert lists and the plan from the selection (idx, gate of all slots).  mask: the experts'
// token masks; off: 2 bytes per expert of scratch.  The selection and its masks lie in shared memory
// (SHARED_SEL), or other CTAs wrote the selection to global memory and the masks are built here.
template <bool SHARED_SEL>
__device__ void few_plan(const FewArgs& p, const FewLists& L, const int32_t* idx, const float* gate,
                         unsigned long long* mask, uint16_t* off) {
    __shared__ int n_in[32], rows_in[32];   // of each 32 experts: entries, rows
    auto load = [](const auto* q) { return SHARED_SEL ? *q : __ldcg(q); };
    const int n = p.T * p.k, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x < 32) n_in[threadIdx.x] = rows_in[threadIdx.x] = 0;
    if (!SHARED_SEL)
        for (int e = threadIdx.x; e < p.E; e += FEW_THREADS) mask[e] = 0ull;
    constexpr int PER = (MOEVIE_FEW_MAX_TOKENS * 32 + FEW_THREADS - 1) / FEW_THREADS;   // slots of a thread
    int my_e[PER];
    float my_g[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = threadIdx.x + i * FEW_THREADS;
        if (s >= n) break;
        my_e[i] = load(idx + s);
        my_g[i] = load(gate + s);
    }
    __syncthreads();
    if (!SHARED_SEL) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int s = threadIdx.x + i * FEW_THREADS;
            if (s >= n) break;
            atomicOr(&mask[my_e[i]], 1ull << few_div(s, p.k, p.inv_k));
        }
        __syncthreads();
    }
    const int sh = p.nb == 16 ? 4 : 5;
    for (int q = warp; q * 32 < p.E; q += FEW_WARPS) {
        const int e = q * 32 + lane, c = e < p.E ? __popcll(mask[e]) : 0;
        const int ent = (int)__reduce_add_sync(0xffffffffu, (unsigned)((c + p.nb - 1) >> sh));
        const int rows = (int)__reduce_add_sync(0xffffffffu, (unsigned)c);
        if (lane == 0) {
            n_in[q] = ent;
            rows_in[q] = rows;
        }
    }
    __syncthreads();
    // inclusive prefixes over the groups of 32, in every warp
    int na = n_in[lane], nrow = rows_in[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, na, o), v = __shfl_up_sync(0xffffffffu, nrow, o);
        if (lane >= o) {
            na += u;
            nrow += v;
        }
    }
    const int n_act = __shfl_sync(0xffffffffu, na, 31);
    for (int q = warp; q * 32 < p.E; q += FEW_WARPS) {
        const int e = q * 32 + lane, c = e < p.E ? __popcll(mask[e]) : 0, ent = (c + p.nb - 1) >> sh;
        int sum = c + (ent << 16);   // inclusive prefixes over the lanes: rows, entries
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        int i = __shfl_sync(0xffffffffu, na, q) - n_in[q] + (sum >> 16) - ent;
        int row = __shfl_sync(0xffffffffu, nrow, q) - rows_in[q] + (sum & 0xffff) - c;
        if (c > 0) off[e] = (uint16_t)row;
        for (int left = c; left > 0; left -= p.nb, ++i, row += p.nb) {
            L.act[i] = (uint16_t)e;
            L.off[i] = (uint16_t)row;
            L.cnt[i] = (uint8_t)min(left, p.nb);
        }
    }
    if (warp == FEW_WARPS - 1) {
        // 64-column items where 128-column ones are too few to keep all SMs streaming; down items
        // may also split K (their partial rows are joined anyway).
        // (shifts and reciprocals: this is on the way of every CTA's first load)
        const int ctas = (int)gridDim.x;
        const int bn = up16(min((int)__fdividef((float)(n + n_act - 1), (float)n_act), p.nb)) * 128;
        const int s_l = 7 - (lane & 1), tw_l = 1 << s_l;
        const int tiles_l = n_act * ((p.h + tw_l - 1) >> s_l) + p.n_sh * ((p.hs + tw_l - 1) >> s_l);
        const bool w128 = s_l == 7;
        const int up_steps = p.W3 ? (w128 ? 2 : 1) * p.nkb_d : w128 ? p.nkb_d : (p.nkb_d + 1) >> 1;
        const int up = few_fastest(
            lane < 2 ? few_time(tiles_l, up_steps, FEW_TILE_BYTES + (w128 || p.W3 ? bn : 2 * bn), ctas) : 3.0e38f);
        const int P_l = (lane >> 1) + 1, ntd_l = (p.d + tw_l - 1) >> s_l;
        const int items_l = ntd_l * P_l * (n_act + p.n_sh * p.sh_ratio);
        const int blocks_l = (int)__fdividef((float)(p.nkb_h + P_l - 1) + 0.5f, (float)P_l);
        const bool pair_l = !w128 && 4 * bn <= FEW_TOKEN_BYTES;
        const int dn = few_fastest(P_l <= FEW_MAX_P2 && P_l <= p.nkb_h
                                       ? few_time(items_l, pair_l ? (blocks_l + 1) >> 1 : blocks_l,
                                                  (pair_l ? 2 : 1) * (tw_l * 128 + 2 * bn), ctas)
                                       : 3.0e38f);
        if (lane == 0) {
            FewPlan& pl = *L.plan;
            const int s1 = 7 - up, s2 = 7 - (dn & 1), P2 = (dn >> 1) + 1;
            pl.n_act = n_act;
            pl.tw = 1 << s1;
            pl.nt = (p.h + pl.tw - 1) >> s1;
            pl.nt_s = (p.hs + pl.tw - 1) >> s1;
            pl.tw2 = 1 << s2;
            pl.P2 = P2;
            pl.ntd = (p.d + pl.tw2 - 1) >> s2;
            // shared down items about as long as the routed ones
            pl.P2s = p.hs > 0 ? min(min(FEW_MAX_P2S, p.nkb_hs),
                                    max(1, (int)__fdividef((float)(p.nkb_hs * P2) + 0.5f * p.nkb_h, (float)p.nkb_h)))
                              : 1;
            pl.n_up_shared = p.n_sh * pl.nt_s;
            pl.n_up = n_act * pl.nt + pl.n_up_shared;
            pl.n_down_shared = p.n_sh * pl.ntd * pl.P2s;
            pl.n_items = pl.n_up + pl.n_down_shared + n_act * pl.ntd * P2;
            pl.inv_sh = __fdividef(1.0f, (float)max(p.n_sh, 1));
            pl.inv_nt = __fdividef(1.0f, (float)pl.nt);
            pl.inv_ntd = __fdividef(1.0f, (float)pl.ntd);
            pl.inv_P2 = __fdividef(1.0f, (float)P2);
            pl.inv_P2s = __fdividef(1.0f, (float)pl.P2s);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = threadIdx.x + i * FEW_THREADS;
        if (s >= n) break;
        const int t = few_div(s, p.k, p.inv_k), e = my_e[i];
        const int row = off[e] + __popcll(mask[e] & ((1ull << t) - 1ull));
        L.row_tok[row] = (uint8_t)t;
        L.row_of[s] = (uint16_t)row;
        L.gate[s] = my_g[i];
    }
}

// -------------------------------------------------------------- 4. roles

struct FewSmem {
    uint32_t ring, full, empty, tfull, tempty, drain;
    uint32_t b_turn;           // barriers of the two warps that load the N operand
    volatile int* b_next;
    int stages, stage_bytes;   // a stage: weights (FEW_TILE_BYTES), then the N operand
};

__device__ __forceinline__ void few_abort(volatile int* flag, DevStatus* st, int site, int a) {
    *flag = 1;
    report(st, MOEVIE_ERR_TIMEOUT, site, (int)blockIdx.x, a);
}

// Weight tiles of every item; never waits for anything but a free stage.
__device__ void few_load_w(const FewArgs& p, const FewSmem& sm, const FewLists& L, volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    const uint64_t pol = l2_policy_evict_first();
    int s = 0;
    uint32_t ph = 0;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x) {
        const FewItem it = few_item(p, L, id);
        const FewSteps st = few_steps(p, it);
        const CUtensorMap* a = it.up ? (it.shared ? &p.tS1 : &p.tW1) : (it.shared ? &p.tS2 : &p.tW2);
        const CUtensorMap* a3 = it.shared ? &p.tS3 : &p.tW3;
        const int n2 = it.n0 + (st.wide ? 64 : 0), dk2 = st.pair ? 64 : 0;
        int k = it.kb0 * 64;
        for (int i = 0; i < st.n; ++i) {
            if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_EMPTY, id);
                return;
            }
            const uint32_t bar = sm.full + 8 * s, dst = sm.ring + s * sm.stage_bytes;
            const int second = i + 1 < st.n ? st.half2 : st.last2, odd = st.alt & i;
            mbar_arrive_expect_tx(bar, (1 + second) * (FEW_TILE_BYTES / 2));
            tma_load_3d_hint(dst, odd ? a3 : a, bar, it.n0, k, it.e, pol);
            if (second)
                tma_load_3d_hint(dst + FEW_TILE_BYTES / 2, st.alt == odd && st.two ? a3 : a, bar, n2, k + dk2, it.e, pol);
            k += st.pair ? 128 : st.alt == odd ? 64 : 0;
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

// The N operand: token rows (up) or the two pieces of the hidden rows (down: hi, then lo N rows
// further), after the entry's up items are done.  Up to 16 tokens: all of them, in order, in one
// copy, whichever the entry has.  More: a gather of the entry's; rows past its last token repeat
// its first.  Rows past the last one hold whatever follows (down).  Columns of D that are not the
// entry's are not read.
//
// Two warps in turn, an item each: while one loads, the other decodes its item and waits for the
// hidden rows (a trip to L2, 0.7 us of the 1.5 us that a short item took).
__device__ void few_load_b(const FewArgs& p, const FewSmem& sm, const FewLists& L, int who, volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    const bool direct = p.T <= 16;
    volatile int* next = sm.b_next;   // stage and phase where the other warp stopped
    uint32_t turn = 0;
    for (int id = blockIdx.x + who * gridDim.x; id < n_items; id += 2 * gridDim.x, turn ^= 1u) {
        const FewItem it = few_item(p, L, id);
        const FewSteps st = few_steps(p, it);
        const int N = up16(it.cnt), bytes = (it.up ? 1 : 2) * N * 128;
        int tok[32];
        if (it.up && !direct) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int j = i < it.cnt ? i : 0;
                if (i < N) tok[i] = it.shared ? it.row0 + j : L.row_tok[it.row0 + j];
            }
        } else if (!it.up) {
            const int32_t* c = p.done_up + (it.shared ? p.na_max + it.i : it.i);
            const int want = it.shared ? L.plan->nt_s : L.plan->nt;
            const uint64_t t0 = globaltimer_ns();
            for (uint32_t i = 1; ld_acquire(c) < want; ++i)
                if ((i & 63u) == 0u && (*abort_flag || globaltimer_ns() - t0 > p.limit_ns)) {
                    few_abort(abort_flag, p.status, SITE_FEW_WAIT_UP, id);
                    return;
                }
            fence_proxy_async_all();   // the hidden rows were written by ordinary stores
        }
        const CUtensorMap* h = it.shared ? &p.tHs : &p.tH;
        // (who 0's first turn passes: the phase before the first)
        if (!mbar_wait(sm.b_turn + 8 * who, turn ^ (who == 0 ? 1u : 0u), p.limit_ns, abort_flag)) {
            few_abort(abort_flag, p.status, SITE_FEW_WAIT_TURN, id);
            return;
        }
        int s = next[0];
        uint32_t ph = (uint32_t)next[1];
        int k = it.kb0 * 64;
        for (int i = 0; i < st.n; ++i) {
            if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_EMPTY, -id);
                return;
            }
            const uint32_t bar = sm.full + 8 * s;
            uint32_t dst = sm.ring + s * sm.stage_bytes + FEW_TILE_BYTES;
            const int blocks = st.pair && (i + 1 < st.n || st.last2) ? 2 : 1;
            mbar_arrive_expect_tx(bar, blocks * bytes);
            for (int k1 = k; k1 < k + 64 * blocks; k1 += 64, dst += bytes) {
                if (!it.up) {
#pragma unroll
                    for (int r = 0; r < 32; r += 16)
                        if (r < N) {
                            tma_load_3d(dst + r * 128, h, bar, k1, it.row0 + r, 0);
                            tma_load_3d(dst + (N + r) * 128, h, bar, k1, it.row0 + r, 1);
                        }
                } else if (direct) {
                    tma_load_3d(dst, &p.tX, bar, k1, 0, 0);
                } else {
#pragma unroll
                    for (int r = 0; r < 32; r += 4)
                        if (r < N) tma_gather4(dst + r * 128, &p.tX, bar, k1, tok[r], tok[r + 1], tok[r + 2], tok[r + 3]);
                }
            }
            k += st.pair ? 128 : st.alt ? (i & 1) * 64 : 64;
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
        next[0] = s;
        next[1] = (int)ph;
        mbar_arrive(sm.b_turn + 8 * (who ^ 1));
    }
}

__device__ void few_mma(const FewArgs& p, const FewSmem& sm, const FewLists& L, uint32_t tmem,
                        volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    // weights MN-major: 64-column atoms 8192 bytes apart, K slices of 16 rows 2048 bytes apart;
    // tokens K-major: K slices 32 bytes apart
    const uint64_t wd0 = smem_desc_sw128(sm.ring, 8192, 1024);
    const uint64_t bd0 = smem_desc_sw128(sm.ring + FEW_TILE_BYTES, 16, 1024);
    int s = 0, n = 0;
    uint32_t ph = 0;
    bool issued = false;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x, ++n) {
        const FewItem it = few_item(p, L, id);
        // down: hi and lo pieces of the tokens side by side, added by the epilogue
        const int N = up16(it.cnt), acc = n & 1;
        const uint32_t idesc = idesc_bf16_f32(128, (it.up ? 1 : 2) * N, true, false);
        const FewSteps st = few_steps(p, it);
        const uint32_t bd2 = st.pair ? ((it.up ? 1 : 2) * N * 128) >> 4 : 0, dd2 = st.two ? p.nb : 0;
        if (!mbar_wait(sm.tempty + 8 * acc, ((uint32_t)(n >> 1) & 1u) ^ 1u, p.limit_ns, abort_flag)) {
            few_abort(abort_flag, p.status, SITE_FEW_WAIT_TEMPTY, id);
            break;
        }
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(acc * p.acc_cols);
        bool ok = true;
        for (int i = 0; i < st.n; ++i) {
            if (!mbar_wait(sm.full + 8 * s, ph, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_FULL, id);
                ok = false;
                break;
            }
            // gate columns into 0 .., up columns into nb ..
            const uint64_t wd = wd0 + (uint64_t)((s * sm.stage_bytes) >> 4);
            const uint64_t bd = bd0 + (uint64_t)((s * sm.stage_bytes) >> 4);
            const uint32_t d0 = d + (st.alt & i ? p.nb : 0), add = i > st.alt ? 1u : 0u;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                tc_mma_bf16(d0, wd + q * (2048 >> 4), bd + q * (32 >> 4), idesc, add | (q != 0 ? 1u : 0u));
            if (!st.wide && (i + 1 < st.n ? st.half2 : st.last2)) {
                const uint32_t add2 = add | (uint32_t)st.pair;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    tc_mma_bf16(d + dd2, wd + ((8192 + q * 2048) >> 4), bd + bd2 + q * (32 >> 4), idesc,
                                add2 | (q != 0 ? 1u : 0u));
            }
            issued = true;
            tc_commit(sm.empty + 8 * s);
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
        if (!ok) break;
        tc_commit(sm.tfull + 8 * acc);
    }
    if (issued) {   // every tcgen05.mma is complete before TMEM is released
        tc_commit(sm.drain);
        if (!mbar_wait(sm.drain, 0, p.limit_ns, nullptr))
            report(p.status, MOEVIE_ERR_TIMEOUT, SITE_FEW_DRAIN, (int)blockIdx.x, 0);
    }
}

// y of the tokens: a warp per token and column tile of the down items (two tokens where tiles have
// 64 columns), the same share for every warp of the grid, each when its tile's last part has been
// counted.  Slots in order, a slot's parts in order.  A lane holds the index and the weight of one
// row; four columns each.  (Summed by whoever came last, a tile of 32 tokens was eight tokens' loads
// one after the other in one warp, while the rest of the grid had finished: 6 us at the end of 64
// tokens of 8 slots.)
__device__ void few_combine(const FewArgs& p, const FewLists& L, const FewPlan& pl, volatile int* abort_flag) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int width = pl.tw2 == 128 ? 32 : 16, sub = lane & (width - 1), half = lane != sub;
    const int per = 32 / width, nr = p.k * pl.P2, na = nr + (p.hs > 0 ? pl.P2s : 0), slots = p.T * p.k;
    for (int u = warp * gridDim.x + blockIdx.x; u < (p.T + per - 1) / per * pl.ntd; u += gridDim.x * FEW_EPI_WARPS) {
        const int tp = few_div(u, pl.ntd, pl.inv_ntd), dt = u - tp * pl.ntd, t = tp * per + half;
        const int cc = dt * pl.tw2 + sub * 4;   // d is a multiple of 8
        const bool in = t < p.T && cc < p.d;
        uint64_t t0 = 0;
        for (uint32_t i = 1;; ++i) {
            const bool done = sub != 0 || t >= p.T || ld_acquire(p.y_cnt + t * pl.ntd + dt) >= na;
            if (__all_sync(0xffffffffu, done)) break;
            __nanosleep(100);
            if ((i & 63u) != 0u) continue;
            const uint64_t now = globaltimer_ns();
            if (t0 == 0) t0 = now;
            if (__any_sync(0xffffffffu, now - t0 > p.limit_ns || *abort_flag)) {
                if (lane == 0) few_abort(abort_flag, p.status, SITE_FEW_WAIT_Y, u);
                return;
            }
        }
        __syncwarp();   // what one lane has acquired, all lanes may read (a vote does not order memory)
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r0 = 0; r0 < na; r0 += width) {
            const int r = r0 + sub;
            int row = 0;
            float g = 0.f;
            if (t < p.T && r < nr) {
                const int j = few_div(r, pl.P2, pl.inv_P2), q = t * p.k + j;
                row = (r - j * pl.P2) * slots + L.row_of[q];
                g = L.gate[q];
            } else if (t < p.T && r < na) {
                row = pl.P2 * slots + (r - nr) * p.T + t;
                g = p.lambda;
            }
            for (int i0 = 0; i0 < width && r0 + i0 < na; i0 += 8) {
                float4 a[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {   // eight rows' loads in flight
                    const int at = __shfl_sync(0xffffffffu, row, i0 + i, width);
                    a[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (in && r0 + i0 + i < na)
                        a[i] = __ldcg(reinterpret_cast<const float4*>(p.y_part + (int64_t)at * p.d + cc));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float gi = __shfl_sync(0xffffffffu, g, i0 + i, width);
                    if (r0 + i0 + i >= na) break;
                    y.x = fmaf(gi, a[i].x, y.x);
                    y.y = fmaf(gi, a[i].y, y.y);
                    y.z = fmaf(gi, a[i].z, y.z);
                    y.w = fmaf(gi, a[i].w, y.w);
                }
            }
        }
        if (in) {
            uint2 o;
            o.x = pack_bf16x2(y.x, y.y);
            o.y = pack_bf16x2(y.z, y.w);
            *reinterpret_cast<uint2*>(p.y + (int64_t)t * p.d + cc) = o;
        }
    }
}

// Two groups of four warps take the CTA's items in turn (accumulator = group), so that the trips
// to L2 of one item's bookkeeping overlap the next item's.  Warp w of a group reads TMEM lanes
// 32 w .. (its columns of W) for all tokens.  One thread waits and decides for its group, so
// that the warps take the same way through its barriers.
__device__ void few_epilogue(const FewArgs& p, const FewSmem& sm, const FewLists& L, uint32_t tmem,
                             volatile int* abort_flag, volatile int* flags) {
    const int group = threadIdx.x >> 7, tid = threadIdx.x & 127, warp = tid >> 5, lane = tid & 31;
    const FewPlan pl = *L.plan;
    const bool two = p.W3 != nullptr;
    const int64_t slots = (int64_t)p.T * p.k;
    const uint32_t tb = tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)(group * p.acc_cols);
    int n = 0;
    for (int id = blockIdx.x + group * gridDim.x; id < pl.n_items; id += 2 * gridDim.x, ++n) {
        const FewItem it = few_item(p, L, id);
        if (tid == 0) {
            const bool ok = mbar_wait(sm.tfull + 8 * group, (uint32_t)n & 1u, p.limit_ns, abort_flag);
            if (!ok) few_abort(abort_flag, p.status, SITE_FEW_WAIT_TFULL, id);
            flags[group] = ok;
        }
        epi_sync(group);
        if (!flags[group]) return;
        tc_fence_after();
        const int c = tid, N = up16(it.cnt);
        const bool active = 32 * warp < it.tw;
        if (it.up) {
            const int col = it.n0 + c, h = it.shared ? p.hs : p.h, ld = it.shared ? p.ldhs : p.ldh;
            const bool ok = c < it.tw && col < h;
            __nv_bfloat16* hi = (it.shared ? p.Hs : p.H) + (int64_t)it.row0 * ld + col;
            __nv_bfloat16* lo = hi + (it.shared ? (int64_t)p.T : slots) * ld;
            // columns of D that are the entry's tokens, in the order of its rows
            uint32_t own = 0xffffffffu >> (32 - it.cnt);
            if (p.T <= 16 && !it.shared) {
                own = 0u;
                for (int j = 0; j < it.cnt; ++j) own |= 1u << L.row_tok[it.row0 + j];
            }
            for (int j0 = 0; j0 < 32 && (own >> j0) != 0u && active; j0 += 8) {
                uint32_t u[8], v[8];
                if ((own >> j0 & 0xffu) == 0u) continue;
                tmem_ld_32x32b_x8(tb + j0, u);
                if (two) tmem_ld_32x32b_x8(tb + p.nb + j0, v);
                tmem_wait_ld();
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(u[i]);
                if (two) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        f[i] = __fdividef(f[i], 1.0f + __expf(-f[i])) * __uint_as_float(v[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i += 2) gelu_erf2(f[i], f[i + 1]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok && (own >> (j0 + i) & 1u)) {   // two bf16 pieces: 16 significant bits
                        const int64_t r = __popc(own & ((1u << (j0 + i)) - 1u));
                        const __nv_bfloat16 a = __float2bfloat16_rn(f[i]);
                        hi[r * ld] = a;
                        lo[r * ld] = __float2bfloat16_rn(f[i] - __bfloat162float(a));
                    }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.tempty + 8 * group);
            fence_proxy_async_all();   // the rows will be read by TMA
            epi_sync(group);
            if (tid == 0) add_release(p.done_up + (it.shared ? p.na_max + it.i : it.i), 1);
        } else {
            // rows of the partial outputs: [P2][T k] routed, then [P2s][T] shared
            const int col = it.n0 + c;
            const bool ok = c < it.tw && col < p.d;
            float* yp = p.y_part + (it.shared ? (int64_t)pl.P2 * slots + (int64_t)it.part * p.T : (int64_t)it.part * slots) * p.d +
                        (int64_t)it.row0 * p.d + col;
            for (int j0 = 0; j0 < it.cnt && active; j0 += 8) {
                uint32_t u[8], v[8];
                tmem_ld_32x32b_x8(tb + j0, u);
                tmem_ld_32x32b_x8(tb + N + j0, v);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok && j0 + i < it.cnt)
                        yp[(int64_t)(j0 + i) * p.d] = __uint_as_float(u[i]) + __uint_as_float(v[i]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.tempty + 8 * group);
            epi_sync(group);
            const int dt = it.tw == 128 ? it.n0 >> 7 : it.n0 >> 6;
            if (tid < it.cnt)
                add_release(p.y_cnt + (it.shared ? it.row0 + tid : L.row_tok[it.row0 + tid]) * pl.ntd + dt, 1);
        }
    }
    few_combine(p, L, pl, abort_flag);
}

// ----------------------------------------------------------------- kernel

// Shared memory, from a 1024-byte boundary: ring, barriers and flags, lists.  The router
// stages use the ring's space before the ring is live.
struct FewSizes {
    int stage_bytes, stages, lists, total;
};
__host__ __device__ inline int few_nb(int T) { return T <= 16 ? 16 : 32; }
__host__ __device__ inline int few_entries(int T, int k, int E) {   // at most
    const int n = T * k;
    return (n < E ? n : E) + n / few_nb(T);
}
__host__ __device__ inline FewSizes few_sizes(int T, int k, int E) {
    FewSizes z;
    const int n = T * k, na = few_entries(T, k, E);
    z.stage_bytes = FEW_TILE_BYTES + FEW_TOKEN_BYTES;
    // plan, gate, row_of, act, off, cnt, row_tok
    z.lists = 128 + ((4 * n + 2 * n + 4 * na + na + n + 15) & ~15);
    const int left = FEW_SMEM_MAX - 1024 - FEW_BAR_BYTES - FEW_FLAG_BYTES - z.lists;
    z.stages = left / z.stage_bytes;
    if (z.stages > 12) z.stages = 12;
    z.total = 1024 + z.stages * z.stage_bytes + FEW_BAR_BYTES + FEW_FLAG_BYTES + z.lists;
    return z;
}

__global__ void __launch_bounds__(FEW_THREADS, 1) few_kernel(const __grid_constant__ FewArgs p) {
    extern __shared__ uint8_t few_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(few_smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    const FewSizes z = few_sizes(p.T, p.k, p.E);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + z.stages * z.stage_bytes);
    uint8_t* after = reinterpret_cast<uint8_t*>(bars) + FEW_BAR_BYTES;
    volatile int* flags = reinterpret_cast<volatile int*>(after);            // of the epilogue groups
    volatile int* abort_flag = flags + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(after) + 3;
    uint8_t* at = after + FEW_FLAG_BYTES;
    const int n = p.T * p.k, na = p.na_max;
    FewLists L;
    L.plan = reinterpret_cast<FewPlan*>(at);
    L.gate = reinterpret_cast<float*>(at + 128);
    L.row_of = reinterpret_cast<uint16_t*>(L.gate + n);
    L.act = L.row_of + n;
    L.off = L.act + na;
    L.cnt = reinterpret_cast<uint8_t*>(L.off + na);
    L.row_tok = L.cnt + na;
    FewSmem sm;
    sm.ring = smem_u32(smem);
    sm.stages = z.stages;
    sm.stage_bytes = z.stage_bytes;
    sm.full = smem_u32(bars);
    sm.empty = sm.full + 8 * 12;
    sm.tfull = sm.empty + 8 * 12;
    sm.tempty = sm.tfull + 16;
    sm.drain = sm.tempty + 16;
    sm.b_turn = sm.drain + 8;
    sm.b_next = flags + 4;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < z.stages; ++s) {
            mbar_init(sm.full + 8 * s, 2);    // weights, tokens
            mbar_init(sm.empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sm.tfull + 8 * a, 1);
            mbar_init(sm.tempty + 8 * a, FEW_EPI_WARPS / 2);
        }
        mbar_init(sm.drain, 1);
        mbar_init(sm.b_turn, 1);
        mbar_init(sm.b_turn + 8, 1);
        sm.b_next[0] = sm.b_next[1] = 0;
        *abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&p.tW1);
        tma_prefetch_desc(&p.tW2);
        tma_prefetch_desc(&p.tX);
        tma_prefetch_desc(&p.tH);
        if (p.W3) tma_prefetch_desc(&p.tW3);
        if (p.hs > 0) {
            tma_prefetch_desc(&p.tS1);
            tma_prefetch_desc(&p.tS2);
            tma_prefetch_desc(&p.tHs);
            if (p.W3) tma_prefetch_desc(&p.tS3);
        }
    }
    __syncwarp();
    if (warp == FEW_WARP_MMA) {
        tmem_alloc(smem_u32(tmem_slot), p.tmem_cols);
        tmem_relinquish();
    }
    auto give_up = [&]() {   // a grid barrier timed out (all threads): nothing but TMEM is held
        __syncthreads();
        if (warp == FEW_WARP_MMA) tmem_dealloc(*tmem_slot, p.tmem_cols);
    };
    pdl_wait();
    // counters of this call, used only after the grid barrier
    for (int i = blockIdx.x * FEW_THREADS + threadIdx.x; i < p.n_counters; i += gridDim.x * FEW_THREADS)
        p.done_up[i] = 0;
    few_logits(p, smem);
    const int sel_bytes = (p.E + 31) / 32 * 32 * FEW_SEL_BYTES, ring_bytes = z.stages * z.stage_bytes;
    // (then the selection and the masks lie behind the tokens' selection buffers)
    const bool everywhere = p.T <= FEW_SEL_WARPS && p.T * sel_bytes + 10 * p.E + 8 * n + 16 <= ring_bytes;
    unsigned long long* mask = reinterpret_cast<unsigned long long*>(smem + (everywhere ? p.T * sel_bytes : 0));
    uint16_t* off = reinterpret_cast<uint16_t*>(mask + p.E);
    if (everywhere)
        for (int e = threadIdx.x; e < p.E; e += FEW_THREADS) mask[e] = 0ull;
    // tokens of this CTA: all, or every gridDim.x-th
    const int t0 = everywhere ? 0 : blockIdx.x, step = everywhere ? 1 : (int)gridDim.x;
    const int mine = everywhere ? p.T : (p.T - t0 + step - 1) / step;
    if (!few_barrier(p.status, p.limit_ns)) return give_up();
    if (everywhere) {
        int32_t* s_idx = reinterpret_cast<int32_t*>(off + ((p.E + 1) & ~1));
        float* s_gate = reinterpret_cast<float*>(s_idx + n);
        few_select(p, 0, 1, mine, smem, s_idx, s_gate, mask);
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i < n; i += FEW_THREADS) {
                p.idx[i] = s_idx[i];
                p.gate[i] = s_gate[i];
            }
        few_plan<true>(p, L, s_idx, s_gate, mask, off);
    } else {
        const int most = min(FEW_SEL_WARPS, ring_bytes / sel_bytes);   // (one batch, unless the GPU is tiny)
        for (int i = 0; i < mine; i += most) {
            few_select(p, t0 + i * step, step, min(most, mine - i), smem, p.idx, p.gate, nullptr);
        }
        if (!few_barrier(p.status, p.limit_ns)) return give_up();
        few_plan<false>(p, L, p.idx, p.gate, mask, off);
    }
    fence_proxy_async_smem();   // the router's use of the ring, before TMA writes to it
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (warp < FEW_EPI_WARPS) {
        few_epilogue(p, sm, L, tmem, abort_flag, flags);
    } else if (warp == FEW_WARP_W) {
        if (elect_one()) few_load_w(p, sm, L, abort_flag);
    } else if (warp == FEW_WARP_MMA) {
        if (elect_one()) few_mma(p, sm, L, tmem, abort_flag);
    } else {
        if (elect_one()) few_load_b(p, sm, L, warp - FEW_WARP_B, abort_flag);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == FEW_WARP_MMA) {
        settle_copies(abort_flag);
        tc_fence_after();
        tmem_dealloc(tmem, p.tmem_cols);
    }
}

inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }
inline int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }

// Router split: parts of d for blocks of 8 experts.
int few_rt_parts(int d, int E, int ctas) {
    const int eb = (E + 7) / 8;
    int p = ctas / eb;
    if (p > 8) p = 8;
    if (p > (d + 63) / 64) p = (d + 63) / 64;
    return p < 1 ? 1 : p;
}

struct FewLayout {
    size_t idx, gate, part, wsq, xsq, counters, H, Hs, y_part, total;
    int64_t n_done, n_y_cnt;
};
FewLayout few_layout(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t hs) {
    FewLayout L;
    size_t o = up256(sizeof(DevStatus));
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    const int64_t n = T * k, na = few_entries((int)T, (int)k, (int)E);
    L.idx = take(4 * n);
    L.gate = take(4 * n);
    L.part = take(4 * 8 * T * E);
    L.wsq = take(4 * 8 * E);
    L.xsq = take(4 * 8 * T);
    L.n_done = na + (T + few_nb((int)T) - 1) / few_nb((int)T);
    L.n_y_cnt = T * ((d + 63) / 64);   // at most: 64-column items
    L.counters = take(4 * (L.n_done + L.n_y_cnt));
    L.H = take(2 * 2 * n * up8(h));
    L.Hs = take(2 * 2 * T * up8(hs));
    L.y_part = take(4 * (FEW_MAX_P2 * n + (hs > 0 ? FEW_MAX_P2S * T : 0)) * d);
    L.total = o;
    return L;
}

}  // namespace

size_t few_workspace_bytes(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t hs) {
    return few_layout(T, d, E, k, h, hs).total;
}

cudaError_t launch_few(FewArgs a, uint8_t* ws, int sms, uint64_t limit_ns, cudaStream_t s) {
    const FewLayout L = few_layout(a.T, a.d, a.E, a.k, a.h, a.hs);
    const int n = a.T * a.k;
    if (!a.idx) a.idx = reinterpret_cast<int32_t*>(ws + L.idx);
    if (!a.gate) a.gate = reinterpret_cast<float*>(ws + L.gate);
    a.part = reinterpret_cast<float*>(ws + L.part);
    a.wsq = reinterpret_cast<float*>(ws + L.wsq);
    a.xsq = reinterpret_cast<float*>(ws + L.xsq);
    a.done_up = reinterpret_cast<int32_t*>(ws + L.counters);
    a.y_cnt = a.done_up + L.n_done;
    a.n_counters = (int)(L.n_done + L.n_y_cnt);
    a.H = reinterpret_cast<__nv_bfloat16*>(ws + L.H);
    a.Hs = reinterpret_cast<__nv_bfloat16*>(ws + L.Hs);
    a.y_part = reinterpret_cast<float*>(ws + L.y_part);
    a.status = reinterpret_cast<DevStatus*>(ws);
    a.limit_ns = limit_ns;
    a.ldh = (int)up8(a.h);
    a.ldhs = (int)up8(a.hs);
    a.na_max = few_entries(a.T, a.k, a.E);
    a.nb = few_nb(a.T);
    a.n_sh = a.hs > 0 ? (a.T + a.nb - 1) / a.nb : 0;
    a.nkb_d = (a.d + 63) / 64;
    a.nkb_h = (a.h + 63) / 64;
    a.nkb_hs = (a.hs + 63) / 64;
    a.acc_cols = 2 * a.nb;   // gate and up projections, or hi and lo pieces
    a.tmem_cols = 32;
    while (a.tmem_cols < 2 * a.acc_cols) a.tmem_cols *= 2;
    a.rt_eb = (a.E + 7) / 8;
    a.inv_k = 1.0f / (float)a.k;
    a.sh_ratio = (a.nkb_hs + a.nkb_h - 1) / a.nkb_h;
    a.rt_parts = few_rt_parts(a.d, a.E, sms);
    a.rt_dch = (int)up8((a.d + a.rt_parts - 1) / a.rt_parts);
    // length of the summation chains of a logit (few_logits): 8 products, their sums (one more per
    // staged block), the lanes, the warps, the parts; times 2^-24, with room for second order
    const int kp = a.rt_kp = FEW_WARPS / ((a.T + 7) / 8), blocks = (a.rt_dch + FEW_RT_K - 1) / FEW_RT_K;
    const int chain = 5 + (a.rt_dch / (64 * kp) + 2 * blocks) + 3 + kp + a.rt_parts;
    a.rt_err = 1.01f * (float)chain * 5.9604645e-8f;

    bool ok = make_weight_tmap_strided(&a.tW1, a.W1, a.h, a.d, a.E, a.hp, (int64_t)a.d * a.hp) &&
              make_weight_tmap_strided(&a.tW2, a.W2, a.d, a.h, a.E, a.d, (int64_t)a.h * a.d) &&
              (a.T <= 16 ? make_kmajor_tmap(&a.tX, a.x, a.d, a.T, 1, a.d, (int64_t)a.T * a.d, 16)
                         : make_gather_tmap(&a.tX, a.x, a.d, a.T, a.d)) &&
              make_kmajor_tmap(&a.tH, a.H, a.h, n, 2, a.ldh, (int64_t)n * a.ldh, 16);
    if (ok && a.W3) ok = make_weight_tmap_strided(&a.tW3, a.W3, a.h, a.d, a.E, a.hp, (int64_t)a.d * a.hp);
    if (ok && a.hs > 0) {
        ok = make_weight_tmap_strided(&a.tS1, a.Ws1, a.hs, a.d, 1, a.hsp, (int64_t)a.d * a.hsp) &&
             make_weight_tmap_strided(&a.tS2, a.Ws2, a.d, a.hs, 1, a.d, (int64_t)a.hs * a.d) &&
             make_kmajor_tmap(&a.tHs, a.Hs, a.hs, a.T, 2, a.ldhs, (int64_t)a.T * a.ldhs, 16);
        if (ok && a.W3) ok = make_weight_tmap_strided(&a.tS3, a.Ws3, a.hs, a.d, 1, a.hsp, (int64_t)a.d * a.hsp);
    }
    if (!ok) return cudaErrorInvalidValue;
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev].load(std::memory_order_acquire)) {   // idempotent: no lock needed
        const cudaError_t e = cudaFuncSetAttribute(few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM_MAX);
        if (e != cudaSuccess) return e;
        attr_set[dev].store(true, std::memory_order_release);
    }
    const FewSizes z = few_sizes(a.T, a.k, a.E);
    const cudaError_t e = launch_pdl_coop(few_kernel, dim3((unsigned)sms), dim3(FEW_THREADS), z.total, s, a);
    count_launches(1);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mv
