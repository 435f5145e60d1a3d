// few.cu -- the whole MoE FFN layer for a few tokens (T <= 64) in one kernel, sm_103a.
//
// With few tokens the layer of Eqs. 1 and 4-7 is a stream of weights: the router, then W1 (and
// W3) and W2 of the experts that some token selects, each byte read once.  One cooperative
// launch, one CTA per SM:
//
//   1. Router logits.  CTA (eb, ds) forms x . W_r for 8 experts and one part of d, in fp32, and
//      the parts' sums of squares of the router columns; grid barrier.
//   2. Selection, one warp per token: keys sigmoid(s) + b from the summed logits, k rounds of
//      arg-max, and a certificate: |error of s| <= n 2^-24 |x| |W_r[:, e]| (n: the length of the
//      summation chains, products of bf16 and fp32 being exact inside an FMA), so a selection
//      whose margin exceeds the key errors is the exact one.  Otherwise the experts near the
//      boundary get 64-bit logits and keys.  Up to FEW_SEL_WARPS tokens every CTA selects for
//      itself (no second barrier); above, the CTAs share the tokens out and meet again.
//   3. Expert products on tcgen05 with the weights as the M operand: D[128 columns of W, tokens]
//      = W^T . x^T.  W tiles go from HBM to shared memory by TMA as they lie (MN-major, 128-byte
//      swizzle) and no thread touches them again; the tokens of the expert (TMA row gather) are
//      the N operand, 16 to 64 columns, so the tensor cores do in passing what would otherwise
//      cost an unpack and an FMA per weight and token.  Items (expert, 128 columns, part of K)
//      are dealt to the CTAs round-robin, K split so that they come out even.
//   4. Up items: the last of an item's K parts to finish adds them in order, applies the
//      activation and stores it as two bf16 pieces (hi + lo, 16 bits) so that y is rounded to
//      bf16 once.  Down items wait for their expert's up items (a counter), while their weights
//      are already on the way: the weight loads run ahead of the wait by the whole ring.
//   5. Down items leave fp32 partial rows; whoever completes the last contribution to a token's
//      128 columns of y adds them up in slot order (no float atomics: results do not depend on
//      timing).
//
// Waits between CTAs rely on co-residency (cooperative launch) and on the item order: every
// CTA takes its up items before its down items, and up items wait for nothing.  All waits have
// time limits.
#include <math.h>

#include "internal.h"

namespace mv {

namespace {

constexpr int FEW_EPI_WARPS = 8;      // two per TMEM lane quadrant, alternate groups of 8 tokens
constexpr int FEW_WARP_W = 8;         // weight loads
constexpr int FEW_WARP_MMA = 9;
constexpr int FEW_WARP_B = 10;        // token / hidden loads
constexpr int FEW_WARPS = 12;
constexpr int FEW_THREADS = FEW_WARPS * 32;
constexpr int FEW_SEL_WARPS = 8;      // tokens that every CTA selects for itself
constexpr int FEW_TILE_BYTES = 128 * 64 * 2;   // 128 columns x 64 K rows of a weight matrix
constexpr int FEW_RT_K = 512;         // rows of W_r staged at a time
constexpr int FEW_RT_XLD = FEW_RT_K + 4;       // float row strides of the staged x and W_r^T
constexpr int FEW_RT_WLD = FEW_RT_K + 16;      //   (bank-conflict-free 16-byte reads)
constexpr int FEW_SMEM_MAX = 232448 - 256;   // 227 KB less the kernel's static variables
constexpr int FEW_BAR_BYTES = 512;
// Splits of K: at most FEW_MAX_P parts of an up item (FEW_MAX_PART items in all when split, the
// size of the partial buffer), FEW_MAX_P2 of a routed and FEW_MAX_P2S of a shared down item.
constexpr int FEW_MAX_P = 8, FEW_MAX_PART = 640, FEW_MAX_P2 = 4, FEW_MAX_P2S = 8;

__device__ __forceinline__ void epi_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ int ld_acquire(const int32_t* p) {
    int v;
    asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// 32 lanes x 8 consecutive 32-bit columns (thread i: lane base + i).
__device__ __forceinline__ void tmem_ld_32x32b_x8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ float act_gelu(float u) { return 0.5f * u * (1.0f + erff(u * 0.70710678118654752f)); }
__device__ __forceinline__ float act_silu(float u) { return u / (1.0f + expf(-u)); }

// ------------------------------------------------------------- 1. logits

// part[ds][t][e] and wsq[ds][e] of this CTA's blocks of 8 experts x parts of d.  smem: staged
// x [8 TG][FEW_RT_XLD], W_r^T [8][FEW_RT_WLD], then the per-warp sums.
__device__ void few_logits(const FewArgs& p, float* smem) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int TG = (p.T + 7) / 8, KP = FEW_WARPS / TG;
    float* xs = smem;
    float* ws = xs + 8 * TG * FEW_RT_XLD;
    float* red = ws + 8 * FEW_RT_WLD;      // [KP][8 TG][8]
    float* redq = red + FEW_WARPS * 64;    // [KP][8]
    const int g = warp % TG, kp = warp / TG, e8 = lane >> 2, ks = lane & 3;
    for (int item = blockIdx.x; item < p.rt_eb * p.rt_parts; item += gridDim.x) {
        const int e0 = item % p.rt_eb * 8, ds = item / p.rt_eb;
        const int d0 = ds * p.rt_dch, d1 = min(p.d, d0 + p.rt_dch);
        float acc2[8] = {}, sq = 0.f;
        for (int k0 = d0; k0 < d1; k0 += FEW_RT_K) {
            const int kc = min(FEW_RT_K, d1 - k0), kcp = (kc + 15) & ~15;
            for (int q = threadIdx.x; q < kcp * 8; q += FEW_THREADS) {
                const int r = q >> 3, e = q & 7;
                ws[e * FEW_RT_WLD + r] =
                    (r < kc && e0 + e < p.E) ? __ldg(p.W_r + (int64_t)(k0 + r) * p.E + e0 + e) : 0.f;
            }
            const int n8 = kcp / 8;   // kc is a multiple of 8, as d and the parts are
            for (int q = threadIdx.x; q < p.T * n8; q += FEW_THREADS) {
                const int t = q / n8, c = (q - t * n8) * 8;
                float v[8] = {};
                if (c < kc) unpack_bf16x8(__ldg(reinterpret_cast<const uint4*>(p.x + (int64_t)t * p.d + k0 + c)), v);
                float4* o = reinterpret_cast<float4*>(xs + t * FEW_RT_XLD + c);
                o[0] = make_float4(v[0], v[1], v[2], v[3]);
                o[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
            __syncthreads();
            if (kp < KP) {
                float acc[8] = {};
                const int nit = kcp / 16;
                int n = 0;
                for (int it = kp; it < nit; it += KP) {
                    const int k = it * 16 + ks * 4;
                    const float4 w = *reinterpret_cast<const float4*>(ws + e8 * FEW_RT_WLD + k);
                    sq = fmaf(w.x, w.x, fmaf(w.y, w.y, fmaf(w.z, w.z, fmaf(w.w, w.w, sq))));
#pragma unroll
                    for (int i = 0; i < 8; ++i) {   // (rows past T hold no token: their sums are dropped)
                        const float4 x = *reinterpret_cast<const float4*>(xs + (8 * g + i) * FEW_RT_XLD + k);
                        acc[i] = fmaf(x.w, w.w, fmaf(x.z, w.z, fmaf(x.y, w.y, fmaf(x.x, w.x, acc[i]))));
                    }
                    if ((++n & 3) == 0) {   // short chains: 16 products, then their sums
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            acc2[i] += acc[i];
                            acc[i] = 0.f;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) acc2[i] += acc[i];
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc2[i] += __shfl_xor_sync(0xffffffffu, acc2[i], 1);
            acc2[i] += __shfl_xor_sync(0xffffffffu, acc2[i], 2);
        }
        sq += __shfl_xor_sync(0xffffffffu, sq, 1);
        sq += __shfl_xor_sync(0xffffffffu, sq, 2);
        if (kp < KP && ks == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) red[(kp * 8 * TG + 8 * g + i) * 8 + e8] = acc2[i];
            if (g == 0) redq[kp * 8 + e8] = sq;
        }
        __syncthreads();
        for (int q = threadIdx.x; q < (p.T + 1) * 8; q += FEW_THREADS) {
            const int t = q >> 3, e = q & 7;
            if (e0 + e >= p.E) continue;
            float s = 0.f;
            if (t < p.T) {
                for (int j = 0; j < KP; ++j) s += red[(j * 8 * TG + t) * 8 + e];
                p.part[((int64_t)ds * p.T + t) * p.E + e0 + e] = s;
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
__device__ __forceinline__ float warp_min(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fminf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// x_t . W_r[:, e] in 64 bits, by one warp (every lane gets the sum).
__device__ double few_exact_logit(const FewArgs& p, int t, int e) {
    const int lane = threadIdx.x & 31;
    double s = 0.0;
#pragma unroll 4
    for (int i = lane; i < p.d; i += 32)
        s = fma((double)__bfloat162float(p.x[(int64_t)t * p.d + i]), (double)__ldg(p.W_r + (int64_t)i * p.E + e), s);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// Selection and gates of token t by one warp.  buf: 24 bytes per expert (E rounded up to 32).
// Lane l holds experts l, l + 32, ...; bit q of its masks stands for expert 32 q + l.
__device__ void few_select(const FewArgs& p, int t, uint8_t* buf, int32_t* out_idx, float* out_gate) {
    const int lane = threadIdx.x & 31, NQ = (p.E + 31) / 32, Ep = NQ * 32;
    double* kd = reinterpret_cast<double*>(buf);
    float* key = reinterpret_cast<float*>(kd + Ep);
    float* lg = key + Ep;
    float* er = lg + Ep;
    const __nv_bfloat16* x = p.x + (int64_t)t * p.d;
    float x2 = 0.f;
    for (int c = lane; c < p.d / 8; c += 32) {
        float v[8];
        unpack_bf16x8(__ldg(reinterpret_cast<const uint4*>(x) + c), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) x2 = fmaf(v[i], v[i], x2);
    }
    const float xn = sqrtf(warp_sum(x2)) * p.rt_err;
    uint32_t have = 0, sel = 0;
    for (int q = 0; q < NQ; ++q) {
        const int e = q * 32 + lane;
        if (e >= p.E) break;
        have |= 1u << q;
        float s = 0.f, w2 = 0.f;
        for (int j = 0; j < p.rt_parts; ++j) {
            s += __ldcg(p.part + ((int64_t)j * p.T + t) * p.E + e);
            w2 += __ldcg(p.wsq + j * p.E + e);
        }
        const float v = 1.0f / (1.0f + expf(-s)) + __ldg(p.b + e);
        lg[e] = s;
        key[e] = v;
        // a quarter of the logit's error (the sigmoid's largest slope) and the fp32 evaluation
        er[e] = 0.25f * xn * sqrtf(w2) + 1e-6f * (1.0f + fabsf(v));
    }
    auto lane_best = [&](uint32_t& bu, int& be) {
        bu = 0u;
        be = 0x7fffffff;
        for (int q = 0; q < NQ; ++q)
            if ((have & ~sel) >> q & 1u) {
                const uint32_t u = key_order(key[q * 32 + lane]);
                if (u > bu) {
                    bu = u;
                    be = q * 32 + lane;
                }
            }
    };
    uint32_t bu;
    int be;
    lane_best(bu, be);
    for (int j = 0; j < p.k; ++j) {
        const uint32_t mu = __reduce_max_sync(0xffffffffu, bu);
        const int me = __reduce_min_sync(0xffffffffu, bu == mu ? be : 0x7fffffff);
        if (me == be) {
            sel |= 1u << (be >> 5);
            lane_best(bu, be);
        }
    }
    if (p.k < p.E) {
        float lo = INFINITY, hi = -INFINITY;   // lowest selected, highest unselected key bounds
        for (int q = 0; q < NQ; ++q) {
            if (!(have >> q & 1u)) continue;
            const float v = key[q * 32 + lane], r = er[q * 32 + lane];
            if (sel >> q & 1u) lo = (v - r == v - r) ? fminf(lo, v - r) : -INFINITY;
            else hi = (v + r == v + r) ? fmaxf(hi, v + r) : INFINITY;
        }
        lo = warp_min(lo);
        hi = warp_max(hi);
        if (!(lo > hi)) {
            // Surely in: the lower bound is above every unselected upper bound; surely out: the
            // upper bound is below every selected lower bound.  The rest get exact keys.
            uint32_t cand = 0;
            for (int q = 0; q < NQ; ++q) {
                if (!(have >> q & 1u)) continue;
                const float v = key[q * 32 + lane], r = er[q * 32 + lane];
                if ((sel >> q & 1u) ? !(v - r > hi) : !(v + r < lo)) cand |= 1u << q;
            }
            for (int q = 0; q < NQ; ++q) {
                uint32_t who = __ballot_sync(0xffffffffu, cand >> q & 1u);
                while (who) {
                    const int l = __ffs(who) - 1;
                    who &= who - 1;
                    const double s = few_exact_logit(p, t, q * 32 + l);
                    if (lane == l) kd[q * 32 + l] = 1.0 / (1.0 + exp(-s)) + (double)__ldg(p.b + q * 32 + l);
                }
            }
            sel &= ~cand;
            int need = p.k - (int)__reduce_add_sync(0xffffffffu, (unsigned)__popc(sel));
            for (; need > 0; --need) {
                double bv = 0.0;
                int b = 0x7fffffff;
                // better: a number before NaN, the larger key, the lower id
                auto better = [](double v, int e, double w, int f) {
                    if (f == 0x7fffffff) return e != 0x7fffffff;
                    if (e == 0x7fffffff) return false;
                    if (isnan(v) != isnan(w)) return (bool)isnan(w);
                    return v > w || (!(w > v) && e < f);
                };
                for (int q = 0; q < NQ; ++q)
                    if ((cand & ~sel) >> q & 1u) {
                        const int e = q * 32 + lane;
                        if (better(kd[e], e, bv, b)) {
                            bv = kd[e];
                            b = e;
                        }
                    }
                const int mine = b;
                for (int o = 16; o; o >>= 1) {
                    const double ov = __shfl_xor_sync(0xffffffffu, bv, o);
                    const int oe = __shfl_xor_sync(0xffffffffu, b, o);
                    if (better(ov, oe, bv, b)) {
                        bv = ov;
                        b = oe;
                    }
                }
                if (mine == b && b != 0x7fffffff) sel |= 1u << (b >> 5);
            }
        }
    }
    float mys = 0.f;
    for (int q = 0; q < NQ; ++q)
        if (sel >> q & 1u) mys += 1.0f / (1.0f + expf(-lg[q * 32 + lane]));
    const float sum = warp_sum(mys);
    int base = 0;
    for (int q = 0; q < NQ; ++q) {
        const bool s = sel >> q & 1u;
        const uint32_t m = __ballot_sync(0xffffffffu, s);
        if (s) {
            const int j = base + __popc(m & ((1u << lane) - 1u));
            out_idx[j] = q * 32 + lane;
            out_gate[j] = 1.0f / (1.0f + expf(-lg[q * 32 + lane])) / sum;
        }
        base += __popc(m);
    }
}

// ----------------------------------------------------- 3. work of a call

// Built by every CTA from the selection; kept in shared memory.
struct FewPlan {
    int n_act;             // experts with tokens
    int P, P2, P2s;        // splits of K: up items, routed and shared down items
    int n_up, n_items;     // items: up, then down
    int n_shared_down;
};

struct FewItem {
    int up, shared, i, e;  // i: active expert index
    int n0, kb0, kb1;
    int tile, part;        // up: index of (expert, columns) and K part; down: K part
    int cnt, row0;         // tokens of the expert, first row
};

struct FewLists {          // shared memory
    FewPlan* plan;
    uint16_t* act;         // [na] expert of active index i
    uint16_t* off;         // [na] its first row
    uint8_t* cnt;          // [na] its tokens
    uint8_t* row_tok;      // [T k] token of a row
    uint16_t* row_of;      // [T k] row of slot t k + j
    float* gate;           // [T k]
};

__device__ __forceinline__ FewItem few_item(const FewArgs& p, const FewLists& L, int id) {
    const FewPlan& pl = *L.plan;
    FewItem it;
    it.up = id < pl.n_up;
    if (it.up) {
        it.tile = id / pl.P;
        it.part = id - it.tile * pl.P;
        it.shared = it.tile < p.nt_s;
        const int q = it.tile - p.nt_s;
        it.i = it.shared ? 0 : q / p.nt;
        it.n0 = (it.shared ? it.tile : q - it.i * p.nt) * 128;
        it.kb0 = it.part * p.nkb_d / pl.P;
        it.kb1 = (it.part + 1) * p.nkb_d / pl.P;
    } else {
        int q = id - pl.n_up;
        it.shared = q < pl.n_shared_down;
        if (!it.shared) q -= pl.n_shared_down;
        const int P = it.shared ? pl.P2s : pl.P2, nkb = it.shared ? p.nkb_hs : p.nkb_h;
        it.part = q % P;
        q /= P;
        it.i = it.shared ? 0 : q / p.ntd;
        it.n0 = (it.shared ? q : q - it.i * p.ntd) * 128;
        it.tile = 0;
        it.kb0 = it.part * nkb / P;
        it.kb1 = (it.part + 1) * nkb / P;
    }
    it.e = it.shared ? 0 : L.act[it.i];
    it.cnt = it.shared ? p.T : L.cnt[it.i];
    it.row0 = it.shared ? 0 : L.off[it.i];
    return it;
}

// Splits of K: the P for which ceil(items P / CTAs) rounds of ceil(nkb / P) blocks (and one
// block's worth of start and finish) are shortest.
__device__ int few_choose_split(int items, int nkb, int ctas, int most, int most_items) {
    int best = 1, cost = 0x7fffffff;
    for (int P = 1; P <= most && P <= nkb; ++P) {
        if (P > 1 && items * P > most_items) break;
        const int c = (items * P + ctas - 1) / ctas * ((nkb + P - 1) / P + 1);
        if (c < cost) {
            cost = c;
            best = P;
        }
    }
    return best;
}

// Expert lists and the plan from the selection (idx, gate of all slots).  tmp: 10 bytes per
// expert of scratch.  The selection lies in shared memory, or in global memory where other CTAs
// wrote it.
template <bool SHARED_SEL>
__device__ void few_plan(const FewArgs& p, const FewLists& L, const int32_t* idx, const float* gate,
                         uint8_t* tmp) {
    unsigned long long* mask = reinterpret_cast<unsigned long long*>(tmp);   // tokens of each expert
    uint16_t* off = reinterpret_cast<uint16_t*>(mask + p.E);                 // first row of each expert
    auto load = [](const auto* q) { return SHARED_SEL ? *q : __ldcg(q); };
    const int n = p.T * p.k;
    for (int e = threadIdx.x; e < p.E; e += FEW_THREADS) mask[e] = 0ull;
    __syncthreads();
    for (int s = threadIdx.x; s < n; s += FEW_THREADS) atomicOr(&mask[load(idx + s)], 1ull << (s / p.k));
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int na = 0, rows = 0;
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            const int e = e0 + lane;
            const int c = e < p.E ? __popcll(mask[e]) : 0;
            int sum = c;   // inclusive prefix over the lanes
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            const uint32_t m = __ballot_sync(0xffffffffu, c > 0);
            if (c > 0) {
                const int i = na + __popc(m & ((1u << lane) - 1u));
                L.act[i] = (uint16_t)e;
                L.off[i] = (uint16_t)(rows + sum - c);
                L.cnt[i] = (uint8_t)c;
                off[e] = (uint16_t)(rows + sum - c);
            }
            na += __popc(m);
            rows += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) {
            FewPlan& pl = *L.plan;
            const int ctas = (int)gridDim.x;
            pl.n_act = na;
            const int tiles = na * p.nt + p.nt_s;
            pl.P = few_choose_split(tiles, p.nkb_d, ctas, FEW_MAX_P, FEW_MAX_PART);
            pl.P2 = few_choose_split(na * p.ntd + (p.hs > 0 ? p.ntd * ((p.nkb_hs + p.nkb_h - 1) / p.nkb_h) : 0),
                                     p.nkb_h, ctas, FEW_MAX_P2, 0x7fffffff);
            pl.P2s = 1;   // shared down items about as long as the routed ones
            if (p.hs > 0) pl.P2s = min(min(FEW_MAX_P2S, p.nkb_hs), max(1, (p.nkb_hs * pl.P2 + p.nkb_h / 2) / p.nkb_h));
            pl.n_up = tiles * pl.P;
            pl.n_shared_down = p.hs > 0 ? p.ntd * pl.P2s : 0;
            pl.n_items = pl.n_up + pl.n_shared_down + na * p.ntd * pl.P2;
        }
    }
    __syncthreads();
    for (int s = threadIdx.x; s < n; s += FEW_THREADS) {
        const int t = s / p.k, e = load(idx + s);
        const int row = off[e] + __popcll(mask[e] & ((1ull << t) - 1ull));
        L.row_tok[row] = (uint8_t)t;
        L.row_of[s] = (uint16_t)row;
        L.gate[s] = load(gate + s);
    }
}

// -------------------------------------------------------------- 4. roles

struct FewSmem {
    uint32_t ring, full, empty, tfull, tempty, drain;
    int stages, stage_bytes, b_off, lo_off;   // within a stage: B (hi) and B lo
};

__device__ __forceinline__ void few_abort(volatile int* flag, DevStatus* st, int site, int a) {
    *flag = 1;
    report(st, MOEVIE_ERR_TIMEOUT, site, (int)blockIdx.x, a);
}

__device__ __forceinline__ int up16(int v) { return (v + 15) & ~15; }

// Weight tiles of every item; never waits for anything but a free stage.
__device__ void few_load_w(const FewArgs& p, const FewSmem& sm, const FewLists& L, volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    int s = 0;
    uint32_t ph = 0;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x) {
        const FewItem it = few_item(p, L, id);
        const bool two = it.up && p.W3;
        const CUtensorMap* a = it.up ? (it.shared ? &p.tS1 : &p.tW1) : (it.shared ? &p.tS2 : &p.tW2);
        const CUtensorMap* a3 = it.shared ? &p.tS3 : &p.tW3;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
            if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_EMPTY, id);
                return;
            }
            const uint32_t bar = sm.full + 8 * s, dst = sm.ring + s * sm.stage_bytes;
            mbar_arrive_expect_tx(bar, two ? 2 * FEW_TILE_BYTES : FEW_TILE_BYTES);
#pragma unroll
            for (int j = 0; j < 2; ++j)
                tma_load_3d(dst + j * (FEW_TILE_BYTES / 2), a, bar, it.n0 + 64 * j, kb * 64, it.e);
            if (two)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    tma_load_3d(dst + FEW_TILE_BYTES + j * (FEW_TILE_BYTES / 2), a3, bar, it.n0 + 64 * j, kb * 64, it.e);
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

// The N operand: token rows (up) or the two pieces of the hidden rows (down), after the
// expert's up items are done.  Rows past the expert's last token repeat its first (up) or hold
// whatever follows (down): their columns of D are not read.
__device__ void few_load_b(const FewArgs& p, const FewSmem& sm, const FewLists& L, volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    int s = 0;
    uint32_t ph = 0;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x) {
        const FewItem it = few_item(p, L, id);
        const int N = up16(it.cnt);
        if (!it.up) {
            const int32_t* c = p.done_up + (it.shared ? p.na_max : it.i);
            const int want = it.shared ? p.nt_s : p.nt;
            const uint64_t t0 = globaltimer_ns();
            for (uint32_t i = 1; ld_acquire(c) < want; ++i)
                if ((i & 63u) == 0u && (*abort_flag || globaltimer_ns() - t0 > p.limit_ns)) {
                    few_abort(abort_flag, p.status, SITE_FEW_WAIT_UP, id);
                    return;
                }
            fence_proxy_async_all();   // the hidden rows were written by ordinary stores
        }
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
            if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_EMPTY, -id);
                return;
            }
            const uint32_t bar = sm.full + 8 * s, dst = sm.ring + s * sm.stage_bytes + sm.b_off;
            mbar_arrive_expect_tx(bar, (it.up ? 1 : 2) * N * 128);
            if (it.up) {
                for (int r = 0; r < N; r += 4) {
                    int tok[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = r + i < it.cnt ? r + i : 0;
                        tok[i] = it.shared ? j : L.row_tok[it.row0 + j];
                    }
                    tma_gather4(dst + r * 128, &p.tX, bar, kb * 64, tok[0], tok[1], tok[2], tok[3]);
                }
            } else {
                const CUtensorMap* h = it.shared ? &p.tHs : &p.tH;
                for (int r = 0; r < N; r += 16) {
                    tma_load_3d(dst + r * 128, h, bar, kb * 64, it.row0 + r, 0);
                    tma_load_3d(dst + sm.lo_off + r * 128, h, bar, kb * 64, it.row0 + r, 1);
                }
            }
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

__device__ void few_mma(const FewArgs& p, const FewSmem& sm, const FewLists& L, uint32_t tmem,
                        volatile int* abort_flag) {
    const int n_items = L.plan->n_items;
    // weights MN-major: 64-column atoms 8192 bytes apart, K slices of 16 rows 2048 bytes apart;
    // tokens K-major: K slices 32 bytes apart
    const uint64_t wd0 = smem_desc_sw128(sm.ring, 8192, 1024);
    const uint64_t bd0 = smem_desc_sw128(sm.ring + sm.b_off, 16, 1024);
    int s = 0, n = 0;
    uint32_t ph = 0;
    bool issued = false;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x, ++n) {
        const FewItem it = few_item(p, L, id);
        const uint32_t idesc = idesc_bf16_f32(128, up16(it.cnt), true, false);
        const int acc = n & 1;
        const bool two = it.up && p.W3;
        if (!mbar_wait(sm.tempty + 8 * acc, ((uint32_t)(n >> 1) & 1u) ^ 1u, p.limit_ns, abort_flag)) {
            few_abort(abort_flag, p.status, SITE_FEW_WAIT_TEMPTY, id);
            break;
        }
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(acc * p.acc_cols);
        bool ok = true;
        for (int kb = it.kb0; kb < it.kb1; ++kb) {
            if (!mbar_wait(sm.full + 8 * s, ph, p.limit_ns, abort_flag)) {
                few_abort(abort_flag, p.status, SITE_FEW_WAIT_FULL, id);
                ok = false;
                break;
            }
            const uint64_t wd = wd0 + (uint64_t)((s * sm.stage_bytes) >> 4);
            const uint64_t bd = bd0 + (uint64_t)((s * sm.stage_bytes) >> 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t add = (kb != it.kb0 || q != 0) ? 1u : 0u;
                tc_mma_bf16(d, wd + q * (2048 >> 4), bd + q * (32 >> 4), idesc, add);
                if (two)
                    tc_mma_bf16(d + p.nb, wd + (FEW_TILE_BYTES >> 4) + q * (2048 >> 4), bd + q * (32 >> 4), idesc, add);
                else if (!it.up)
                    tc_mma_bf16(d, wd + q * (2048 >> 4), bd + (uint64_t)(sm.lo_off >> 4) + q * (32 >> 4), idesc, 1u);
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

// hi and lo pieces of one hidden activation.
__device__ __forceinline__ void store_hidden(const FewArgs& p, const FewItem& it, int j, int col, float a) {
    const int ld = it.shared ? p.ldhs : p.ldh;
    __nv_bfloat16* H = it.shared ? p.Hs : p.H;
    const int64_t rows = it.shared ? p.T : (int64_t)p.T * p.k;
    const int64_t at = (int64_t)(it.row0 + j) * ld + col;
    const __nv_bfloat16 hi = __float2bfloat16_rn(a);
    H[at] = hi;
    H[rows * ld + at] = __float2bfloat16_rn(a - __bfloat162float(hi));
}

// Eight warps: warp w reads TMEM lanes 32 (w % 4) .. (its columns of W) and the token groups
// of 8 w / 4, w / 4 + 2, ...  One thread waits and decides for all, so that the warps take
// the same way through the barriers below.
__device__ void few_epilogue(const FewArgs& p, const FewSmem& sm, const FewLists& L, uint32_t tmem,
                             volatile int* abort_flag, volatile int* flags) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int quad = warp & 3, half = warp >> 2, c = quad * 32 + lane;
    const int n_items = L.plan->n_items, P = L.plan->P;
    const int mats = p.W3 ? 2 : 1;
    int n = 0;
    for (int id = blockIdx.x; id < n_items; id += gridDim.x, ++n) {
        const FewItem it = few_item(p, L, id);
        const int acc = n & 1;
        if (tid == 0) {
            const bool ok = mbar_wait(sm.tfull + 8 * acc, (uint32_t)(n >> 1) & 1u, p.limit_ns, abort_flag);
            if (!ok) few_abort(abort_flag, p.status, SITE_FEW_WAIT_TFULL, id);
            flags[64] = ok;
        }
        epi_sync();
        if (!flags[64]) return;
        tc_fence_after();
        const uint32_t tb = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * p.acc_cols);
        const int groups = (it.cnt + 7) / 8;
        if (it.up) {
            const int h = it.shared ? p.hs : p.h, col = it.n0 + c;
            float* part = P > 1 ? p.up_part + (int64_t)(it.tile * P + it.part) * mats * p.nb * 128 : nullptr;
            for (int g = half; g < groups; g += 2) {
                uint32_t u[8], v[8];
                tmem_ld_32x32b_x8(tb + 8 * g, u);
                if (mats == 2) tmem_ld_32x32b_x8(tb + p.nb + 8 * g, v);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int j = 8 * g + i;
                    if (j >= it.cnt) break;
                    if (part) {
                        part[j * 128 + c] = __uint_as_float(u[i]);
                        if (mats == 2) part[(p.nb + j) * 128 + c] = __uint_as_float(v[i]);
                    } else if (col < h) {
                        const float f = __uint_as_float(u[i]);
                        store_hidden(p, it, j, col, mats == 2 ? act_silu(f) * __uint_as_float(v[i]) : act_gelu(f));
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.tempty + 8 * acc);
            fence_proxy_async_all();
            __threadfence();
            epi_sync();
            int32_t* done = p.done_up + (it.shared ? p.na_max : it.i);
            if (!part) {
                if (tid == 0) atomicAdd(done, 1);
                continue;
            }
            if (tid == 0) flags[65] = atomicAdd(p.up_cnt + it.tile, 1) == P - 1;
            epi_sync();
            if (!flags[65]) continue;
            __threadfence();   // the other parts' stores, before they are read
            const float* all = p.up_part + (int64_t)it.tile * P * mats * p.nb * 128;
            const int64_t step = (int64_t)mats * p.nb * 128;
            for (int q = tid; q < it.cnt * 128; q += FEW_EPI_WARPS * 32) {
                const int j = q >> 7, cc = q & 127;
                if (it.n0 + cc >= h) continue;
                float u = 0.f, v = 0.f;
                for (int pp = 0; pp < P; ++pp) {
                    u += __ldcg(all + pp * step + j * 128 + cc);
                    if (mats == 2) v += __ldcg(all + pp * step + (p.nb + j) * 128 + cc);
                }
                store_hidden(p, it, j, it.n0 + cc, mats == 2 ? act_silu(u) * v : act_gelu(u));
            }
            fence_proxy_async_all();
            __threadfence();
            epi_sync();
            if (tid == 0) atomicAdd(done, 1);
        } else {
            const int64_t slots = (int64_t)p.T * p.k;
            // rows of the partial outputs: [P2][T k] routed, then [P2s][T] shared
            float* yp = it.shared ? p.y_part + (int64_t)L.plan->P2 * slots * p.d + (int64_t)it.part * p.T * p.d
                                  : p.y_part + ((int64_t)it.part * slots + it.row0) * p.d;
            const int col = it.n0 + c;
            for (int g = half; g < groups; g += 2) {
                uint32_t u[8];
                tmem_ld_32x32b_x8(tb + 8 * g, u);
                tmem_wait_ld();
                if (col < p.d) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = 8 * g + i;
                        if (j < it.cnt) yp[(int64_t)j * p.d + col] = __uint_as_float(u[i]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.tempty + 8 * acc);
            __threadfence();
            epi_sync();
            const int dt = it.n0 / 128, want = p.k * L.plan->P2 + (p.hs > 0 ? L.plan->P2s : 0);
            if (tid < it.cnt) {
                const int t = it.shared ? tid : L.row_tok[it.row0 + tid];
                flags[tid] = atomicAdd(p.y_cnt + t * p.ntd + dt, 1) == want - 1 ? t : -1;
            }
            epi_sync();
            for (int j = warp; j < it.cnt; j += FEW_EPI_WARPS) {
                const int t = flags[j];
                if (t < 0) continue;
                __threadfence();
                const int cc = it.n0 + lane * 4;   // d is a multiple of 8: whole groups of 4
                if (cc >= p.d) continue;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int q = 0; q < p.k; ++q) {
                    const float gt = L.gate[t * p.k + q];
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int pp = 0; pp < L.plan->P2; ++pp) {
                        const float4 a = __ldcg(reinterpret_cast<const float4*>(
                            p.y_part + ((int64_t)pp * slots + L.row_of[t * p.k + q]) * p.d + cc));
                        o.x += a.x;
                        o.y += a.y;
                        o.z += a.z;
                        o.w += a.w;
                    }
                    y.x = fmaf(gt, o.x, y.x);
                    y.y = fmaf(gt, o.y, y.y);
                    y.z = fmaf(gt, o.z, y.z);
                    y.w = fmaf(gt, o.w, y.w);
                }
                if (p.hs > 0) {
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int pp = 0; pp < L.plan->P2s; ++pp) {
                        const float4 a = __ldcg(reinterpret_cast<const float4*>(
                            p.y_part + ((int64_t)L.plan->P2 * slots + (int64_t)pp * p.T + t) * p.d + cc));
                        o.x += a.x;
                        o.y += a.y;
                        o.z += a.z;
                        o.w += a.w;
                    }
                    y.x = fmaf(p.lambda, o.x, y.x);
                    y.y = fmaf(p.lambda, o.y, y.y);
                    y.z = fmaf(p.lambda, o.z, y.z);
                    y.w = fmaf(p.lambda, o.w, y.w);
                }
                uint2 u;
                u.x = pack_bf16x2(y.x, y.y);
                u.y = pack_bf16x2(y.z, y.w);
                *reinterpret_cast<uint2*>(p.y + (int64_t)t * p.d + cc) = u;
            }
        }
    }
}

// ----------------------------------------------------------------- kernel

// Shared memory, from a 1024-byte boundary: ring, barriers and flags, lists.  The router
// stages use the ring's space before the ring is live.
struct FewSizes {
    int stage_bytes, stages, lists, total;
};
__host__ __device__ inline FewSizes few_sizes(int T, int k, int E, bool swiglu) {
    FewSizes z;
    const int nb = (T + 15) / 16 * 16, n = T * k, na = n < E ? n : E;
    z.stage_bytes = (swiglu ? 2 : 1) * FEW_TILE_BYTES + 2 * nb * 128;
    // plan, gate, row_of, act, off, cnt, row_tok
    z.lists = 64 + ((4 * n + 2 * n + 4 * na + na + n + 15) & ~15);
    const int left = FEW_SMEM_MAX - 1024 - FEW_BAR_BYTES - 320 - z.lists;
    z.stages = left / z.stage_bytes;
    if (z.stages > 12) z.stages = 12;
    z.total = 1024 + z.stages * z.stage_bytes + FEW_BAR_BYTES + 320 + z.lists;
    return z;
}

__global__ void __launch_bounds__(FEW_THREADS, 1) few_kernel(const __grid_constant__ FewArgs p) {
    extern __shared__ uint8_t few_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(few_smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    const FewSizes z = few_sizes(p.T, p.k, p.E, p.W3 != nullptr);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + z.stages * z.stage_bytes);
    uint8_t* after = reinterpret_cast<uint8_t*>(bars) + FEW_BAR_BYTES;
    volatile int* flags = reinterpret_cast<volatile int*>(after);            // 66 ints
    volatile int* abort_flag = flags + 68;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(after) + 69;
    uint8_t* at = after + 320;
    const int n = p.T * p.k, na = n < p.E ? n : p.E;
    FewLists L;
    L.plan = reinterpret_cast<FewPlan*>(at);
    L.gate = reinterpret_cast<float*>(at + 64);
    L.row_of = reinterpret_cast<uint16_t*>(L.gate + n);
    L.act = L.row_of + n;
    L.off = L.act + na;
    L.cnt = reinterpret_cast<uint8_t*>(L.off + na);
    L.row_tok = L.cnt + na;
    FewSmem sm;
    sm.ring = smem_u32(smem);
    sm.stages = z.stages;
    sm.stage_bytes = z.stage_bytes;
    sm.b_off = z.stage_bytes - 2 * p.nb * 128;
    sm.lo_off = p.nb * 128;
    sm.full = smem_u32(bars);
    sm.empty = sm.full + 8 * 12;
    sm.tfull = sm.empty + 8 * 12;
    sm.tempty = sm.tfull + 16;
    sm.drain = sm.tempty + 16;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < z.stages; ++s) {
            mbar_init(sm.full + 8 * s, 2);    // weights, tokens
            mbar_init(sm.empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sm.tfull + 8 * a, 1);
            mbar_init(sm.tempty + 8 * a, FEW_EPI_WARPS);
        }
        mbar_init(sm.drain, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    pdl_wait();
    // counters of this call, used only after the grid barrier
    for (int i = blockIdx.x * FEW_THREADS + threadIdx.x; i < p.n_counters; i += gridDim.x * FEW_THREADS)
        p.done_up[i] = 0;
    few_logits(p, reinterpret_cast<float*>(smem));
    if (!grid_barrier(p.status, gridDim.x, p.limit_ns, SITE_FEW_BARRIER)) return;

    const int sel_bytes = (p.E + 31) / 32 * 32 * 24, ring_bytes = z.stages * z.stage_bytes;
    const int sel_warps = min(FEW_SEL_WARPS, ring_bytes / sel_bytes);
    uint8_t* sel = smem + warp * sel_bytes;
    if (p.T <= FEW_SEL_WARPS && p.T * sel_bytes + 8 * n <= ring_bytes) {   // every CTA selects
        int32_t* s_idx = reinterpret_cast<int32_t*>(smem + p.T * sel_bytes);
        float* s_gate = reinterpret_cast<float*>(s_idx + n);
        if (warp < p.T) few_select(p, warp, sel, s_idx + warp * p.k, s_gate + warp * p.k);
        __syncthreads();
        if (blockIdx.x == 0)
            for (int i = threadIdx.x; i < n; i += FEW_THREADS) {
                p.idx[i] = s_idx[i];
                p.gate[i] = s_gate[i];
            }
        few_plan<true>(p, L, s_idx, s_gate, smem);
    } else {
        if (warp < sel_warps)
            for (int t = blockIdx.x + (int)gridDim.x * warp; t < p.T; t += (int)gridDim.x * sel_warps)
                few_select(p, t, sel, p.idx + t * p.k, p.gate + t * p.k);
        if (!grid_barrier(p.status, gridDim.x, p.limit_ns, SITE_FEW_BARRIER)) return;
        few_plan<false>(p, L, p.idx, p.gate, smem);
    }
    __syncwarp();
    if (warp == FEW_WARP_MMA) {
        tmem_alloc(smem_u32(tmem_slot), p.tmem_cols);
        tmem_relinquish();
    }
    fence_proxy_async_smem();   // the router's use of the ring, before TMA writes to it
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (warp < FEW_EPI_WARPS) {
        few_epilogue(p, sm, L, tmem, abort_flag, flags);
    } else if ((threadIdx.x & 31) == 0) {
        if (warp == FEW_WARP_W) few_load_w(p, sm, L, abort_flag);
        else if (warp == FEW_WARP_MMA) few_mma(p, sm, L, tmem, abort_flag);
        else if (warp == FEW_WARP_B) few_load_b(p, sm, L, abort_flag);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == FEW_WARP_MMA) {
        tc_fence_after();
        tmem_dealloc(tmem, p.tmem_cols);
    }
}

inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }
inline int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
inline int64_t tiles128(int64_t v) { return (v + 127) / 128; }

// Router split: parts of d for blocks of 8 experts.
int few_rt_parts(int d, int E, int ctas) {
    const int eb = (E + 7) / 8;
    int p = ctas / eb;
    if (p > 8) p = 8;
    if (p > (d + 63) / 64) p = (d + 63) / 64;
    return p < 1 ? 1 : p;
}

struct FewLayout {
    size_t idx, gate, part, wsq, counters, up_part, H, Hs, y_part, total;
    int64_t n_done, n_up_cnt, n_y_cnt;
};
FewLayout few_layout(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t hs) {
    FewLayout L;
    size_t o = up256(sizeof(DevStatus));
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    const int64_t n = T * k, na = n < E ? n : E, nb = (T + 15) / 16 * 16;
    L.idx = take(4 * n);
    L.gate = take(4 * n);
    L.part = take(4 * 8 * T * E);
    L.wsq = take(4 * 8 * E);
    L.n_done = na + 1;
    L.n_up_cnt = na * tiles128(h) + tiles128(hs);
    L.n_y_cnt = T * tiles128(d);
    L.counters = take(4 * (L.n_done + L.n_up_cnt + L.n_y_cnt));
    L.up_part = take((size_t)4 * FEW_MAX_PART * 2 * nb * 128);
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
    a.done_up = reinterpret_cast<int32_t*>(ws + L.counters);
    a.up_cnt = a.done_up + L.n_done;
    a.y_cnt = a.up_cnt + L.n_up_cnt;
    a.n_counters = (int)(L.n_done + L.n_up_cnt + L.n_y_cnt);
    a.up_part = reinterpret_cast<float*>(ws + L.up_part);
    a.H = reinterpret_cast<__nv_bfloat16*>(ws + L.H);
    a.Hs = reinterpret_cast<__nv_bfloat16*>(ws + L.Hs);
    a.y_part = reinterpret_cast<float*>(ws + L.y_part);
    a.status = reinterpret_cast<DevStatus*>(ws);
    a.limit_ns = limit_ns;
    a.ldh = (int)up8(a.h);
    a.ldhs = (int)up8(a.hs);
    a.na_max = n < a.E ? n : a.E;
    a.nb = (a.T + 15) / 16 * 16;
    a.nt = (int)tiles128(a.h);
    a.nt_s = (int)tiles128(a.hs);
    a.ntd = (int)tiles128(a.d);
    a.nkb_d = (a.d + 63) / 64;
    a.nkb_h = (a.h + 63) / 64;
    a.nkb_hs = (a.hs + 63) / 64;
    a.acc_cols = a.nb * (a.W3 ? 2 : 1);
    a.tmem_cols = 32;
    while (a.tmem_cols < 2 * a.acc_cols) a.tmem_cols *= 2;
    a.rt_eb = (a.E + 7) / 8;
    a.rt_parts = few_rt_parts(a.d, a.E, sms);
    a.rt_dch = (int)up8((a.d + a.rt_parts - 1) / a.rt_parts);
    // length of the summation chains of a logit (few_logits): 16 products, their sums, the
    // lanes, the warps, the parts; times 2^-24, with room for the second-order terms
    const int kp = FEW_WARPS / ((a.T + 7) / 8);
    const int chain = 16 + (a.rt_dch / (64 * kp) + a.rt_dch / FEW_RT_K + 2) + 2 + kp + a.rt_parts + 2;
    a.rt_err = 1.01f * (float)chain * 5.9604645e-8f;

    bool ok = make_weight_tmap_strided(&a.tW1, a.W1, a.h, a.d, a.E, a.hp, (int64_t)a.d * a.hp) &&
              make_weight_tmap_strided(&a.tW2, a.W2, a.d, a.h, a.E, a.d, (int64_t)a.h * a.d) &&
              make_gather_tmap(&a.tX, a.x, a.d, a.T, a.d) &&
              make_kmajor_tmap(&a.tH, a.H, a.h, n, 2, a.ldh, (int64_t)n * a.ldh, 16);
    if (ok && a.W3) ok = make_weight_tmap_strided(&a.tW3, a.W3, a.h, a.d, a.E, a.hp, (int64_t)a.d * a.hp);
    if (ok && a.hs > 0) {
        ok = make_weight_tmap_strided(&a.tS1, a.Ws1, a.hs, a.d, 1, a.hsp, (int64_t)a.d * a.hsp) &&
             make_weight_tmap_strided(&a.tS2, a.Ws2, a.d, a.hs, 1, a.d, (int64_t)a.hs * a.d) &&
             make_kmajor_tmap(&a.tHs, a.Hs, a.hs, a.T, 2, a.ldhs, (int64_t)a.T * a.ldhs, 16);
        if (ok && a.W3) ok = make_weight_tmap_strided(&a.tS3, a.Ws3, a.hs, a.d, 1, a.hsp, (int64_t)a.d * a.hsp);
    }
    if (!ok) return cudaErrorInvalidValue;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM_MAX);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    const FewSizes z = few_sizes(a.T, a.k, a.E, a.W3 != nullptr);
    const cudaError_t e = launch_pdl_coop(few_kernel, dim3((unsigned)sms), dim3(FEW_THREADS), z.total, s, a);
    count_launches(1);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mv
