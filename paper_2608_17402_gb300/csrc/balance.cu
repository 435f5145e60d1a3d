// balance.cu -- the auxiliary loss of expert loads, the loads and the gradient of the router's
// logits, sm_103a.
//
// With the tokens of run b (all of them, or one sequence's), n_be = the number of their ids that are
// e and f_be = E n_be / (k T_b) (1 for every expert of an even load), and p_te = softmax(s_t)_e or
// sigmoid(s_te) / sum_j sigmoid(s_tj):
//   L = coef sum_b (T_b / T) sum_e f_be P_be,   P_be = mean over the run of p_te
//     = sum_t p_t . C_b(t) with C_be = coef f_be / T.
// The counts have no gradient, so C is known before the logits are read, and one pass over them
// gives the loss and ds.  p_t adds up to 1: with c_be = C_be - coef / T, formed from the whole number
// E n_be - k T_b, nothing cancels where loads are nearly even:
//   p.C = p.c + coef / T,   softmax: ds = p (c - p.c),   sigmoid: ds = p (1 - sigmoid(s)) (c - p.c).
// s is read and ds written once, 8 T E bytes; 65536 x 256, sigmoid: 32.7 us, 4.2 TB/s, about 7 of them counting and
// starting, 21 the pass (instructions and their latency: 60% of the issue slots, DRAM 39% busy), 3 the last CTAs and
// the loss.  Where ids are few, every CTA
// of bal_main_kernel counts those of its runs by itself; otherwise bal_count_kernel first counts them in
// parts, which bal_main_kernel adds up.
#include <math.h>

#include <algorithm>

#include "internal.h"

namespace mv {

namespace {

constexpr int BAL_COUNT_THREADS = 1024;
constexpr int BAL_PART_IDS = 8192;    // ids a CTA of bal_count_kernel counts, about
// Up to so many ids, and so many a run in the mean, CTAs of bal_main_kernel count for themselves: a launch less, but
// each counts every run that it has rows of.  64 experts, 8 ids a token, counted so and by bal_count_kernel, us:
// one run of 4096 ids 6.1 and 8.3, 16384 8.7 and 8.9, 65536 17.3 and 9.0; 32 runs of 65536 ids together 7.2 and 9.3
// (16 and 256 experts change sides at the same numbers).  Alike runs would gain beyond the first limit (262144 ids
// in 32 runs: 9.8 and 11.2); it bounds what a single long one among them can cost.
constexpr int64_t BAL_FEW_IDS = 65536, BAL_FEW_IDS_RUN = 16384;
constexpr int BAL_THREADS = 512;
constexpr int BAL_AHEAD = 2;   // rounds

// Rows of run b; runs outside [0, T) are cut off (and are an error, which bal_main_kernel reports).
__device__ __forceinline__ void run_rows(const BalanceArgs& a, int64_t b, int64_t& t0, int64_t& t1) {
    t0 = a.seg ? max((int64_t)a.seg[b], (int64_t)0) : 0;
    t1 = a.seg ? min((int64_t)a.seg[b + 1], a.T) : a.T;
    if (t1 < t0) t1 = t0;
}

// hist += the ids [i0, i1) of idx, by all threads of the CTA; 16 bytes at a time where idx allows it.
__device__ __forceinline__ void count_ids(const BalanceArgs& a, int64_t i0, int64_t i1, int* hist) {
    auto one = [&](int64_t i, int e) {
        if (e >= 0 && e < a.E) atomicAdd(&hist[e], 1);
        else report(a.st, MOEVIE_ERR_DEVICE, SITE_BALANCE_ID, (int)i, e);
    };
    if ((reinterpret_cast<uintptr_t>(a.idx) & 15) == 0) {
        const int64_t v0 = min((i0 + 3) / 4 * 4, i1), v1 = max(i1 / 4 * 4, v0);
        for (int64_t i = i0 + threadIdx.x; i < v0; i += blockDim.x) one(i, a.idx[i]);
#pragma unroll 4
        for (int64_t i = v0 + 4 * threadIdx.x; i < v1; i += 4 * blockDim.x) {
            const int4 e = *reinterpret_cast<const int4*>(a.idx + i);
            one(i, e.x);
            one(i + 1, e.y);
            one(i + 2, e.z);
            one(i + 3, e.w);
        }
        for (int64_t i = v1 + threadIdx.x; i < i1; i += blockDim.x) one(i, a.idx[i]);
    } else {
#pragma unroll 4
        for (int64_t i = i0 + threadIdx.x; i < i1; i += blockDim.x) one(i, a.idx[i]);
    }
}

// part[b][p][e] = the ids e among part p of run b.  blockIdx.x: p, blockIdx.y: runs.
__global__ void __launch_bounds__(BAL_COUNT_THREADS) bal_count_kernel(const BalanceArgs a) {
    __shared__ int hist[1024];
    pdl_wait();
    asm volatile("griddepcontrol.launch_dependents;");   // bal_main_kernel may start, and waits for this one's end
    const int p = blockIdx.x;
    for (int64_t b = blockIdx.y; b < a.G; b += gridDim.y) {
        for (int e = threadIdx.x; e < a.E; e += BAL_COUNT_THREADS) hist[e] = 0;
        __syncthreads();
        int64_t t0, t1;
        run_rows(a, b, t0, t1);
        const int64_t len = t1 - t0;
        count_ids(a, (t0 + len * p / a.parts) * a.k, (t0 + len * (p + 1) / a.parts) * a.k, hist);
        __syncthreads();
        int32_t* out = a.part + (b * a.parts + p) * a.E;
        for (int e = threadIdx.x; e < a.E; e += BAL_COUNT_THREADS) out[e] = hist[e];
        __syncthreads();
    }
}

// e^x for x <= 0: 2^(x / ln 2), whose exponent's rounding makes it off by up to |x| 2^-24 of itself
// and a few units; 0 at minus infinity.
__device__ __forceinline__ float exp_neg(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.44269504088896341f));
    return r;
}
__device__ __forceinline__ uint64_t f2_of(float v) { return f2_pack(v, v); }
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// v[n] <- its sum over the LP lanes of a token, in all of them.  Four sums share the shuffles: after
// the first two steps each lane carries one of them, the n-th lanes n LP / 4 on.
template <int LP, int N>
__device__ __forceinline__ void lane_sums(float (&v)[N]) {
    if constexpr (N == 4 && LP >= 8) {
        const int lane = threadIdx.x & 31;
        const bool up = lane & (LP / 2), up2 = lane & (LP / 4);
        const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], LP / 2);
        const float b = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], LP / 2);
        float x = (up2 ? b : a) + __shfl_xor_sync(0xffffffffu, up2 ? a : b, LP / 4);
#pragma unroll
        for (int o = LP / 8; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = __shfl_sync(0xffffffffu, x, (lane & ~(LP - 1)) + n * (LP / 4));
    } else {
#pragma unroll
        for (int o = LP / 2; o; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
    }
}

// The even load less than the run's: c of every expert, in s_c[0, n) (0 behind the last).  s_hist: scratch.
__device__ __forceinline__ void run_loads(const BalanceArgs& a, int64_t b, int64_t r0, int64_t r1, float per_row,
                                          bool mine, int n, int* s_hist, float* s_c) {
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += BAL_THREADS) s_hist[e] = 0;
    __syncthreads();
    if (a.parts == 0) {
        count_ids(a, r0 * a.k, r1 * a.k, s_hist);
    } else {   // threads share the parts of an expert
        const int lanes = max(1, BAL_THREADS / a.E);
        for (int i = threadIdx.x; i < a.E * lanes; i += BAL_THREADS) {
            const int e = i % a.E;
            int sum = 0;
#pragma unroll 16
            for (int p = i / a.E; p < a.parts; p += lanes) sum += a.part[(b * a.parts + p) * a.E + e];
            atomicAdd(&s_hist[e], sum);
        }
    }
    __syncthreads();
    const float scale = per_row / ((float)a.k * (float)(r1 - r0));   // coef / (T k T_b)
    for (int e = threadIdx.x; e < n; e += BAL_THREADS) {
        const int count = e < a.E ? s_hist[e] : 0;
        if (mine && e < a.E) a.counts[b * a.E + e] = count;
        s_c[e] = e < a.E ? scale * (float)((int64_t)a.E * count - (int64_t)a.k * (r1 - r0)) : 0.f;
    }
    __syncthreads();
}

// LP lanes hold a token's logits, VPL groups of VEC columns each; a warp takes 32 / LP tokens at a
// time, TU times over (the loads of all of them under way together, their sums in one set of
// shuffles).  8 columns a lane wherever there are as many: fewer leave more of the time to the shuffles.
// No fp64 on the way: the card's rate for it is 1 / 64 of that for fp32.
template <int VEC, int LP, int VPL, int TU>
__global__ void __launch_bounds__(BAL_THREADS, VEC * VPL > 8 ? 1 : 2) bal_main_kernel(const BalanceArgs a) {
    constexpr int NV = VEC * VPL, NP = NV / 2, TPW = 32 / LP, WARPS = BAL_THREADS / 32;
    static_assert(NV % 2 == 0, "pairs of columns");
    __shared__ __align__(16) float s_c[1024];
    __shared__ int s_hist[1024];
    __shared__ float s_sum[WARPS];
    __shared__ int s_rows[WARPS];
    __shared__ unsigned s_last;
    // While bal_count_kernel runs, the logits of this CTA's first rounds (of rows without padding in front) on their
    // way to L2: 65536 x 256 in 32.4 us instead of 33.2.
    if (a.parts > 0) {
        const int64_t from = a.T * blockIdx.x / gridDim.x;
        const int64_t to = min(from + BAL_AHEAD * WARPS * TPW * TU, a.T * (blockIdx.x + 1) / gridDim.x);
        const int lines = (a.E + 31) / 32;
        for (int64_t i = threadIdx.x; i < (to - from) * lines; i += BAL_THREADS)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(a.s + (from + i / lines) * a.ld_s + i % lines * 32));
    }
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / LP, l = lane % LP;
    auto column = [&](int i) { return (i / VEC * LP + l) * VEC + i % VEC; };

    // runs that do not ascend within [0, T], and the loads of runs without a token
    for (int64_t b = (int64_t)blockIdx.x * BAL_THREADS + threadIdx.x; a.seg && b < a.G; b += (int64_t)gridDim.x * BAL_THREADS) {
        const int x = a.seg[b], y = a.seg[b + 1];
        if (x < 0 || y < x || y > a.T) report(a.st, MOEVIE_ERR_DEVICE, SITE_RUNS, (int)b, y);
        if (min((int64_t)y, a.T) <= max(x, 0))
            for (int e = 0; e < a.E; ++e) a.counts[b * a.E + e] = 0;
    }

    int64_t lo = 0, hi = a.T;   // rows that lie in some run
    if (a.seg) {
        lo = max((int64_t)a.seg[0], (int64_t)0);
        hi = max(lo, min((int64_t)a.seg[a.G], a.T));
    }
    const int64_t n_rows = hi - lo;
    const float per_row = n_rows > 0 ? a.coef / (float)n_rows : 0.f;
    const int64_t t0 = lo + n_rows * blockIdx.x / gridDim.x, t1 = lo + n_rows * (blockIdx.x + 1) / gridDim.x;
    constexpr uint64_t NONE = 0xff800000ff800000ull;   // two logits of minus infinity
    bool in[VPL];
#pragma unroll
    for (int v = 0; v < VPL; ++v) in[v] = column(VEC * v) < a.E;
    float dots = 0.f;   // of the tokens of this lane's group
    int rows = 0;
    int64_t b = a.seg && t0 < t1 ? warp_run_of(a.seg, a.G, t0) : 0;
    for (int64_t t = t0; t < t1 && b < a.G; ++b) {
        int64_t r0, r1;
        run_rows(a, b, r0, r1);
        const int64_t end = min(r1, t1);
        if (end <= t) continue;
        run_loads(a, b, r0, r1, per_row, r0 >= t0 && r0 < t1, LP * NV, s_hist, s_c);
        uint64_t c_reg[NP];   // lanes of more than 8 columns read them from shared memory each time
        auto c_mem = [&](int i) { return *reinterpret_cast<const uint64_t*>(s_c + column(2 * i)); };
        if constexpr (VEC == 1) {
#pragma unroll
            for (int i = 0; i < NP; ++i) c_reg[i] = f2_pack(s_c[column(2 * i)], s_c[column(2 * i + 1)]);
        } else if constexpr (NV <= 8) {
#pragma unroll
            for (int i = 0; i < NP; ++i) c_reg[i] = c_mem(i);
        }
        auto c = [&](int i) {
            if constexpr (VEC == 1 || NV <= 8) return c_reg[i];
            else return c_mem(i);
        };
        auto load_row = [&](const float* src, bool live, uint64_t (&x)[NP]) {
            if constexpr (VEC == 4) {
#pragma unroll
                for (int v = 0; v < VPL; ++v) {
                    ulonglong2 f = make_ulonglong2(NONE, NONE);
                    if (live && in[v]) f = *reinterpret_cast<const ulonglong2*>(src + 4 * LP * v);
                    x[2 * v] = f.x;
                    x[2 * v + 1] = f.y;
                }
            } else {
                float f[NV];
#pragma unroll
                for (int i = 0; i < NV; ++i) f[i] = live && column(i) < a.E ? src[LP * i] : -INFINITY;
#pragma unroll
                for (int i = 0; i < NP; ++i) x[i] = f2_pack(f[2 * i], f[2 * i + 1]);
            }
        };
        auto add_up = [&](const uint64_t& p, int i, uint64_t (&s)[2]) {
            s[0] = i ? f2_add(s[0], p) : p;
            s[1] = i ? f2_fma(p, c(i), s[1]) : f2_mul(p, c(i));
        };
        auto total = [&](const uint64_t (&s)[2], float* out) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                float y, z;
                f2_unpack(s[n], y, z);
                out[n] = y + z;
            }
        };
        // x <- e^(x - the row's largest logit) = p of a softmax but for its sum, and s its sums, in the
        // lane; a row without a logit has no probability
        auto soft = [&](uint64_t (&x)[NP], uint64_t (&s)[2]) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float y, z;
                f2_unpack(x[i], y, z);
                m = fmaxf(m, fmaxf(y, z));
            }
#pragma unroll
            for (int o = LP / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const uint64_t shift = f2_of(m == -INFINITY ? 0.f : -m);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float y, z;
                f2_unpack(f2_add(x[i], shift), y, z);
                x[i] = f2_pack(exp_neg(y), exp_neg(z));
                add_up(x[i], i, s);
            }
            return m;
        };
        // rows left to this lane's first one of a round; and where its logits and their gradients lie
        const float* src = a.s + (t + warp * (TPW * TU) + sub) * a.ld_s + l * VEC;
        float* dst = a.ds + (t + warp * (TPW * TU) + sub) * a.ld_ds + l * VEC;
        const int64_t src_u = TPW * a.ld_s, dst_u = TPW * a.ld_ds;
        int left = (int)(end - t) - warp * (TPW * TU) - sub;
        const int rounds = (int)((end - t + WARPS * TPW * TU - 1) / (WARPS * TPW * TU));   // of all warps alike
#pragma unroll 1
        for (int round = 0; round < rounds; ++round) {
            uint64_t x[TU][NP];   // logits, then p times its slope by the logit but for sums
            float sums[2 * TU];   // of p, and of p c
#pragma unroll
            for (int u = 0; u < TU; ++u) load_row(src + u * src_u, u * TPW < left, x[u]);
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                uint64_t s[2] = {0, 0};
                if (a.score == MOEVIE_SCORE_SOFTMAX) {
                    soft(x[u], s);
                } else {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {   // sigmoid(v) = r or z r with z = e^-|v|, r = 1 / (1 + z)
                        float v[2], z[2], r[2];
                        f2_unpack(x[u][i], v[0], v[1]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) z[j] = exp_neg(-fabsf(v[j]));
                        const uint64_t zz = f2_pack(z[0], z[1]);
                        float d[2];
                        f2_unpack(f2_add(zz, f2_of(1.f)), d[0], d[1]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) r[j] = rcp_approx(d[j]);
                        const uint64_t rr = f2_pack(r[0], r[1]), zr = f2_mul(zz, rr);
                        float y[2];
                        f2_unpack(zr, y[0], y[1]);
                        add_up(f2_pack(v[0] >= 0.f ? r[0] : y[0], v[1] >= 0.f ? r[1] : y[1]), i, s);
                        x[u][i] = f2_mul(rr, zr);   // sigmoid (1 - sigmoid)
                    }
                }
                total(s, sums + 2 * u);
            }
            lane_sums<LP>(sums);
            if (a.score == MOEVIE_SCORE_SIGMOID) {
                // Of a row whose logits all lie below -17, sigmoid(s) is e^s to e^-17 of itself, and vanishes
                // in the end: its probabilities are a softmax.  Its scores add up to less than 1024 e^-17.
                bool low = false;
#pragma unroll
                for (int u = 0; u < TU; ++u) low |= sums[2 * u] < 4.3e-5f;
                if (__any_sync(0xffffffffu, low)) {
#pragma unroll 1
                    for (int u = 0; u < TU; ++u) {
                        uint64_t y[NP], s[2] = {0, 0};
                        load_row(src + u * src_u, u * TPW < left, y);
                        const bool done = soft(y, s) < -17.f;
                        float w[2];
                        total(s, w);
                        lane_sums<LP>(w);
#pragma unroll
                        for (int k = 0; k < TU; ++k) {
                            if (k != u || !done) continue;
                            sums[2 * k] = w[0];
                            sums[2 * k + 1] = w[1];
#pragma unroll
                            for (int i = 0; i < NP; ++i) x[k][i] = y[i];
                        }
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                if (u * TPW >= left) continue;
                // (Sums are 0, or at least 1 of a softmax and e^-17 of sigmoids, whose largest logit lies at -17 or above,
                // and at most 1024: the approximate reciprocal is as good as a division there.)
                const float inv = sums[2 * u] == 0.f ? 0.f : rcp_approx(sums[2 * u]);
                const float dot = sums[2 * u + 1] * inv;
                if (l == 0) {
                    dots += dot;
                    rows += sums[2 * u] == 0.f ? 0 : 1;
                }
                if (!a.ds) continue;
                float* out = dst + u * dst_u;
                const uint64_t scale = f2_of(inv), less = f2_of(-dot);
                uint64_t g[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) g[i] = f2_mul(f2_mul(x[u][i], scale), f2_add(c(i), less));
                if constexpr (VEC == 4) {
#pragma unroll
                    for (int v = 0; v < VPL; ++v)
                        if (in[v]) *reinterpret_cast<ulonglong2*>(out + 4 * LP * v) = make_ulonglong2(g[2 * v], g[2 * v + 1]);
                } else {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        float y, z;
                        f2_unpack(g[i], y, z);
                        if (column(2 * i) < a.E) out[LP * 2 * i] = y;
                        if (column(2 * i + 1) < a.E) out[LP * (2 * i + 1)] = z;
                    }
                }
            }
            left -= WARPS * TPW * TU;
            src += (WARPS * TU) * src_u;
            dst += (WARPS * TU) * dst_u;
        }
        t = end;
    }

    // the loss: every CTA's sums, added up in order by the CTA that is done last
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        dots += __shfl_xor_sync(0xffffffffu, dots, o);
        rows += __shfl_xor_sync(0xffffffffu, rows, o);
    }
    if (lane == 0) {
        s_sum[warp] = dots;
        s_rows[warp] = rows;
    }
    __syncthreads();
    if (warp != 0) return;
    dots = lane < WARPS ? s_sum[lane] : 0.f;
    rows = lane < WARPS ? s_rows[lane] : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        dots += __shfl_xor_sync(0xffffffffu, dots, o);
        rows += __shfl_xor_sync(0xffffffffu, rows, o);
    }
    if (lane == 0) {
        __stcg(&a.cta_sum[blockIdx.x], make_float2(dots, __int_as_float(rows)));
        __threadfence();
        s_last = atomicInc(&a.st->bal_ticket, gridDim.x - 1) == gridDim.x - 1;   // back to 0 for the next call
        __threadfence();
    }
    __syncwarp();
    if (!s_last) return;
    dots = 0.f;
    int64_t all = 0;
    for (unsigned i = lane; i < gridDim.x; i += 32) {
        const float2 v = __ldcg(&a.cta_sum[i]);
        dots += v.x;
        all += __float_as_int(v.y);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        dots += __shfl_xor_sync(0xffffffffu, dots, o);
        all += __shfl_xor_sync(0xffffffffu, all, o);
    }
    if (lane == 0) *a.loss = all == n_rows && all > 0 ? a.coef + dots : fmaf(per_row, (float)all, dots);
}

template <int VEC, int LP, int VPL, int TU>
cudaError_t run_main(const BalanceArgs& a, cudaStream_t s) {
    const int64_t rows_cta = (int64_t)(BAL_THREADS / 32) * (32 / LP) * TU;   // one round of its warps
    const int most = VEC * VPL > 8 ? GB300_SMS : BAL_MAX_GRID;                // one CTA to an SM, or two
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>((a.T + rows_cta - 1) / rows_cta, most));
    return launch_pdl(bal_main_kernel<VEC, LP, VPL, TU>, dim3(grid), dim3(BAL_THREADS), 0, s, a);
}

}  // namespace

int bal_parts(int64_t T, int64_t k, int64_t G) {
    if (T * k <= std::min(BAL_FEW_IDS, G * BAL_FEW_IDS_RUN)) return 0;
    const int64_t n = (T * k + G * BAL_PART_IDS - 1) / (G * BAL_PART_IDS);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, BAL_MAX_PARTS));
}

int64_t bal_max_parts(int64_t T, int64_t k, int64_t G) {
    return std::min<int64_t>(BAL_MAX_PARTS * G, (T * k + BAL_PART_IDS - 1) / BAL_PART_IDS + G);
}

cudaError_t launch_balance(const BalanceArgs& a, cudaStream_t s) {
    cudaError_t e;
    if (a.parts > 0) {
        e = launch_pdl(bal_count_kernel, dim3(a.parts, (unsigned)std::min<int64_t>(a.G, 4096)), dim3(BAL_COUNT_THREADS), 0,
                       s, a);
        count_launches(1);
        if (e != cudaSuccess) return e;
    }
    const bool wide = a.E % 4 == 0 && a.ld_s % 4 == 0 && (reinterpret_cast<uintptr_t>(a.s) & 15u) == 0 &&
                      (!a.ds || (a.ld_ds % 4 == 0 && (reinterpret_cast<uintptr_t>(a.ds) & 15u) == 0));
    const int E = a.E;
    if (wide) {   // 16 bytes to a lane's access
        if (E <= 16) e = run_main<4, 2, 2, 2>(a, s);
        else if (E <= 32) e = run_main<4, 4, 2, 2>(a, s);
        else if (E <= 64) e = run_main<4, 8, 2, 2>(a, s);
        else if (E <= 128) e = run_main<4, 16, 2, 2>(a, s);
        else if (E <= 256) e = run_main<4, 32, 2, 2>(a, s);
        else if (E <= 512) e = run_main<4, 32, 4, 1>(a, s);
        else e = run_main<4, 32, 8, 1>(a, s);
    } else {   // rows at any alignment
        if (E <= 16) e = run_main<1, 8, 2, 2>(a, s);
        else if (E <= 32) e = run_main<1, 8, 4, 2>(a, s);
        else if (E <= 64) e = run_main<1, 8, 8, 2>(a, s);
        else if (E <= 128) e = run_main<1, 16, 8, 2>(a, s);
        else if (E <= 256) e = run_main<1, 32, 8, 2>(a, s);
        else if (E <= 512) e = run_main<1, 32, 16, 1>(a, s);
        else e = run_main<1, 32, 32, 1>(a, s);
    }
    count_launches(1);
    return e;
}

}  // namespace mv
