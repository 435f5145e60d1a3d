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
// HBM bounds it: s is read and ds written once, 8 T E bytes.  Where all ids together are few, every CTA
// of bal_main_kernel counts those of its runs by itself; otherwise bal_count_kernel first counts them in
// parts, which bal_main_kernel adds up.
#include <math.h>

#include <algorithm>

#include "internal.h"

namespace mv {

namespace {

constexpr int BAL_COUNT_THREADS = 1024;
constexpr int BAL_PART_IDS = 8192;    // ids a CTA of bal_count_kernel counts, about
constexpr int64_t BAL_FEW_IDS = 65536;   // up to here CTAs of bal_main_kernel count for themselves
constexpr int BAL_THREADS = 512;

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

// e^x for x <= 0 to a few units in the last place: 2^t with t = x / ln 2 in two pieces, the lower one
// by its first-order term (x below -126 ln 2: 0).
__device__ __forceinline__ float exp_neg(float x) {
    constexpr float L2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
    const float t = x * L2E;
    const float low = fmaf(x, L2E, -t);   // exact; the rounding of L2E itself is below 2^-26 of t
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return t < -126.f ? 0.f : fmaf(r, low * LN2, r);
}

// LP lanes hold a token's logits, VPL groups of VEC columns each; a warp takes 32 / LP tokens at a
// time, TU times over (the loads of all of them under way together, their sums in one set of
// shuffles).  8 columns a lane wherever there are as many: fewer leave more of the time to the shuffles.
template <int VEC, int LP, int VPL, int TU>
__global__ void __launch_bounds__(BAL_THREADS, VEC * VPL > 8 ? 1 : 2) bal_main_kernel(const BalanceArgs a) {
    constexpr int NV = VEC * VPL, TPW = 32 / LP, WARPS = BAL_THREADS / 32;
    __shared__ __align__(16) float s_c[1024];
    __shared__ int s_hist[1024];
    __shared__ double s_sum[WARPS];
    __shared__ int s_rows[WARPS];
    __shared__ unsigned s_last;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / LP, l = lane % LP;
    auto column = [&](int v, int j) { return (v * LP + l) * VEC + j; };

    // runs that do not ascend within [0, T]; the loads of runs without a token, and, where they are
    // counted in parts, of this CTA's share of all runs
    for (int64_t b = (int64_t)blockIdx.x * BAL_THREADS + threadIdx.x; a.seg && b < a.G; b += (int64_t)gridDim.x * BAL_THREADS) {
        const int x = a.seg[b], y = a.seg[b + 1];
        if (x < 0 || y < x || y > a.T) report(a.st, MOEVIE_ERR_DEVICE, SITE_RUNS, (int)b, y);
    }
    for (int64_t b = blockIdx.x; b < a.G; b += gridDim.x) {
        int64_t r0, r1;
        run_rows(a, b, r0, r1);
        if (a.parts == 0 && r1 > r0) continue;
        for (int e = threadIdx.x; e < a.E; e += BAL_THREADS) {
            int n = 0;
#pragma unroll 16
            for (int p = 0; p < a.parts; ++p) n += a.part[(b * a.parts + p) * a.E + e];
            a.counts[b * a.E + e] = n;
        }
    }

    int64_t lo = 0, hi = a.T;   // rows that lie in some run
    if (a.seg) {
        lo = max((int64_t)a.seg[0], (int64_t)0);
        hi = max(lo, min((int64_t)a.seg[a.G], a.T));
    }
    const double per_row = hi > lo ? (double)a.coef / (double)(hi - lo) : 0.0;
    const int64_t n_rows = hi - lo;
    const int64_t t0 = lo + n_rows * blockIdx.x / gridDim.x, t1 = lo + n_rows * (blockIdx.x + 1) / gridDim.x;
    float dots = 0.f;   // of the tokens of this lane's group
    int rows = 0;
    int64_t b = a.seg && t0 < t1 ? warp_run_of(a.seg, a.G, t0) : 0;
    for (int64_t t = t0; t < t1 && b < a.G; ++b) {
        int64_t r0, r1;
        run_rows(a, b, r0, r1);
        const int64_t end = min(r1, t1);
        if (end <= t) continue;
        __syncthreads();
        if (a.parts == 0) {
            for (int e = threadIdx.x; e < a.E; e += BAL_THREADS) s_hist[e] = 0;
            __syncthreads();
            count_ids(a, r0 * a.k, r1 * a.k, s_hist);
            __syncthreads();
        }
        {   // c of the run: coef / (T k T_b) (E n - k T_b)
            const double scale = per_row / ((double)a.k * (double)(r1 - r0));
            const bool mine = a.parts == 0 && r0 >= t0 && r0 < t1;   // its loads are this CTA's to write
            for (int e = threadIdx.x; e < LP * NV; e += BAL_THREADS) {
                int n = 0;
                if (e < a.E) {
                    if (a.parts == 0) n = s_hist[e];
#pragma unroll 16
                    for (int p = 0; p < a.parts; ++p) n += a.part[(b * a.parts + p) * a.E + e];
                    if (mine) a.counts[b * a.E + e] = n;
                }
                s_c[e] = (float)(scale * (double)((int64_t)a.E * n - (int64_t)a.k * (r1 - r0)));
            }
        }
        __syncthreads();
        float c_reg[NV];   // lanes of more than 8 columns read them from shared memory each time
        if constexpr (NV <= 8) {
#pragma unroll
            for (int i = 0; i < NV; ++i) c_reg[i] = s_c[column(i / VEC, i % VEC)];
        }
        auto c = [&](int i) {
            if constexpr (NV <= 8) return c_reg[i];
            else return s_c[column(i / VEC, i % VEC)];
        };
        for (int64_t tb = t + (int64_t)warp * TPW * TU; tb < end; tb += (int64_t)WARPS * TPW * TU) {
            float x[TU][NV], q[TU][NV];   // logits, then scores; and the scores' slopes over themselves
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                const int64_t tt = tb + u * TPW + sub;
#pragma unroll
                for (int v = 0; v < VPL; ++v) {
                    const bool ok = tt < end && column(v, 0) < a.E;
                    if constexpr (VEC == 4) {
                        float4 f = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                        if (ok) f = *reinterpret_cast<const float4*>(a.s + tt * a.ld_s + column(v, 0));
                        x[u][v * 4] = f.x, x[u][v * 4 + 1] = f.y, x[u][v * 4 + 2] = f.z, x[u][v * 4 + 3] = f.w;
                    } else {
                        x[u][v] = ok ? a.s[tt * a.ld_s + column(v, 0)] : -INFINITY;
                    }
                }
            }
            // e^(x - the row's largest logit), for a softmax; a row without a logit has no probability
            auto soft = [&](int u) {
                float m = -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; ++i) m = fmaxf(m, x[u][i]);
#pragma unroll
                for (int o = LP / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                if (m == -INFINITY) m = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const float d = x[u][i] - m;
                    x[u][i] = d != d ? d : exp_neg(d);   // (infinity - infinity)
                    q[u][i] = 1.f;
                }
            };
            float sums[2 * TU];
            auto add_up = [&]() {
#pragma unroll
                for (int u = 0; u < TU; ++u) {
                    sums[2 * u] = sums[2 * u + 1] = 0.f;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        sums[2 * u] += x[u][i];
                        sums[2 * u + 1] = fmaf(x[u][i], c(i), sums[2 * u + 1]);
                    }
                }
#pragma unroll
                for (int o = LP / 2; o; o >>= 1)
#pragma unroll
                    for (int n = 0; n < 2 * TU; ++n) sums[n] += __shfl_xor_sync(0xffffffffu, sums[n], o);
            };
            if (a.score == MOEVIE_SCORE_SOFTMAX) {
#pragma unroll
                for (int u = 0; u < TU; ++u) soft(u);
                add_up();
            } else {
                float keep[TU][NV];
                bool low = false;
#pragma unroll
                for (int u = 0; u < TU; ++u) {
                    float most = 0.f;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const float v = x[u][i];
                        const float z = exp_neg(-fabsf(v));
                        float r;
                        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + z));
                        keep[u][i] = v;
                        x[u][i] = v >= 0.f ? r : z * r;
                        q[u][i] = v >= 0.f ? z * r : r;
                        most = fmaxf(most, x[u][i]);
                    }
                    low |= !(most > 1e-18f);
                }
                // Sigmoids of a row whose logits all lie below -41 would lose bits, and vanish: there
                // sigmoid(s) is e^s to e^-41 of itself, and the row's probabilities are a softmax.  (The
                // rows of a warp go together; whether it is so for a row goes by its largest logit alone.)
                if (__any_sync(0xffffffffu, low)) {
#pragma unroll
                    for (int u = 0; u < TU; ++u) {
                        float m = -INFINITY;
#pragma unroll
                        for (int i = 0; i < NV; ++i) m = fmaxf(m, keep[u][i]);
#pragma unroll
                        for (int o = LP / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                        if (!(m < -41.f)) continue;
                        const float shift = m == -INFINITY ? 0.f : m;
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            const float d = keep[u][i] - shift;
                            x[u][i] = d != d ? d : exp_neg(d);
                            q[u][i] = 1.f;
                        }
                    }
                }
                add_up();
            }
#pragma unroll
            for (int u = 0; u < TU; ++u) {
                const int64_t tt = tb + u * TPW + sub;
                if (tt >= end) continue;
                float(&p)[NV] = x[u];
                const float inv = sums[2 * u] == 0.f ? 0.f : 1.f / sums[2 * u];
                const float dot = sums[2 * u + 1] * inv;
                if (l == 0) {
                    dots += dot;
                    rows += sums[2 * u] == 0.f ? 0 : 1;
                }
                if (!a.ds) continue;
#pragma unroll
                for (int i = 0; i < NV; ++i) p[i] *= inv * q[u][i] * (c(i) - dot);
                float* out = a.ds + tt * a.ld_ds;
#pragma unroll
                for (int v = 0; v < VPL; ++v) {
                    if (column(v, 0) >= a.E) continue;
                    if constexpr (VEC == 4)
                        *reinterpret_cast<float4*>(out + column(v, 0)) =
                            make_float4(p[v * 4], p[v * 4 + 1], p[v * 4 + 2], p[v * 4 + 3]);
                    else
                        out[column(v, 0)] = p[v];
                }
            }
        }
        t = end;
    }

    // the loss: every CTA's sums, added up in order by the CTA that is done last
    double sum = dots;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        rows += __shfl_xor_sync(0xffffffffu, rows, o);
    }
    if (lane == 0) {
        s_sum[warp] = sum;
        s_rows[warp] = rows;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        rows = 0;
        for (int w = 0; w < WARPS; ++w) sum += s_sum[w], rows += s_rows[w];
        a.cta_sum[blockIdx.x] = make_double2(sum, (double)rows);
        __threadfence();
        s_last = atomicInc(&a.st->bal_ticket, gridDim.x - 1) == gridDim.x - 1;   // back to 0 for the next call
    }
    __syncthreads();
    if (!s_last || warp != 0) return;
    __threadfence();
    double total = 0.0, all = 0.0;
    for (unsigned i = lane; i < gridDim.x; i += 32) {
        total += __ldcg(&a.cta_sum[i].x);
        all += __ldcg(&a.cta_sum[i].y);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, o);
        all += __shfl_xor_sync(0xffffffffu, all, o);
    }
    if (lane == 0) *a.loss = (float)(total + per_row * all);
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
    if (T * k <= BAL_FEW_IDS) return 0;
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
        if (E <= 8) e = run_main<1, 8, 1, 2>(a, s);
        else if (E <= 16) e = run_main<1, 8, 2, 2>(a, s);
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
