// norm_back.cu -- the backward of the steps around the layer in a residual block (norm.cu), sm_103a.
#include "norm.cuh"

namespace mv {

namespace {

// Sums of this thread's 8 columns.
struct Sums {
    P8 v;
    __device__ __forceinline__ Sums() { clear(); }
    __device__ __forceinline__ void clear() { v = p8_of(0.f); }
    __device__ __forceinline__ void add(const P8& x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.p[i] = f2_add(x.p[i], v.p[i]);
    }
    __device__ __forceinline__ void add(const P8& x, const P8& y) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.p[i] = f2_fma(x.p[i], y.p[i], v.p[i]);
    }
    __device__ __forceinline__ void store(float* p) const { st_f32(p, v); }
};

// Of row t, with x1, x2 the normed rows before weight and bias and inv_s their 1 / deviation:
//   dR = dr1 + inv_1 (a - [mean a] - x1 mean(a x1)),   a = du w_pre          (mean a: layer norms)
//   dr = alpha dR,   c = gate w_post dR,   df = inv_2 (c - [mean c] - x2 mean(c x2))
// and, summed over rows,
//   dw_pre = sum du x1, db_pre = sum du, A = sum dR x2, B = sum dR (A, B run by run):
//   dgate = w_post A + b_post B,   dw_post = sum_runs gate A,   db_post = sum_runs gate B.
// Each group of warps leaves its sums in the workspace: dw_pre and db_pre at record gid, A and B
// of run g at record g + gid (along the rows g and gid never fall, so that no two share one).
// Bound by HBM where rows are whole: 65536 x 1664 in fp32 342 us, 6.4 TB/s with one gate.  From checkpoints, whose
// decoding adds a quarter to the instructions, 8192 x 1280 31 us, 4.1 TB/s (54% of the issue slots at 16 warps an
// SM, all that 128 registers a thread leave).
// KIND: what the call has, beside r1, du and dr1: both norms (ALL); f's gate alone, or not even that (PLAIN, the
// layer's output added as it is); or anything (ANY, asked as it goes, at the price of 160 bytes of spills a thread:
// 65536 x 1664 in fp32, first norm 321 us, last join 330, no dr1 461, where both norms take 339).  Q8: r1 and f may be
// checkpoints.
// BIAS: db_pre and B as well.
enum Kind { ANY, ALL, PLAIN };
template <bool F32, bool DUF32, Kind KIND, bool Q8, bool BIAS, bool WIDE>
__global__ void __launch_bounds__(NORM_THREADS, 2) norm_backward_kernel(const NormBwdArgs a) {
    constexpr int PR = F32 ? 2 : 1, PU = DUF32 ? 2 : 1, PIECES = 2 * PR + PU + 2;   // the last: the row's statistics
    extern __shared__ __align__(16) uint8_t s_dyn[];   // Kept, the ring
    __shared__ __align__(16) float s_part[PART_FLOATS];
    pdl_wait();
    RowGroup g = row_group<WIDE>(a.gw, a.ranks, s_part);
    if (a.seg) check_runs(a.seg, a.G, a.T, a.st);
    const int first_col = WIDE ? g.rank * a.span : 0;               // of this CTA's share of a row,
    const int cols = WIDE ? min(a.span, a.d - first_col) : a.d;     // and its columns
    const int col = first_col + (g.wi * 32 + g.lane) * 8;
    const bool act = col - first_col < cols;
    const int64_t gid = WIDE ? blockIdx.x / a.ranks : (int64_t)blockIdx.x * a.groups + g.group;
    if (gid >= a.n_groups) return;   // (whole clusters alike)
    int64_t t0 = first_row(a.T, gid, a.n_groups), t1 = first_row(a.T, gid + 1, a.n_groups);
    clip_rows(a, t0, t1);

    const bool norm = KIND != ANY || a.du != nullptr, has_f = KIND == ALL || a.f != nullptr;
    const bool join = KIND != ANY || a.df != nullptr, has_dr = KIND != ANY || a.dr1 != nullptr;
    const bool post = KIND == ALL || (KIND == ANY && a.post != MOEVIE_NORM_NONE);
    const RowRing<BWD_SLOTS, PIECES> ring(s_dyn + KEPT_BYTES * blockDim.x, cols - g.wi * 256);
    const Operand<F32, false> Dr{a.dr1, nullptr, 0};
    const Operand<F32, Q8> R1{a.r1, a.r1_scale, a.r_q8};
    const Operand<DUF32, false> Du{a.du, nullptr, 0};
    const Operand<false, Q8> Fo{a.f, a.f_scale, a.f_q8};
    const int n = t0 < t1 ? (int)(t1 - t0) : 0, d = a.d;   // rows count from t0
    int64_t at = t0 * d + col;   // of the row in hand
    // Two sets of copies: dr1, du, r1 and the single words, whose slots are free as soon as a row is begun, and f, which
    // is read half-way.  Both sets of a row are under way while the two rows before it are worked on.
    // `on`: rows from the one in hand
    int slot = 0;
    // A row's last piece: the statistics of N_pre (words 0, 1) and, with the second set, of N_post (2, 3), by
    // lane 0; the scales of the warp's two blocks of r1 (4, 5) and of f (6, 7), by lanes 0 and 1, zeros for a block
    // behind the row's end (its codes are zeros, but what lay there before may be a NaN).
    const float2 *st1_at = a.stats_pre + t0, *st2_at = a.stats_post + t0;   // of the row in hand
    const int block = first_col / 128 + g.wi * 2 + g.lane;
    const int scale_bytes = block < a.nb ? 4 : 0;
    const int64_t scale_at = t0 * a.nb + block;
    const float* s1_at = Q8 && g.lane < 2 && a.r_q8 ? a.r1_scale + scale_at : nullptr;
    const float* s2_at = Q8 && g.lane < 2 && a.f_q8 ? a.f_scale + scale_at : nullptr;
    const uint32_t scale_word = (4 + (g.lane >> 4)) * 4;   // r1's; f's two words on
    auto copy_first = [&](int to, int i, int on) {
        const bool live = i + on < n;
        if (has_dr) Dr.copy(ring, to, 0, at + on * d, live);
        if (norm) {
            Du.copy(ring, to, PR, at + on * d, live);
            R1.copy(ring, to, PR + PU, at + on * d, live);
        }
        const uint32_t words = ring.at(to, PIECES - 1);
        if (norm && g.lane == 0) copy8(words, st1_at + on, live ? 8 : 0);
        if (Q8 && s1_at) copy4(words + 16 + g.lane * 4, s1_at + on * a.nb, live ? scale_bytes : 0);
    };
    auto copy_second = [&](int to, int i, int on) {
        const bool live = i + on < n;
        if (has_f) Fo.copy(ring, to, 2 * PR + PU, at + on * d, live);
        const uint32_t words = ring.at(to, PIECES - 1);
        if (post && g.lane == 0) copy8(words + 8, st2_at + on, live ? 8 : 0);
        if (Q8 && s2_at) copy4(words + 24 + g.lane * 4, s2_at + on * a.nb, live ? scale_bytes : 0);
    };
    copy_first(0, 0, 0);
    copy_first(1, 0, 1);
    cp_async_commit();
    copy_second(0, 0, 0);
    copy_second(1, 0, 1);
    cp_async_commit();

    const float inv_d = 1.0f / (float)d;
    const Kept w1(s_dyn, 0), cw(s_dyn, 1);   // cw: gate * weight
    w1.set(ld_param(a.w_pre, col, act, 1.f));
    Sums sw, sb, sA, sB;   // dw_pre, db_pre, A, B
    int64_t run = 0;
    int run_end = n;

    auto flush_run = [&]() {
        if (!a.rec_post || !act) return;
        float* p = a.rec_post + (run + gid) * 2 * d + col;
        sA.store(p);
        if (BIAS) sB.store(p + d);
        sA.clear();
        sB.clear();
    };
    auto load_run = [&]() {
        if (!join) return;
        const P8 gt = ld_param(a.gate ? a.gate + run * d : nullptr, col, act, 1.f);
        P8 w = ld_param(a.w_post, col, act, 1.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) w.p[j] = f2_mul(w.p[j], gt.p[j]);
        cw.set(w);
    };
    // the end of a run, counted from t0: the last one's rows go to the group's end
    auto end_of_run = [&]() { return run + 1 < a.G ? (int)(min((int64_t)a.seg[run + 1], t1) - t0) : n; };
    if (n > 0) {
        if (a.seg) {
            run = warp_run_of(a.seg, a.G, t0);
            run_end = end_of_run();
        }
        load_run();
    }
    const int64_t first_run = run;
    if (WIDE || g.gw > 1) row_barrier<WIDE>(g);   // the zeros of row_group; the cluster's CTAs are there

#pragma unroll 1
    for (int i = 0; i < n;) {
        if (i >= run_end) {
            do {   // runs without rows get zeros
                flush_run();
                ++run;
            } while (run + 1 < a.G && a.seg[run + 1] <= t0 + i);
            run_end = end_of_run();
            load_run();
        }
        // rows i and, of the same run, i + 1
        const bool two = i + 1 < run_end;
        P8 dR[ROWS], x1[ROWS], du[ROWS], x2[ROWS];
        float2 st1[ROWS], st2[ROWS];
        cp_async_wait<1>();
        __syncwarp();   // the other lanes' copies
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint32_t words = ring.at(slot ^ k, PIECES - 1);
            if (has_dr) dR[k] = Dr.get(ring, slot ^ k, 0, 0);
            else dR[k] = p8_of(0.f);
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(st1[k].x), "=f"(st1[k].y) : "r"(words) : "memory");
            if (norm) {
                x1[k] = Q8 ? R1.normed(ring, slot ^ k, PR + PU, words + scale_word, st1[k])
                           : R1.get(ring, slot ^ k, PR + PU, 0);
                du[k] = Du.get(ring, slot ^ k, PR, 0);
            }
        }
        __syncwarp();   // read by all lanes
        copy_first(slot, i, 2);
        if (two) copy_first(slot ^ 1, i, 3);
        cp_async_commit();
        if (!two) {   // i + 1 is not of this run: nothing of it counts here
            dR[ROWS - 1] = x1[ROWS - 1] = du[ROWS - 1] = p8_of(0.f);
            st1[ROWS - 1] = make_float2(0.f, 0.f);
        }
        if (norm) {
            float s[2 * ROWS];
            const P8 w = w1.get();
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {   // behind the row's end du and dR are zeros
                if (!Q8) normed(x1[k], st1[k]);   // (no earlier: 65536 x 1664 in fp32 343 us, earlier 357)
                sw.add(du[k], x1[k]);
                if (BIAS) sb.add(du[k]);
#pragma unroll
                for (int j = 0; j < 4; ++j) du[k].p[j] = f2_mul(du[k].p[j], w.p[j]);
                s[2 * k] = p8_sum(du[k]);
                s[2 * k + 1] = p8_dot(du[k], x1[k]);
            }
            row_sum<WIDE>(g, s);
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t m0 = f2_of(a.pre == MOEVIE_NORM_LAYER ? -s[2 * k] * inv_d : 0.f);
                const uint64_t m1 = f2_of(-s[2 * k + 1] * inv_d), q = f2_of(st1[k].y);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    dR[k].p[j] = f2_fma(q, f2_fma(x1[k].p[j], m1, f2_add(du[k].p[j], m0)), dR[k].p[j]);
            }
        }
        const uint64_t al = f2_of(a.alpha);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            P8 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.p[j] = f2_mul(al, dR[k].p[j]);
            if (act && (k == 0 || two)) st_rows<F32>(a.dr, at + k * d, o);
        }
        cp_async_wait<1>();
        __syncwarp();   // the other lanes' words
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint32_t words = ring.at(slot ^ k, PIECES - 1) + 8;
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(st2[k].x), "=f"(st2[k].y) : "r"(words) : "memory");
            if (Q8 && post) x2[k] = Fo.normed(ring, slot ^ k, 2 * PR + PU, words + scale_word, st2[k]);
            else if (has_f) x2[k] = Fo.get(ring, slot ^ k, 2 * PR + PU, words + scale_word);
            else x2[k] = p8_of(0.f);
        }
        __syncwarp();
        copy_second(slot, i, 2);
        if (two) copy_second(slot ^ 1, i, 3);
        cp_async_commit();
        if (!two) {
            x2[ROWS - 1] = p8_of(0.f);
            st2[ROWS - 1] = make_float2(0.f, 0.f);
            slot ^= 1;
        }
        if (join) {
            const P8 w = cw.get();
            if (post) {
                float s[2 * ROWS];
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    if (!Q8) normed(x2[k], st2[k]);
                    sA.add(dR[k], x2[k]);
                    if (BIAS) sB.add(dR[k]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) dR[k].p[j] = f2_mul(dR[k].p[j], w.p[j]);   // (zeros behind the row's end)
                    s[2 * k] = p8_sum(dR[k]);
                    s[2 * k + 1] = p8_dot(dR[k], x2[k]);
                }
                row_sum<WIDE>(g, s);
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const uint64_t m0 = f2_of(a.post == MOEVIE_NORM_LAYER ? -s[2 * k] * inv_d : 0.f);
                    const uint64_t m1 = f2_of(-s[2 * k + 1] * inv_d), q = f2_of(st2[k].y);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        dR[k].p[j] = f2_mul(q, f2_fma(x2[k].p[j], m1, f2_add(dR[k].p[j], m0)));
                }
            } else {
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    sA.add(dR[k], x2[k]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) dR[k].p[j] = f2_mul(dR[k].p[j], w.p[j]);
                }
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (act && (k == 0 || two)) st_bf16(a.df + at + k * d, dR[k]);
        }
        i += two ? 2 : 1;
        at += two ? 2 * d : d;
        st1_at += two ? 2 : 1;
        st2_at += two ? 2 : 1;
        if (Q8 && s1_at) s1_at += two ? 2 * a.nb : a.nb;
        if (Q8 && s2_at) s2_at += two ? 2 * a.nb : a.nb;
    }
    if (n > 0 || a.G == 1) flush_run();   // a group without rows leaves zeros where only one run is
    if (a.group_runs && g.rank == 0 && g.wi == 0 && g.lane == 0)
        a.group_runs[gid] = n > 0 ? make_int2((int)first_run, (int)run) : make_int2(0, -1);
    if (a.rec_pre && act) {
        float* p = a.rec_pre + gid * 2 * a.d + col;
        sw.store(p);
        if (BIAS) sb.store(p + a.d);
    }
}

// The records of norm_backward_kernel added up, in a fixed order, by CTAs of 32 x 32 threads that take
// 32 columns each.  blockIdx.y: 0 dw_pre and db_pre; 1 dw_post and db_post (and dgate, where there is
// one run); 2 and on dgate of several runs, 32 / lanes runs to a CTA.  Rows of threads share the
// records out (of a run: `lanes` rows).
__global__ void __launch_bounds__(1024) norm_sums_kernel(const NormSumArgs a, int lanes) {
    __shared__ float s_a[32][33], s_b[32][33];
    pdl_wait();
    const int x = threadIdx.x, y = threadIdx.y;
    const int col = blockIdx.x * 32 + x;
    const bool act = col < a.d, pre = blockIdx.y == 0;
    const int64_t row = 2 * (int64_t)a.d;   // floats of a record
    const float* rec = pre ? a.rec_pre : a.rec_post;
    if (!rec) return;
    rec += col;
    float va = 0.f, vb = 0.f;
    int64_t run = 0;   // of this thread, for dgate
    if (blockIdx.y >= 2) {
        run = (int64_t)(blockIdx.y - 2) * (32 / lanes) + y / lanes;
        if (act && run < a.G) {
            const int64_t r0 = max((int64_t)a.seg[run], (int64_t)0), r1 = min((int64_t)a.seg[run + 1], a.T);
            if (r0 < r1) {
                const int64_t hi = group_of(a.T, r1 - 1, a.n_groups);
                const float* p = rec + run * row;
#pragma unroll 4
                for (int64_t i = group_of(a.T, r0, a.n_groups) + y % lanes; i <= hi; i += lanes) {
                    va += p[i * row];
                    if (a.bias) vb += p[i * row + a.d];
                }
            }
        }
    } else if (act) {
        if (pre || a.G == 1) {
#pragma unroll 8
            for (int64_t i = y; i < a.n_groups; i += 32) {
                va += rec[i * row];
                if (a.bias) vb += rec[i * row + a.d];
            }
        } else {   // each record by the gate of its run
            const float* gate = a.gate ? a.gate + col : nullptr;
            for (int64_t i = y; i < a.n_groups; i += 4 * 32) {
                int2 runs[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    runs[u] = i + 32 * u < a.n_groups ? a.group_runs[i + 32 * u] : make_int2(0, -1);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (runs[u].x > runs[u].y) continue;
                    const int64_t g = runs[u].x;
                    const float* p = rec + (g + i + 32 * u) * row;
                    const float gt = gate ? gate[g * a.d] : 1.f;
                    va = fmaf(gt, p[0], va);
                    if (a.bias) vb = fmaf(gt, p[a.d], vb);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    for (int64_t g = (int64_t)runs[u].x + 1; g <= runs[u].y; ++g) {
                        const float* p = rec + (g + i + 32 * u) * row;
                        const float gt = gate ? gate[g * a.d] : 1.f;
                        va = fmaf(gt, p[0], va);
                        if (a.bias) vb = fmaf(gt, p[a.d], vb);
                    }
            }
        }
    }
    const int share = blockIdx.y >= 2 ? lanes : 32;   // rows of threads to one result
    if (share > 1) {
        s_a[y][x] = va;
        s_b[y][x] = vb;
        __syncthreads();
        if (y % share != 0) return;
        va = vb = 0.f;
#pragma unroll 8
        for (int i = 0; i < share; ++i) va += s_a[y + i][x], vb += s_b[y + i][x];
    }
    if (!act || run >= a.G) return;
    if (pre) {
        if (a.dw_pre) a.dw_pre[col] = va;
        if (a.db_pre) a.db_pre[col] = vb;
        return;
    }
    if (blockIdx.y == 1) {
        const float gt = a.G == 1 && a.gate ? a.gate[col] : 1.f;
        if (a.dw_post) a.dw_post[col] = gt * va;
        if (a.db_post) a.db_post[col] = gt * vb;
        if (a.G > 1) return;
    }
    if (a.dgate)
        a.dgate[run * a.d + col] = fmaf(a.w_post ? a.w_post[col] : 1.f, va, (a.b_post ? a.b_post[col] : 0.f) * vb);
}

}  // namespace

int64_t norm_groups(int64_t T, int d) {
    return std::max<int64_t>(1, norm_plan(T, d, NORM_BWD_THREADS, true).n_groups);
}

template <bool F32, bool DUF32, Kind KIND, bool Q8, bool BIAS, bool WIDE>
static cudaError_t norm_backward(NormBwdArgs& a, cudaStream_t s) {
    static RowsKernel k;
    return launch_rows<false>(norm_backward_kernel<F32, DUF32, KIND, Q8, BIAS, WIDE>, k, true, NORM_BWD_THREADS,
                              KEPT_BYTES + 16 * BWD_SLOTS * (2 * (F32 ? 2 : 1) + (DUF32 ? 2 : 1) + 2), s, a);
}
template <bool F32, bool DUF32, bool WIDE>
static cudaError_t norm_backward(NormBwdArgs& a, bool bias, cudaStream_t s) {
    const bool q8 = a.r_q8 || a.f_q8;
    if (a.du && a.dr1 && a.df && a.post == MOEVIE_NORM_NONE)
        return bias || WIDE ? norm_backward<F32, DUF32, PLAIN, true, true, WIDE>(a, s)
                            : norm_backward<F32, DUF32, PLAIN, true, false, WIDE>(a, s);
    if (!a.du || !a.dr1 || !a.df || !a.f) return norm_backward<F32, DUF32, ANY, true, true, WIDE>(a, s);
    if (q8)
        return bias ? norm_backward<F32, DUF32, ALL, true, true, WIDE>(a, s)
                    : norm_backward<F32, DUF32, ALL, true, false, WIDE>(a, s);
    return bias ? norm_backward<F32, DUF32, ALL, false, true, WIDE>(a, s)
                : norm_backward<F32, DUF32, ALL, false, false, WIDE>(a, s);
}
template <bool F32, bool DUF32>
static cudaError_t norm_backward(NormBwdArgs& a, bool bias, cudaStream_t s) {
    return a.d > 2048 ? norm_backward<F32, DUF32, true>(a, bias, s) : norm_backward<F32, DUF32, false>(a, bias, s);
}

cudaError_t launch_norm_backward(NormBwdArgs a, int r_f32, int du_f32, NormSumArgs sums, cudaStream_t s) {
    cudaError_t e;
    const bool bias = sums.db_pre || sums.db_post || (sums.dgate && sums.b_post);
    sums.bias = bias;
    if (r_f32) e = du_f32 ? norm_backward<true, true>(a, bias, s) : norm_backward<true, false>(a, bias, s);
    else e = du_f32 ? norm_backward<false, true>(a, bias, s) : norm_backward<false, false>(a, bias, s);
    count_launches(1);
    if (e != cudaSuccess || (!a.rec_pre && !a.rec_post)) return e;
    sums.n_groups = a.n_groups;
    int64_t gates = 0;   // CTAs of a column block for dgate of several runs
    int lanes = 1;
    if (sums.G > 1 && sums.dgate) {
        while (lanes < 32 && a.n_groups / sums.G >= 4 * lanes) lanes *= 2;   // a few records to a thread
        gates = (sums.G + 32 / lanes - 1) / (32 / lanes);
        if (gates > 65533) return cudaErrorInvalidValue;
    }
    e = launch_pdl(norm_sums_kernel, dim3((unsigned)((a.d + 31) / 32), (unsigned)(2 + gates)), dim3(32, 32), 0, s, sums, lanes);
    count_launches(1);
    return e;
}

}  // namespace mv
