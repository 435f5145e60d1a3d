// norm.cu -- the steps around the layer in a residual block, forward (the backward: norm_back.cu), and
// activation checkpoints in 8 bits, sm_103a.
//
//   r1 = alpha r + gate * N_post(f),   u = N_pre(r1)
//
// with N an RMS or layer norm over a row's d columns.  A row's operands are read once, its results written
// once, and all arithmetic is fp32.  One thread owns 8 columns (16 bytes of bf16, 32 of fp32), ceil(d / 256) warps
// own a row, and a group of such warps walks a contiguous range of rows, so that weights, the gate and the sums of
// the weights' gradients stay on chip over the whole range.  Measured, bytes that have to move over the time:
// forward of 65536 x 1664 in fp32 6.4 TB/s, bound by HBM (95% of a plain copy's rate); of 8192 x 1024 in bf16 with
// two checkpoints 3.7 TB/s (36 us), bound by the instructions, of which the codes are more than half, and their
// latency: 60% of the issue slots at a third of the warps an SM could hold.
#include "norm.cuh"

namespace mv {

namespace {

// Blocks of 128 columns (the last one of a row may be shorter), 16 threads each; a thread takes
// UNITS blocks at a time, their loads under way together.  Blocks are counted row by row; the ones
// of a thread are `step` apart = step_rows rows and step_blocks blocks.  4 blocks to a thread; rows
// written as bf16 take 2 (32768 x 1536: read back in 25.7 us instead of 27.2, kept in 34.6 instead of 32.7).
// 65536 x 1664 in fp32: kept at 6.8 TB/s, read back (mostly writes) at 5.8; 32768 x 1536 in bf16: 4.7 (60% of
// the issue slots) and 5.9.
constexpr int Q8_UNITS = 4, Q8_LOAD16_UNITS = 2;

struct BlockWalk {
    int64_t u, at;   // the block's number, and this thread's first element of it
    int block;       // its place in its row
    __device__ __forceinline__ BlockWalk(int nb, int d) {
        u = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
        const int64_t row = u / nb;
        block = (int)(u - row * nb);
        at = row * d + block * 128 + (threadIdx.x & 15) * 8;
    }
    // step blocks on: step_at elements and step_blocks places, or so much less a row's
    __device__ __forceinline__ void advance(int64_t step, int64_t step_at, int step_blocks, int nb, int d) {
        u += step;
        at += step_at;
        block += step_blocks;
        if (block >= nb) {
            block -= nb;
            at += d - nb * 128;
        }
    }
    __device__ __forceinline__ bool in_row(int d) const { return block * 128 + (int)(threadIdx.x & 15) * 8 < d; }
};

template <bool F32>
__global__ void __launch_bounds__(256, F32 ? 3 : 4) q8_store_kernel(const void* x, int64_t blocks, int d, int nb, int64_t step_at,
                                                          int step_blocks, int8_t* codes, float* scales) {
    pdl_wait();
    const int64_t step = (int64_t)gridDim.x * 16;
    BlockWalk w(nb, d);
    // a warp's two blocks leave the loop together: its shuffles need both
    while (__any_sync(0xffffffffu, w.u < blocks)) {
        uint4 lo[Q8_UNITS], hi[Q8_UNITS];
        BlockWalk r = w;
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            lo[n] = hi[n] = make_uint4(0u, 0u, 0u, 0u);
            if (r.u < blocks && r.in_row(d)) {
                if constexpr (F32) {
                    lo[n] = ld16(static_cast<const float*>(x) + r.at);
                    hi[n] = ld16(static_cast<const float*>(x) + r.at + 4);
                } else {
                    lo[n] = ld16(static_cast<const __nv_bfloat16*>(x) + r.at);
                }
            }
            r.advance(step, step_at, step_blocks, nb, d);
        }
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            float scale;
            const uint2 c = q8_block(F32 ? p8_f32(lo[n], hi[n]) : p8_bf16(lo[n]), scale);
            if (w.u < blocks) {
                if (w.in_row(d)) *reinterpret_cast<uint2*>(codes + w.at) = c;
                if ((threadIdx.x & 15) == 0) scales[w.u] = scale;
            }
            w.advance(step, step_at, step_blocks, nb, d);
        }
    }
}

template <bool F32>
__global__ void __launch_bounds__(256) q8_load_kernel(const int8_t* codes, const float* scales, int64_t blocks, int d,
                                                      int nb, int64_t step_at, int step_blocks, void* x) {
    constexpr int UNITS = F32 ? Q8_UNITS : Q8_LOAD16_UNITS;
    pdl_wait();
    const int64_t step = (int64_t)gridDim.x * 16;
    BlockWalk w(nb, d);
    while (w.u < blocks) {
        uint2 c[UNITS];
        float scale[UNITS];
        BlockWalk r = w;
#pragma unroll
        for (int n = 0; n < UNITS; ++n) {
            if (r.u < blocks && r.in_row(d)) {
                c[n] = ld8(codes + r.at);
                scale[n] = scales[r.u];
            }
            r.advance(step, step_at, step_blocks, nb, d);
        }
#pragma unroll
        for (int n = 0; n < UNITS; ++n) {
            if (w.u < blocks && w.in_row(d)) st_rows<F32>(x, w.at, p8_codes(c[n].x, c[n].y, scale[n]));
            w.advance(step, step_at, step_blocks, nb, d);
        }
    }
}

// ------------------------------------------------------------ forward

// JOIN: r1 = alpha r + gate * N_post(f), and its norm; otherwise the norm of r alone.  BOTH: a join with
// both norms and their statistics (the others ask as they go).  SAVE: 8-bit checkpoints of what is read.
// BIG: rows of more than 2048 columns, by CTAs of up to 1024 threads of 64 registers, a row at a time (over
// the CTAs of a cluster, as in the backward, its up to four barriers a row cost more: 8192 x 4096 bf16 135 us
// instead of 70).
template <bool F32, bool JOIN, bool BOTH, bool SAVE, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : NORM_THREADS, BIG ? 1 : norm_more(F32, SAVE) ? 3 : 2)
norm_forward_kernel(const NormArgs a) {
    constexpr int ROWS = BIG ? 1 : mv::ROWS, SLOTS = fwd_slots(F32, BIG), PR = F32 ? 2 : 1, PIECES = PR + (JOIN ? 1 : 0);
    extern __shared__ __align__(16) uint8_t s_dyn[];
    __shared__ __align__(16) float s_part[PART_FLOATS];
    pdl_wait();
    RowGroup g = row_group<false>(a.gw, 1, s_part);
    if (a.seg) check_runs(a.seg, a.G, a.T, a.st);
    const int col = (g.wi * 32 + g.lane) * 8;
    const bool act = col < a.d;
    const int64_t gid = (int64_t)blockIdx.x * a.groups + g.group;
    if (gid >= a.n_groups) return;
    int64_t t0 = first_row(a.T, gid, a.n_groups), t1 = first_row(a.T, gid + 1, a.n_groups);
    clip_rows(a, t0, t1);
    if (t0 >= t1) return;

    const RowRing<SLOTS, PIECES> ring(s_dyn + (BIG ? 1 : 2) * KEPT_BYTES * blockDim.x, a.d - g.wi * 256);
    const Operand<F32, !JOIN> R{a.r, a.r_scale, a.r_q8};
    const Operand<false, false> Fo{a.f, nullptr, 0};
    const int n = (int)(t1 - t0), d = a.d;
    int slot = 0, fill = 0, ahead = 0;   // rows count from t0
    int64_t at_ahead = t0 * d + col, sat_ahead = t0 * a.nb + (col >> 7);
    auto copy_row = [&]() {   // of row `ahead`
        const bool live = ahead < n;
        R.copy(ring, fill, 0, at_ahead, live);
        if constexpr (JOIN) Fo.copy(ring, fill, PR, at_ahead, live);
        if (!JOIN && a.r_q8) copy4(ring.at(fill, 0) + 256 + g.lane * 4, a.r_scale + sat_ahead, live && act ? 4 : 0);
        cp_async_commit();
        fill = ring.next(fill);
        ++ahead;
        at_ahead += d;
        if (!JOIN) sat_ahead += a.nb;
    };
#pragma unroll 1
    for (int i = 0; i < SLOTS; ++i) copy_row();

    const float inv_d = 1.0f / (float)d;
    const Kept w1(s_dyn, 0), b1(s_dyn, 1);
    w1.set(ld_param(a.w_pre, col, act, 1.f));
    b1.set(ld_param(a.b_pre, col, act, 0.f));
    const Kept w2(s_dyn, BIG ? 0 : 2), b2(s_dyn, BIG ? 1 : 3);   // gate * weight, gate * bias
    P8 w2_reg = p8_of(0.f), b2_reg = p8_of(0.f);                   // BIG: in registers, shared memory is full
    int64_t run = -1;
    int run_end = 0;
    const bool first = g.wi == 0 && g.lane == 0;
    float2 *const stats_pre = a.stats_pre + t0, *const stats_post = a.stats_post + t0;
    int64_t at = t0 * d + col;
    if (g.gw > 1) row_barrier<false>(g);   // the zeros of row_group

#pragma unroll 1
    for (int i = 0; i < n;) {
        if (JOIN && i >= run_end) {   // the next run's gate, times the norm's weight and bias
            run_end = n;
            if (a.seg) {
                const int64_t t = t0 + i;
                run = run < 0 ? warp_run_of(a.seg, a.G, t) : run + 1;
                while (run + 1 < a.G && a.seg[run + 1] <= t) ++run;
                run_end = (int)(min((int64_t)a.seg[run + 1], t1) - t0);
            } else {
                run = 0;
            }
            const P8 gt = ld_param(a.gate ? a.gate + run * d : nullptr, col, act, 1.f);
            w2_reg = ld_param(a.w_post, col, act, 1.f);
            b2_reg = ld_param(a.b_post, col, act, 0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w2_reg.p[j] = f2_mul(w2_reg.p[j], gt.p[j]), b2_reg.p[j] = f2_mul(b2_reg.p[j], gt.p[j]);
            if (!BIG) w2.set(w2_reg), b2.set(b2_reg);
        }
        // rows i and, of the same run, i + 1
        const bool two = ROWS == 2 && i + 1 < (JOIN ? run_end : n);
        cp_async_wait<SLOTS - ROWS>();
        __syncwarp();   // the other lanes' copies
        P8 r[ROWS], x[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int from = k ? ring.next(slot) : slot;
            r[k] = R.get(ring, from, 0, ring.at(from, 0) + 256 + g.lane * 4);
            if constexpr (JOIN) x[k] = Fo.get(ring, from, PR, 0);
        }
        slot = ring.next(slot);
        __syncwarp();   // read by all lanes
        copy_row();
        if (two) {
            slot = ring.next(slot);
            copy_row();
        }
        if constexpr (SAVE) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const bool live = act && (k == 0 || two);
                const int64_t sat = (t0 + i + k) * a.nb + (col >> 7);
                if (a.qr) {
                    float scale;
                    const uint2 c = q8_block(r[k], scale);
                    if (live) *reinterpret_cast<uint2*>(a.qr + at + k * d) = c;
                    if (live && (g.lane & 15) == 0) a.qr_scale[sat] = scale;
                }
                if (JOIN && a.qf) {
                    float scale;
                    const uint2 c = q8_block(x[k], scale);
                    if (live) *reinterpret_cast<uint2*>(a.qf + at + k * d) = c;
                    if (live && (g.lane & 15) == 0) a.qf_scale[sat] = scale;
                }
            }
        }
        float2 st[ROWS];
        if constexpr (JOIN) {
            if (BOTH || a.post != MOEVIE_NORM_NONE) {
                row_stats(g, x, act, a.post, inv_d, a.eps, st);
                if ((BOTH || a.stats_post) && first) {
                    stats_post[i] = st[0];
                    if (two) stats_post[i + 1] = st[ROWS - 1];
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const uint64_t q = f2_of(st[k].y);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[k].p[j] = f2_mul(x[k].p[j], q);
                }
            }
            const uint64_t al = f2_of(a.alpha);
            if (!BIG) w2_reg = w2.get(), b2_reg = b2.get();
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    r[k].p[j] = f2_fma(al, r[k].p[j], f2_fma(x[k].p[j], w2_reg.p[j], b2_reg.p[j]));
                if (act && (k == 0 || two)) st_rows<F32>(a.r_out, at + k * d, r[k]);
            }
        }
        if (BOTH || a.u) {
            row_stats(g, r, act, a.pre, inv_d, a.eps, st);
            if ((BOTH || a.stats_pre) && first) {
                stats_pre[i] = st[0];
                if (two) stats_pre[i + 1] = st[ROWS - 1];
            }
            const P8 w = w1.get(), b = b1.get();
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t q = f2_of(st[k].y);
#pragma unroll
                for (int j = 0; j < 4; ++j) r[k].p[j] = f2_fma(f2_mul(r[k].p[j], q), w.p[j], b.p[j]);
                if (act && (k == 0 || two)) st_bf16(a.u + at + k * d, r[k]);
            }
        }
        i += two ? 2 : 1;
        at += two ? 2 * d : d;
    }
}

// Grid of the checkpoint kernels and the step of their walk over the blocks, CTAs_SM to an SM at most.
struct BlockPlan {
    int nb, grid, step_blocks;
    int64_t blocks, step_at;
    BlockPlan(int64_t T, int d, int ctas_sm, int units) : nb((d + 127) / 128), blocks(T * nb) {
        grid = (int)std::min<int64_t>((blocks + 16 * units - 1) / (16 * units), (int64_t)GB300_SMS * ctas_sm);
        const int64_t step = (int64_t)grid * 16;
        step_blocks = (int)(step % nb);
        step_at = step / nb * d + step_blocks * 128;
    }
};
template <bool F32>
cudaError_t q8_store(const void* x, int64_t T, int d, int8_t* codes, float* scales, cudaStream_t s) {
    const BlockPlan p(T, d, F32 ? 3 : 4, Q8_UNITS);
    return launch_pdl(q8_store_kernel<F32>, dim3(p.grid), dim3(256), 0, s, x, p.blocks, d, p.nb, p.step_at,
                      p.step_blocks, codes, scales);
}
template <bool F32>
cudaError_t q8_load(const int8_t* codes, const float* scales, int64_t T, int d, void* x, cudaStream_t s) {
    const BlockPlan p(T, d, 6, F32 ? Q8_UNITS : Q8_LOAD16_UNITS);
    return launch_pdl(q8_load_kernel<F32>, dim3(p.grid), dim3(256), 0, s, codes, scales, p.blocks, d, p.nb, p.step_at,
                      p.step_blocks, x);
}

}  // namespace

cudaError_t launch_q8_store(const void* x, int x_f32, int64_t T, int d, int8_t* codes, float* scales, cudaStream_t s) {
    const cudaError_t e = x_f32 ? q8_store<true>(x, T, d, codes, scales, s) : q8_store<false>(x, T, d, codes, scales, s);
    count_launches(1);
    return e;
}

cudaError_t launch_q8_load(const int8_t* codes, const float* scales, int64_t T, int d, void* x, int x_f32,
                           cudaStream_t s) {
    const cudaError_t e = x_f32 ? q8_load<true>(codes, scales, T, d, x, s) : q8_load<false>(codes, scales, T, d, x, s);
    count_launches(1);
    return e;
}

template <bool F32, bool JOIN, bool BOTH, bool SAVE, bool BIG>
static cudaError_t norm_forward(NormArgs& a, cudaStream_t s) {
    static RowsKernel k;
    return launch_rows<BIG>(norm_forward_kernel<F32, JOIN, BOTH, SAVE, BIG>, k, false,
                            BIG ? NORM_BIG_THREADS : norm_more(F32, SAVE) ? NORM_MORE_THREADS : NORM_FWD_THREADS,
                            (BIG ? 1 : 2) * KEPT_BYTES + 16 * fwd_slots(F32, BIG) * ((F32 ? 2 : 1) + (JOIN ? 1 : 0)), s, a);
}
template <bool F32, bool JOIN, bool SAVE>
static cudaError_t norm_forward(NormArgs& a, cudaStream_t s) {
    if (a.d > 2048) return norm_forward<F32, JOIN, false, SAVE, true>(a, s);
    if (JOIN && a.post != MOEVIE_NORM_NONE && a.u && a.stats_pre && a.stats_post)
        return norm_forward<F32, JOIN, JOIN, SAVE, false>(a, s);
    return norm_forward<F32, JOIN, false, SAVE, false>(a, s);
}
template <bool F32>
static cudaError_t norm_forward(NormArgs& a, cudaStream_t s) {
    const bool save = a.qr || a.qf;
    if (!a.f) return save ? norm_forward<F32, false, true>(a, s) : norm_forward<F32, false, false>(a, s);
    return save ? norm_forward<F32, true, true>(a, s) : norm_forward<F32, true, false>(a, s);
}

cudaError_t launch_norm_forward(NormArgs a, int r_f32, cudaStream_t s) {
    const cudaError_t e = r_f32 ? norm_forward<true>(a, s) : norm_forward<false>(a, s);
    count_launches(1);
    return e;
}

}  // namespace mv
