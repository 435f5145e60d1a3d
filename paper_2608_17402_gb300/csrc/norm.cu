// norm.cu -- the steps around the layer in a residual block, forward and backward, and activation
// checkpoints in 8 bits, sm_103a.
//
//   r1 = alpha r + gate * N_post(f),   u = N_pre(r1)
//
// with N an RMS or layer norm over a row's d columns.  Every kernel here is bound by HBM: a row's
// operands are read once, its results written once, and all arithmetic is fp32.  One thread owns 8
// columns (16 bytes of bf16, 32 of fp32), ceil(d / 256) warps own a row, and a group of such warps
// walks a contiguous range of rows, so that weights, the gate and the sums of the weights'
// gradients stay in registers over the whole range.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "internal.h"

namespace mv {

namespace {

constexpr int MAX_GROUPS = 8;      // row groups of a CTA
constexpr float Q8_LEAST = 7.70371978e-34f;   // 2^-110: blocks of smaller values are kept as zeros

// ------------------------------------------------------------ rows of 8 columns

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 r;
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "l"(p));
    return r;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
    uint2 r;
    asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
    return r;
}
// 8 fp32 values; rows start 16 bytes apart
__device__ __forceinline__ void ld_f8(const float* p, float (&v)[8]) {
    const uint4 a = ld16(p), b = ld16(p + 4);
    v[0] = __uint_as_float(a.x), v[1] = __uint_as_float(a.y), v[2] = __uint_as_float(a.z), v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x), v[5] = __uint_as_float(b.y), v[6] = __uint_as_float(b.z), v[7] = __uint_as_float(b.w);
}
__device__ __forceinline__ void st_f8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void st_b8(__nv_bfloat16* p, const float (&v)[8]) {
    uint4 u;
    u.x = pack_bf16x2(v[0], v[1]);
    u.y = pack_bf16x2(v[2], v[3]);
    u.z = pack_bf16x2(v[4], v[5]);
    u.w = pack_bf16x2(v[6], v[7]);
    *reinterpret_cast<uint4*>(p) = u;
}
// n values of an optional vector (NULL: `other` everywhere)
__device__ __forceinline__ void ld_param(const float* p, int col, bool act, float other, float (&v)[8]) {
    if (p && act) {
        ld_f8(p + col, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = other;
    }
}

// 8 columns as they lie in memory: bf16 (raw.x .. w), fp32 (all of it) or codes (raw.x, raw.y) with
// their block's scale.
template <bool F32>
struct Raw;
template <>
struct Raw<false> {
    uint4 a;
    float scale;
};
template <>
struct Raw<true> {
    uint4 a, b;
    float scale;
};

template <bool F32>
__device__ __forceinline__ void ld_whole(const void* base, int64_t at, Raw<F32>& raw) {
    if constexpr (F32) {
        const float* p = static_cast<const float*>(base) + at;
        raw.a = ld16(p);
        raw.b = ld16(p + 4);
    } else {
        raw.a = ld16(static_cast<const __nv_bfloat16*>(base) + at);
    }
}
template <bool F32>
__device__ __forceinline__ void ld_codes(const void* base, int64_t at, const float* scale, int64_t sat, Raw<F32>& raw) {
    const uint2 c = ld8(static_cast<const int8_t*>(base) + at);
    raw.a.x = c.x;
    raw.a.y = c.y;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(raw.scale) : "l"(scale + sat));
}
template <bool F32>
__device__ __forceinline__ void whole_values(const Raw<F32>& raw, float (&v)[8]) {
    if constexpr (F32) {
        v[0] = __uint_as_float(raw.a.x), v[1] = __uint_as_float(raw.a.y);
        v[2] = __uint_as_float(raw.a.z), v[3] = __uint_as_float(raw.a.w);
        v[4] = __uint_as_float(raw.b.x), v[5] = __uint_as_float(raw.b.y);
        v[6] = __uint_as_float(raw.b.z), v[7] = __uint_as_float(raw.b.w);
    } else {
        unpack_bf16x8(raw.a, v);
    }
}
__device__ __forceinline__ void code_values(uint32_t lo, uint32_t hi, float scale, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (float)(int8_t)(lo >> (8 * i)) * scale;
        v[4 + i] = (float)(int8_t)(hi >> (8 * i)) * scale;
    }
}

// ------------------------------------------------------------ 8-bit checkpoints

// The whole number nearest to 127 x / amax, an even one between two.  y is that value in fp32, off
// by less than 2^-15: where it is that near to a border, 254 x and (2 n + 1) amax, both exact in
// fp64, decide.
__device__ __forceinline__ float q8_code(float x, float y, float amax) {
    float q = rintf(y);
    if (fabsf(y - q) > 0.4999f) {
        const float n = floorf(y);
        const double t = 254.0 * (double)x - (2.0 * (double)n + 1.0) * (double)amax;
        const bool even = ((int)n & 1) == 0;
        q = (t > 0.0 || (t == 0.0 && !even)) ? n + 1.0f : n;
    }
    return q;
}

// Codes of this thread's 8 columns and the scale of the block of 128 that 16 threads share (all of
// them here).  A block that holds an infinity or a NaN gets scale NaN; one whose values all lie
// below 2^-110 is kept as zeros.
__device__ __forceinline__ uint2 q8_block(const float (&x)[8], bool act, float& scale) {
    uint32_t m = 0;   // the bits of |x| order as the values do, infinities and NaN above them
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    if (!act) m = 0;
#pragma unroll
    for (int o = 8; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    uint2 c = make_uint2(0u, 0u);
    if (m >= 0x7f800000u) {
        scale = __uint_as_float(0x7fffffffu);
        return c;
    }
    const float amax = __uint_as_float(m);
    if (amax < Q8_LEAST) {
        scale = 0.f;
        return c;
    }
    const float inv = 127.0f / amax;
    scale = amax / 127.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c.x |= ((uint32_t)(int)q8_code(x[i], x[i] * inv, amax) & 0xffu) << (8 * i);
        c.y |= ((uint32_t)(int)q8_code(x[4 + i], x[4 + i] * inv, amax) & 0xffu) << (8 * i);
    }
    return c;
}


// Blocks of 128 columns (the last one of a row may be shorter), 16 threads each; a thread takes
// UNITS blocks at a time, their loads under way together.  Blocks are counted row by row; the ones
// of a thread are `step` apart = step_rows rows and step_blocks blocks.
constexpr int Q8_UNITS = 4;

struct BlockWalk {
    int64_t row;
    int block;
    __device__ __forceinline__ BlockWalk(int64_t u, int nb) : row(u / nb), block((int)(u - row * nb)) {}
    __device__ __forceinline__ void advance(int64_t step_rows, int step_blocks, int nb) {
        row += step_rows;
        block += step_blocks;
        if (block >= nb) {
            block -= nb;
            ++row;
        }
    }
};

template <bool F32>
__global__ void __launch_bounds__(256) q8_store_kernel(const void* x, int64_t T, int d, int nb, int64_t step_rows,
                                                       int step_blocks, int8_t* codes, float* scales) {
    pdl_wait();
    const int lane16 = threadIdx.x & 15;
    BlockWalk w((int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), nb);
    // a warp's two blocks leave the loop together: its shuffles need both
    while (__any_sync(0xffffffffu, w.row < T)) {
        Raw<F32> raw[Q8_UNITS];
        int64_t at[Q8_UNITS], sat[Q8_UNITS];
        bool act[Q8_UNITS];
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            const int col = w.block * 128 + lane16 * 8;
            act[n] = w.row < T && col < d;
            at[n] = w.row * d + col;
            sat[n] = w.row < T ? w.row * nb + w.block : -1;
            if (act[n]) ld_whole<F32>(x, at[n], raw[n]);
            w.advance(step_rows, step_blocks, nb);
        }
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            float v[8], scale;
            if (act[n]) {
                whole_values<F32>(raw[n], v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 0.f;
            }
            const uint2 c = q8_block(v, act[n], scale);
            if (act[n]) *reinterpret_cast<uint2*>(codes + at[n]) = c;
            if (lane16 == 0 && sat[n] >= 0) scales[sat[n]] = scale;
        }
    }
}

template <bool F32>
__global__ void __launch_bounds__(256) q8_load_kernel(const int8_t* codes, const float* scales, int64_t T, int d, int nb,
                                                      int64_t step_rows, int step_blocks, void* x) {
    pdl_wait();
    const int lane16 = threadIdx.x & 15;
    BlockWalk w((int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), nb);
    while (w.row < T) {
        uint2 c[Q8_UNITS];
        float scale[Q8_UNITS];
        int64_t at[Q8_UNITS];
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            const int col = w.block * 128 + lane16 * 8;
            at[n] = w.row < T && col < d ? w.row * d + col : -1;
            if (at[n] >= 0) {
                c[n] = ld8(codes + at[n]);
                scale[n] = scales[w.row * nb + w.block];
            }
            w.advance(step_rows, step_blocks, nb);
        }
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            if (at[n] < 0) continue;
            float v[8];
            code_values(c[n].x, c[n].y, scale[n], v);
            if constexpr (F32)
                st_f8(static_cast<float*>(x) + at[n], v);
            else
                st_b8(static_cast<__nv_bfloat16*>(x) + at[n], v);
        }
    }
}

// ------------------------------------------------------------ sums over a row

// One row's warps: wi of gw, of group `group` of the CTA (named barrier group + 1).
struct RowGroup {
    int gw, wi, lane, group;
    int buf;        // which half of the group's shared memory the next sum takes
    float* part;    // [2][2][32]
};

__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// v[n] <- the sum of v[n] over the row's threads, the same bits in all of them.  One barrier: a
// warp that passes the next one's has read this one's half.
template <int N>
__device__ __forceinline__ void row_sum(RowGroup& g, float (&v)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = warp_sum_f(v[n]);
    if (g.gw == 1) return;
    float* p = g.part + g.buf * 64;
    if (g.lane == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) p[n * 32 + g.wi] = v[n];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(g.group + 1), "r"(g.gw * 32) : "memory");
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = warp_sum_f(g.lane < g.gw ? p[n * 32 + g.lane] : 0.f);
    g.buf ^= 1;
}

// Mean (0 for an RMS norm) and 1 / sqrt(mean square about it + eps) of a row's values.
__device__ __forceinline__ float2 row_stats(RowGroup& g, const float (&x)[8], bool act, int kind, float inv_d, float eps) {
    float mean = 0.f;
    if (kind == MOEVIE_NORM_LAYER) {
        float s[1] = {0.f};
        if (act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += x[i];
        }
        row_sum(g, s);
        mean = s[0] * inv_d;
    }
    float q[1] = {0.f};
    if (act) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = x[i] - mean;
            q[0] = fmaf(z, z, q[0]);
        }
    }
    row_sum(g, q);
    return make_float2(mean, rsqrtf(fmaf(q[0], inv_d, eps)));
}

// ------------------------------------------------------------ runs of rows

// The run (segment) that row t lies in: the last g with seg[g] <= t, 0 where there is none.
__device__ __forceinline__ int64_t run_of(const int32_t* seg, int64_t G, int64_t t) {
    int64_t lo = 0, hi = G;   // seg[lo] <= t < seg[hi], as far as seg says
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (seg[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Rows [t0, t1) of group gid of n_groups <= T (each has some); group_of is its inverse.
__device__ __forceinline__ int64_t first_row(int64_t T, int64_t gid, int64_t n_groups) { return T * gid / n_groups; }
__device__ __forceinline__ int64_t group_of(int64_t T, int64_t t, int64_t n_groups) { return ((t + 1) * n_groups - 1) / T; }

// Ends of runs have to ascend within [0, T]; one that does not is a device error (rows are then
// taken as far as they lie in [0, T)).
__device__ __forceinline__ void check_runs(const int32_t* seg, int64_t G, int64_t T, DevStatus* st) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < G; i += (int64_t)gridDim.x * blockDim.x) {
        const int a = seg[i], b = seg[i + 1];
        if (a < 0 || b < a || b > T) report(st, MOEVIE_ERR_DEVICE, SITE_RUNS, (int)i, b);
    }
}

// The rows of a group that lie in some run.
template <typename Args>
__device__ __forceinline__ void clip_rows(const Args& a, int64_t& t0, int64_t& t1) {
    if (!a.seg) return;
    t0 = max(t0, (int64_t)a.seg[0]);
    t1 = min(t1, (int64_t)a.seg[a.G]);
}

// ------------------------------------------------------------ forward

template <bool F32, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : 512, BIG ? 1 : 2) norm_forward_kernel(const NormArgs a) {
    __shared__ float s_part[MAX_GROUPS * 128];
    pdl_wait();
    RowGroup g;
    g.lane = threadIdx.x & 31;
    g.gw = a.gw;
    g.group = (threadIdx.x >> 5) / a.gw;
    g.wi = (threadIdx.x >> 5) - g.group * a.gw;
    g.buf = 0;
    g.part = s_part + g.group * 128;
    if (a.seg) check_runs(a.seg, a.G, a.T, a.st);
    const int col = (g.wi * 32 + g.lane) * 8;
    const bool act = col < a.d;
    const int64_t gid = (int64_t)blockIdx.x * a.groups + g.group;
    if (gid >= a.n_groups) return;
    int64_t t0 = first_row(a.T, gid, a.n_groups), t1 = first_row(a.T, gid + 1, a.n_groups);
    clip_rows(a, t0, t1);
    if (t0 >= t1) return;

    const bool join = a.f != nullptr;
    const float inv_d = 1.0f / (float)a.d;
    float w1[8], b1[8];
    ld_param(a.w_pre, col, act, 1.f, w1);
    ld_param(a.b_pre, col, act, 0.f, b1);
    float w2[8], b2[8];   // gate * weight, gate * bias
    int64_t run = 0, run_end = t1;
    bool fresh = true;

    Raw<F32> rr;
    uint4 rf = make_uint4(0u, 0u, 0u, 0u);
    auto fetch = [&](int64_t t) {
        if (!act) return;
        const int64_t at = t * a.d + col;
        if (a.r_q8) ld_codes<F32>(a.r, at, a.r_scale, t * a.nb + (col >> 7), rr);
        else ld_whole<F32>(a.r, at, rr);
        if (join) rf = ld16(a.f + at);
    };
    fetch(t0);
    for (int64_t t = t0; t < t1; ++t) {
        float r[8], x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = x[i] = 0.f;
        if (act) {
            if (a.r_q8) code_values(rr.a.x, rr.a.y, rr.scale, r);
            else whole_values<F32>(rr, r);
            if (join) unpack_bf16x8(rf, x);
        }
        if (t + 1 < t1) fetch(t + 1);
        if (a.qr) {
            float scale;
            const uint2 c = q8_block(r, act, scale);
            if (act) *reinterpret_cast<uint2*>(a.qr + t * a.d + col) = c;
            if (act && (g.lane & 15) == 0) a.qr_scale[t * a.nb + (col >> 7)] = scale;
        }
        if (a.qf) {
            float scale;
            const uint2 c = q8_block(x, act, scale);
            if (act) *reinterpret_cast<uint2*>(a.qf + t * a.d + col) = c;
            if (act && (g.lane & 15) == 0) a.qf_scale[t * a.nb + (col >> 7)] = scale;
        }
        if (join) {
            if (fresh || t >= run_end) {   // the run's gate, times the norm's weight and bias
                if (a.seg) {
                    run = fresh ? run_of(a.seg, a.G, t) : run + 1;
                    while (run + 1 < a.G && a.seg[run + 1] <= t) ++run;
                    run_end = a.seg[run + 1];
                }
                fresh = false;
                float gt[8];
                ld_param(a.gate ? a.gate + run * a.d : nullptr, col, act, 1.f, gt);
                ld_param(a.w_post, col, act, 1.f, w2);
                ld_param(a.b_post, col, act, 0.f, b2);
#pragma unroll
                for (int i = 0; i < 8; ++i) w2[i] *= gt[i], b2[i] *= gt[i];
            }
            float2 s = make_float2(0.f, 1.f);
            if (a.post != MOEVIE_NORM_NONE) {
                s = row_stats(g, x, act, a.post, inv_d, a.eps);
                if (a.stats_post && g.wi == 0 && g.lane == 0) a.stats_post[t] = s;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = fmaf(a.alpha, r[i], fmaf((x[i] - s.x) * s.y, w2[i], b2[i]));
            if (act) {
                if constexpr (F32) st_f8(static_cast<float*>(a.r_out) + t * a.d + col, r);
                else st_b8(static_cast<__nv_bfloat16*>(a.r_out) + t * a.d + col, r);
            }
        }
        if (a.u) {
            const float2 s = row_stats(g, r, act, a.pre, inv_d, a.eps);
            if (a.stats_pre && g.wi == 0 && g.lane == 0) a.stats_pre[t] = s;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = fmaf((r[i] - s.x) * s.y, w1[i], b1[i]);
            if (act) st_b8(a.u + t * a.d + col, r);
        }
    }
}

// ------------------------------------------------------------ backward

// Sums of this thread's 8 columns: in registers, or, for the rows of more than 16 warps whose
// threads have 64 registers, in shared memory (each thread its own words, no bank shared).
template <bool SHARED>
struct Sums {
    float v[8];
    __device__ __forceinline__ Sums(float*, int) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    __device__ __forceinline__ void add(int i, float x, float y) { v[i] = fmaf(x, y, v[i]); }
    __device__ __forceinline__ void store(float* p) const { st_f8(p, v); }
};
template <>
struct Sums<true> {
    float* p;
    __device__ __forceinline__ Sums(float* base, int which) : p(base + which * 8 * blockDim.x + threadIdx.x) { clear(); }
    __device__ __forceinline__ float& at(int i) const { return p[i * blockDim.x]; }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) at(i) = 0.f;
    }
    __device__ __forceinline__ void add(int i, float x, float y) { at(i) = fmaf(x, y, at(i)); }
    __device__ __forceinline__ void store(float* out) const {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at(i);
        st_f8(out, v);
    }
};

// Of row t, with x1, x2 the normed rows before weight and bias and inv_s their 1 / deviation:
//   dR = dr1 + inv_1 (a - [mean a] - x1 mean(a x1)),   a = du w_pre          (mean a: layer norms)
//   dr = alpha dR,   c = gate w_post dR,   df = inv_2 (c - [mean c] - x2 mean(c x2))
// and, summed over rows,
//   dw_pre = sum du x1, db_pre = sum du, A = sum dR x2, B = sum dR (A, B run by run):
//   dgate = w_post A + b_post B,   dw_post = sum_runs gate A,   db_post = sum_runs gate B.
// Each group of warps leaves its sums in the workspace: dw_pre and db_pre at record gid, A and B
// of run g at record g + gid (along the rows g and gid never fall, so that no two share one).
template <bool F32, bool DUF32, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : 512, 1) norm_backward_kernel(const NormBwdArgs a) {
    extern __shared__ float s_acc[];   // BIG: 4 sums of 8 columns for each thread
    __shared__ float s_part[MAX_GROUPS * 128];
    pdl_wait();
    RowGroup g;
    g.lane = threadIdx.x & 31;
    g.gw = a.gw;
    g.group = (threadIdx.x >> 5) / a.gw;
    g.wi = (threadIdx.x >> 5) - g.group * a.gw;
    g.buf = 0;
    g.part = s_part + g.group * 128;
    if (a.seg) check_runs(a.seg, a.G, a.T, a.st);
    const int col = (g.wi * 32 + g.lane) * 8;
    const bool act = col < a.d;
    const int64_t gid = (int64_t)blockIdx.x * a.groups + g.group;
    if (gid >= a.n_groups) return;
    int64_t t0 = first_row(a.T, gid, a.n_groups), t1 = first_row(a.T, gid + 1, a.n_groups);
    clip_rows(a, t0, t1);

    const float inv_d = 1.0f / (float)a.d;
    const bool has_f = a.f != nullptr;
    const bool join = a.df != nullptr;
    float w1[8], cw[8];
    ld_param(a.w_pre, col, act, 1.f, w1);
#pragma unroll
    for (int i = 0; i < 8; ++i) cw[i] = 1.f;
    Sums<BIG> sw(s_acc, 0), sb(s_acc, 1), sA(s_acc, 2), sB(s_acc, 3);   // dw_pre, db_pre, A, B
    int64_t run = 0, run_end = t1;

    auto flush_run = [&]() {
        if (!a.rec_post || !act) return;
        float* p = a.rec_post + (run + gid) * 2 * a.d + col;
        sA.store(p);
        sB.store(p + a.d);
        sA.clear();
        sB.clear();
    };
    auto load_run = [&]() {
        if (!join) return;
        float gt[8];
        ld_param(a.gate ? a.gate + run * a.d : nullptr, col, act, 1.f, gt);
        ld_param(a.w_post, col, act, 1.f, cw);
#pragma unroll
        for (int i = 0; i < 8; ++i) cw[i] *= gt[i];
    };
    if (t0 < t1) {
        if (a.seg) {
            run = run_of(a.seg, a.G, t0);
            run_end = a.seg[run + 1];
        }
        load_run();
    }
    const int64_t first_run = run;

    Raw<F32> rdr, rr1;
    Raw<DUF32> rdu;
    Raw<false> rf;
    float2 s1 = make_float2(0.f, 0.f), s2 = make_float2(0.f, 1.f);
    auto fetch = [&](int64_t t) {
        if (a.du) s1 = a.stats_pre[t];
        if (a.post != MOEVIE_NORM_NONE) s2 = a.stats_post[t];
        if (!act) return;
        const int64_t at = t * a.d + col, sat = t * a.nb + (col >> 7);
        if (a.dr1) ld_whole<F32>(a.dr1, at, rdr);
        if (a.du) {
            ld_whole<DUF32>(a.du, at, rdu);
            if (a.r_q8) ld_codes<F32>(a.r1, at, a.r1_scale, sat, rr1);
            else ld_whole<F32>(a.r1, at, rr1);
        }
        if (has_f) {
            if (a.f_q8) ld_codes<false>(a.f, at, a.f_scale, sat, rf);
            else ld_whole<false>(a.f, at, rf);
        }
    };
    if (!BIG && t0 < t1) fetch(t0);
    for (int64_t t = t0; t < t1; ++t) {
        if (BIG) fetch(t);
        if (t >= run_end && run + 1 < a.G) {
            do {   // runs without rows get zeros
                flush_run();
                ++run;
            } while (run + 1 < a.G && a.seg[run + 1] <= t);
            run_end = a.seg[run + 1];
            load_run();
        }
        float dR[8], x2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) dR[i] = x2[i] = 0.f;
        if (act && a.dr1) whole_values<F32>(rdr, dR);
        const float2 st2 = s2;
        if (act && has_f) {
            if (a.f_q8) code_values(rf.a.x, rf.a.y, rf.scale, x2);
            else unpack_bf16x8(rf.a, x2);
        }
        if (a.du) {
            float x1[8], du[8];
            const float2 st1 = s1;
#pragma unroll
            for (int i = 0; i < 8; ++i) x1[i] = du[i] = 0.f;
            if (act) {
                if (a.r_q8) code_values(rr1.a.x, rr1.a.y, rr1.scale, x1);
                else whole_values<F32>(rr1, x1);
                whole_values<DUF32>(rdu, du);
            }
            if (!BIG && t + 1 < t1) fetch(t + 1);
            float s[2] = {0.f, 0.f};
            if (act) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x1[i] = (x1[i] - st1.x) * st1.y;
                    sw.add(i, du[i], x1[i]);
                    sb.add(i, du[i], 1.f);
                    du[i] *= w1[i];
                    s[0] += du[i];
                    s[1] = fmaf(du[i], x1[i], s[1]);
                }
            }
            row_sum(g, s);
            const float m0 = a.pre == MOEVIE_NORM_LAYER ? s[0] * inv_d : 0.f, m1 = s[1] * inv_d;
#pragma unroll
            for (int i = 0; i < 8; ++i) dR[i] = fmaf(st1.y, fmaf(-x1[i], m1, du[i] - m0), dR[i]);
        } else if (!BIG && t + 1 < t1) {
            fetch(t + 1);
        }
        if (act && a.dr) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = a.alpha * dR[i];
            if constexpr (F32) st_f8(static_cast<float*>(a.dr) + t * a.d + col, o);
            else st_b8(static_cast<__nv_bfloat16*>(a.dr) + t * a.d + col, o);
        }
        if (!join) continue;
        if (a.post == MOEVIE_NORM_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sA.add(i, dR[i], x2[i]);
                dR[i] *= cw[i];
            }
            if (act) st_b8(a.df + t * a.d + col, dR);
            continue;
        }
        float s[2] = {0.f, 0.f};
        if (act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x2[i] = (x2[i] - st2.x) * st2.y;
                sA.add(i, dR[i], x2[i]);
                sB.add(i, dR[i], 1.f);
                dR[i] *= cw[i];
                s[0] += dR[i];
                s[1] = fmaf(dR[i], x2[i], s[1]);
            }
        }
        row_sum(g, s);
        const float m0 = a.post == MOEVIE_NORM_LAYER ? s[0] * inv_d : 0.f, m1 = s[1] * inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) dR[i] = st2.y * fmaf(-x2[i], m1, dR[i] - m0);
        if (act) st_b8(a.df + t * a.d + col, dR);
    }
    const bool any = t0 < t1;
    if (any || a.G == 1) flush_run();   // a group without rows leaves zeros where only one run is
    if (a.group_runs && g.wi == 0 && g.lane == 0)
        a.group_runs[gid] = any ? make_int2((int)first_run, (int)run) : make_int2(0, -1);
    if (a.rec_pre && act) {
        float* p = a.rec_pre + gid * 2 * a.d + col;
        sw.store(p);
        sb.store(p + a.d);
    }
}

// The records of norm_backward_kernel added up, in a fixed order.  A CTA of 32 x 32 threads takes
// 32 columns; its rows of threads share the records out.  blockIdx.y: 0 dw_pre and db_pre; 1 dw_post
// and db_post (and dgate, where there is one run); 2 and on the gradients of the runs' gates.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const NormSumArgs a) {
    __shared__ float s_a[32][33], s_b[32][33];
    pdl_wait();
    const int x = threadIdx.x, y = threadIdx.y;
    const int col = blockIdx.x * 32 + x;
    const bool act = col < a.d;
    const int64_t row = 2 * (int64_t)a.d;   // floats of a record

    auto total = [&](float& va, float& vb) {   // over the 32 rows of threads, in row 0
        s_a[y][x] = va;
        s_b[y][x] = vb;
        __syncthreads();
        va = vb = 0.f;
        if (y == 0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) va += s_a[i][x], vb += s_b[i][x];
        }
        __syncthreads();
    };
    auto add_records = [&](const float* rec, int64_t lo, int64_t hi, float& va, float& vb) {
        if (!act) return;
#pragma unroll 4
        for (int64_t i = lo + y; i < hi; i += 32) {
            const float* p = rec + i * row + col;
            va += p[0];
            vb += p[a.d];
        }
    };
    const float w2 = act && a.w_post ? a.w_post[col] : 1.f;
    const float b2 = act && a.b_post ? a.b_post[col] : 0.f;

    if (blockIdx.y == 0) {
        if (!a.rec_pre) return;
        float va = 0.f, vb = 0.f;
        add_records(a.rec_pre, 0, a.n_groups, va, vb);
        total(va, vb);
        if (y == 0 && act) {
            if (a.dw_pre) a.dw_pre[col] = va;
            if (a.db_pre) a.db_pre[col] = vb;
        }
        return;
    }
    if (!a.rec_post) return;
    if (blockIdx.y == 1) {
        float va = 0.f, vb = 0.f;
        if (a.G == 1) {
            add_records(a.rec_post, 0, a.n_groups, va, vb);
        } else if (act) {
            for (int64_t gid = y; gid < a.n_groups; gid += 32) {
                const int2 runs = a.group_runs[gid];
                for (int64_t g = runs.x; g <= runs.y; ++g) {
                    const float* p = a.rec_post + (g + gid) * row + col;
                    const float gt = a.gate ? a.gate[g * a.d + col] : 1.f;
                    va = fmaf(gt, p[0], va);
                    vb = fmaf(gt, p[a.d], vb);
                }
            }
        }
        total(va, vb);
        if (y == 0 && act) {
            const float gt = a.G == 1 && a.gate ? a.gate[col] : 1.f;
            if (a.dw_post) a.dw_post[col] = gt * va;
            if (a.db_post) a.db_post[col] = gt * vb;
            if (a.G == 1 && a.dgate) a.dgate[col] = fmaf(w2, va, b2 * vb);
        }
        return;
    }
    for (int64_t g = blockIdx.y - 2; g < a.G; g += gridDim.y - 2) {
        float va = 0.f, vb = 0.f;
        const int64_t r0 = max((int64_t)a.seg[g], (int64_t)0), r1 = min((int64_t)a.seg[g + 1], a.T);
        if (r0 < r1) {
            const int64_t lo = group_of(a.T, r0, a.n_groups), hi = group_of(a.T, r1 - 1, a.n_groups);
            add_records(a.rec_post + g * row, lo, hi + 1, va, vb);
        }
        total(va, vb);
        if (y == 0 && act) a.dgate[g * a.d + col] = fmaf(w2, va, b2 * vb);
    }
}

// Warps of a row, row groups of a CTA and the grid: about `threads_sm` threads to an SM.
struct NormPlan {
    int gw, groups, threads, grid;
    int64_t n_groups;   // at most T; the last CTA's groups beyond them have nothing to do
};
NormPlan norm_plan(int64_t T, int d, int threads_sm) {
    NormPlan p;
    p.gw = (d / 8 + 31) / 32;
    p.groups = p.gw == 1 ? 8 : p.gw == 2 ? 4 : p.gw <= 4 ? 2 : 1;
    p.threads = p.gw * 32 * p.groups;
    const int64_t most = (int64_t)GB300_SMS * std::max(1, threads_sm / p.threads);
    p.grid = (int)std::max<int64_t>(1, std::min<int64_t>(most, (T + p.groups - 1) / p.groups));
    p.n_groups = std::min<int64_t>(T, (int64_t)p.grid * p.groups);
    return p;
}
constexpr int NORM_BIG_WARPS = 16;   // rows of more warps: the kernels for d > 4096
constexpr int NORM_FWD_THREADS = 1024, NORM_BWD_THREADS = 512;

template <bool F32>
cudaError_t q8_store(const void* x, int64_t T, int d, int8_t* codes, float* scales, cudaStream_t s) {
    const int nb = (d + 127) / 128;
    const int64_t grid = std::min<int64_t>((T * nb + 16 * Q8_UNITS - 1) / (16 * Q8_UNITS), (int64_t)GB300_SMS * 8);
    const int64_t step = grid * 16;
    return launch_pdl(q8_store_kernel<F32>, dim3((unsigned)grid), dim3(256), 0, s, x, T, d, nb, step / nb, (int)(step % nb),
                      codes, scales);
}
template <bool F32>
cudaError_t q8_load(const int8_t* codes, const float* scales, int64_t T, int d, void* x, cudaStream_t s) {
    const int nb = (d + 127) / 128;
    const int64_t grid = std::min<int64_t>((T * nb + 16 * Q8_UNITS - 1) / (16 * Q8_UNITS), (int64_t)GB300_SMS * 8);
    const int64_t step = grid * 16;
    return launch_pdl(q8_load_kernel<F32>, dim3((unsigned)grid), dim3(256), 0, s, codes, scales, T, d, nb, step / nb,
                      (int)(step % nb), x);
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

cudaError_t launch_norm_forward(NormArgs a, int r_f32, cudaStream_t s) {
    const NormPlan p = norm_plan(a.T, a.d, NORM_FWD_THREADS);
    a.gw = p.gw;
    a.groups = p.groups;
    a.n_groups = p.n_groups;
    a.nb = (a.d + 127) / 128;
    const dim3 grid(p.grid), block(p.threads);
    cudaError_t e;
    if (p.gw > NORM_BIG_WARPS)
        e = r_f32 ? launch_pdl(norm_forward_kernel<true, true>, grid, block, 0, s, a)
                  : launch_pdl(norm_forward_kernel<false, true>, grid, block, 0, s, a);
    else
        e = r_f32 ? launch_pdl(norm_forward_kernel<true, false>, grid, block, 0, s, a)
                  : launch_pdl(norm_forward_kernel<false, false>, grid, block, 0, s, a);
    count_launches(1);
    return e;
}

int64_t norm_groups(int64_t T, int d) {
    return std::max<int64_t>(1, norm_plan(T, d, NORM_BWD_THREADS).n_groups);
}

template <bool F32, bool DUF32>
static cudaError_t norm_backward(const NormBwdArgs& a, const NormPlan& p, cudaStream_t s) {
    const dim3 grid(p.grid), block(p.threads);
    if (p.gw <= NORM_BIG_WARPS) return launch_pdl(norm_backward_kernel<F32, DUF32, false>, grid, block, 0, s, a);
    const size_t smem = (size_t)32 * 4 * p.threads;
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev].load(std::memory_order_acquire)) {   // idempotent: no lock needed
        const cudaError_t e = cudaFuncSetAttribute(norm_backward_kernel<F32, DUF32, true>,
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * 4 * 1024);
        if (e != cudaSuccess) return e;
        attr_set[dev].store(true, std::memory_order_release);
    }
    return launch_pdl(norm_backward_kernel<F32, DUF32, true>, grid, block, smem, s, a);
}

cudaError_t launch_norm_backward(NormBwdArgs a, int r_f32, int du_f32, NormSumArgs sums, cudaStream_t s) {
    const NormPlan p = norm_plan(a.T, a.d, NORM_BWD_THREADS);
    a.gw = p.gw;
    a.groups = p.groups;
    a.n_groups = p.n_groups;
    a.nb = (a.d + 127) / 128;
    cudaError_t e;
    if (r_f32) e = du_f32 ? norm_backward<true, true>(a, p, s) : norm_backward<true, false>(a, p, s);
    else e = du_f32 ? norm_backward<false, true>(a, p, s) : norm_backward<false, false>(a, p, s);
    count_launches(1);
    if (e != cudaSuccess || (!a.rec_pre && !a.rec_post)) return e;
    sums.n_groups = a.n_groups;
    const int64_t gates = sums.G > 1 && sums.dgate ? std::min<int64_t>(sums.G, 4096) : 0;
    e = launch_pdl(norm_sums_kernel, dim3((unsigned)((a.d + 31) / 32), (unsigned)(2 + gates)), dim3(32, 32), 0, s, sums);
    count_launches(1);
    return e;
}

}  // namespace mv
