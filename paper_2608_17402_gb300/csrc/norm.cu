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

// Rows that a row's warps work on at a time: their sums share shuffles and barriers (one row at a time took
// 400 us for 65536 x 1664 in fp32 where two took 299, bound by issued instructions).
constexpr int ROWS = 2;
constexpr int NORM_THREADS = 256;   // of a CTA, at most, but for the forward of rows of more than 2048 columns
constexpr int fwd_slots(bool f32, bool big) { return f32 || big ? 3 : 4; }   // rows under way
constexpr int BWD_SLOTS = 2;
constexpr float Q8_LEAST = 7.70371978e-34f;   // 2^-110: blocks of smaller values are kept as zeros

// ------------------------------------------------------------ 8 columns of a row

// 8 fp32 values as four register pairs, for the two-wide fp32 instructions.
struct P8 {
    uint64_t p[4];
};

__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f2_of(float v) { return f2_pack(v, v); }
__device__ __forceinline__ uint64_t f2_bits(uint32_t lo, uint32_t hi) {
    return f2_pack(__uint_as_float(lo), __uint_as_float(hi));
}
__device__ __forceinline__ P8 p8_of(float v) {
    P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = f2_of(v);
    return r;
}
// the sum of all eight, and of the products of two eights
__device__ __forceinline__ float p8_sum(const P8& a) {
    float x, y;
    f2_unpack(f2_add(f2_add(a.p[0], a.p[1]), f2_add(a.p[2], a.p[3])), x, y);
    return x + y;
}
__device__ __forceinline__ float p8_dot(const P8& a, const P8& b) {
    uint64_t s = f2_mul(a.p[0], b.p[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = f2_fma(a.p[i], b.p[i], s);
    float x, y;
    f2_unpack(s, x, y);
    return x + y;
}

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
__device__ __forceinline__ P8 p8_bf16(const uint4& u) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = f2_bits(w[i] << 16, w[i] & 0xffff0000u);
    return r;
}
__device__ __forceinline__ P8 p8_f32(const uint4& a, const uint4& b) {
    P8 r;
    r.p[0] = f2_bits(a.x, a.y), r.p[1] = f2_bits(a.z, a.w);
    r.p[2] = f2_bits(b.x, b.y), r.p[3] = f2_bits(b.z, b.w);
    return r;
}
// int8 codes times their scale: a code + 128 as the low byte of 2^23 is a float that is off by 2^23 + 128
__device__ __forceinline__ P8 p8_codes(uint32_t lo, uint32_t hi, float scale) {
    const uint32_t w[2] = {lo ^ 0x80808080u, hi ^ 0x80808080u};
    const uint64_t off = f2_of(-8388736.0f), s = f2_of(scale);
    P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = w[i / 2];
        const uint64_t v = f2_bits(__byte_perm(x, 0x4b000000u, 0x7540 + 2 * (i & 1)),
                                   __byte_perm(x, 0x4b000000u, 0x7541 + 2 * (i & 1)));
        r.p[i] = f2_mul(f2_add(v, off), s);
    }
    return r;
}
// 8 fp32 values in one access, where rows start 32 bytes apart from a multiple of 32
__device__ __forceinline__ void st_f32_32(float* p, const P8& v) {
    asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(v.p[0]), "l"(v.p[1]), "l"(v.p[2]), "l"(v.p[3])
                 : "memory");
}
__device__ __forceinline__ void st_f32(float* p, const P8& v) {
    if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
        st_f32_32(p, v);
        return;
    }
    reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(v.p[0], v.p[1]);
    reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(v.p[2], v.p[3]);
}
__device__ __forceinline__ void st_bf16(__nv_bfloat16* p, const P8& v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x, y;
        f2_unpack(v.p[i], x, y);
        w[i] = pack_bf16x2(x, y);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool F32>
__device__ __forceinline__ void st_rows(void* base, int64_t at, const P8& v) {
    if constexpr (F32) st_f32(static_cast<float*>(base) + at, v);
    else st_bf16(static_cast<__nv_bfloat16*>(base) + at, v);
}
// 8 of an optional vector (NULL: `other` everywhere), zeros behind a row's end
__device__ __forceinline__ P8 ld_param(const float* p, int col, bool act, float other) {
    if (!p || !act) return p8_of(act ? other : 0.f);
    return p8_f32(ld16(p + col), ld16(p + col + 4));
}

// ------------------------------------------------------------ 8-bit checkpoints

// The whole number nearest to 127 x / amax, an even one between two, where y, that value in fp32
// (off by at most 127 * 2^-21), is too near to a border to tell: 254 x and (2 n + 1) amax, both exact
// in fp64, decide.
__device__ __noinline__ float q8_border(float x, float y, float amax) {
    const float n = floorf(y);
    const double t = 254.0 * (double)x - (2.0 * (double)n + 1.0) * (double)amax;
    const bool even = ((int)n & 1) == 0;
    return (t > 0.0 || (t == 0.0 && !even)) ? n + 1.0f : n;
}
// the largest of three sizes, and the same but NaN where one of them is
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_abs_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Codes of this thread's 8 columns (zeros behind a row's end) and the scale of the block of 128 that
// 16 threads share, all of them here.  A block that holds an infinity or a NaN gets scale NaN; one
// whose values all lie below 2^-110 is kept as zeros.
__device__ __forceinline__ uint2 q8_block(const P8& v, float& scale) {
    constexpr float ROUND = 12582912.0f;   // 1.5 * 2^23: adding it rounds to a whole number, whose low byte it shows
    constexpr float NEAR = 0.4999f;        // 0.5 less more than y can be off
    constexpr float R127 = 1.0f / 127.0f;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) f2_unpack(v.p[i], x[2 * i], x[2 * i + 1]);
    float amax = max_nan(max_abs_nan(max_abs_nan(x[0], x[1], x[2]), x[3], x[4]), max_abs_nan(x[5], x[6], x[7]));
#pragma unroll
    for (int o = 8; o; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if (!(amax >= Q8_LEAST && amax <= 3.402823466e38f)) {
        scale = amax < Q8_LEAST ? 0.f : __uint_as_float(0x7fffffffu);
        return make_uint2(0u, 0u);
    }
    // 127 / amax, a little more than that (by 2^-22): the one border that whole blocks meet often,
    // 63.5 at x = amax / 2, is then rounded to 64, as it has to be
    float inv;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(amax));
    inv *= 127.0f * (1.0f + 0x1p-22f);
    // amax / 127, correctly rounded (Markstein: the remainder of a quotient within one unit corrects it)
    const float guess = amax * R127;
    scale = fmaf(fmaf(-127.0f, guess, amax), R127, guess);
    uint32_t q[8];
    float e[8], worst = 0.f;
    const uint64_t in2 = f2_of(inv), up = f2_of(ROUND), down = f2_of(-ROUND), minus = f2_of(-1.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t y = f2_mul(v.p[i], in2), r = f2_add(y, up);
        float r0, r1;
        f2_unpack(r, r0, r1);
        q[2 * i] = __float_as_uint(r0);
        q[2 * i + 1] = __float_as_uint(r1);
        f2_unpack(f2_fma(f2_add(r, down), minus, y), e[2 * i], e[2 * i + 1]);
        worst = max_abs(worst, e[2 * i], e[2 * i + 1]);
    }
    if (worst > NEAR) {
        bool border = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) border |= fabsf(e[i]) > NEAR && fabsf(x[i]) != 0.5f * amax;
        if (border) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (fabsf(e[i]) > NEAR) q[i] = __float_as_uint(q8_border(x[i], x[i] * inv, amax) + ROUND);
        }
    }
    uint2 c;
    c.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    c.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    return c;
}

// Blocks of 128 columns (the last one of a row may be shorter), 16 threads each; a thread takes
// UNITS blocks at a time, their loads under way together.  Blocks are counted row by row; the ones
// of a thread are `step` apart = step_rows rows and step_blocks blocks.
constexpr int Q8_UNITS = 4;

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
    pdl_wait();
    const int64_t step = (int64_t)gridDim.x * 16;
    BlockWalk w(nb, d);
    while (w.u < blocks) {
        uint2 c[Q8_UNITS];
        float scale[Q8_UNITS];
        BlockWalk r = w;
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            if (r.u < blocks && r.in_row(d)) {
                c[n] = ld8(codes + r.at);
                scale[n] = scales[r.u];
            }
            r.advance(step, step_at, step_blocks, nb, d);
        }
#pragma unroll
        for (int n = 0; n < Q8_UNITS; ++n) {
            if (w.u < blocks && w.in_row(d)) st_rows<F32>(x, w.at, p8_codes(c[n].x, c[n].y, scale[n]));
            w.advance(step, step_at, step_blocks, nb, d);
        }
    }
}

// ------------------------------------------------------------ sums over a row

// A row's warps in this CTA: wi of gw, of group `group` (named barrier group + 1).  In the backward a row of
// more than 2048 columns (WIDE) is shared out over the CTAs of a cluster, `ranks` of them, with one
// group each.
struct RowGroup {
    int gw, wi, lane, group, rank, ranks;
    int buf;        // which half of the group's shared memory the next sum takes
    float* part;    // two halves: 32 floats (zeros behind the gw-th warp's), WIDE 128
};
constexpr int PART_FLOATS = 256;   // 4 groups of more than one warp, or one of a cluster's 32

template <bool WIDE>
__device__ __forceinline__ RowGroup row_group(int gw, int ranks, float* s_part) {
    RowGroup g;
    g.lane = threadIdx.x & 31;
    g.gw = gw;
    g.group = WIDE ? 0 : (threadIdx.x >> 5) / gw;
    g.wi = (threadIdx.x >> 5) - g.group * gw;
    g.rank = WIDE ? (int)cluster_rank() : 0;
    g.ranks = WIDE ? ranks : 1;
    g.buf = 0;
    g.part = s_part + g.group * 64;   // (of groups of one warp never touched)
    if (!WIDE && gw > 1)
        for (int i = g.wi * 32 + g.lane; i < 64; i += gw * 32) g.part[i] = 0.f;
    return g;
}
// All of a row's warps, in all CTAs that share it.
template <bool WIDE>
__device__ __forceinline__ void row_barrier(const RowGroup& g) {
    __syncwarp();
    if constexpr (WIDE) cluster_sync();
    else asm volatile("bar.sync %0, %1;" ::"r"(g.group + 1), "r"(g.gw * 32) : "memory");
}

// v[n] <- the sum of v[n] over the row's threads, the same bits in all of them; N = 1, 2 or 4.  The sums
// share one set of shuffles: after the first steps each lane carries one of them, the n-th lanes
// 32 n / N on.  Then a word for each warp and sum (WIDE: in every CTA of the cluster), read back one or a
// few to a lane.  One barrier: a warp that passes the next one's has read this one's half.
template <bool WIDE, int N>
__device__ __forceinline__ void row_sum(RowGroup& g, float (&v)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "");
    constexpr int SPAN = 32 / N;   // lanes of one sum
    float x;
    if constexpr (N == 4) {
        const bool up = g.lane & 16, up8 = g.lane & 8;
        const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], 16);
        const float b = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], 16);
        x = (up8 ? b : a) + __shfl_xor_sync(0xffffffffu, up8 ? a : b, 8);
    } else if constexpr (N == 2) {
        const bool up = g.lane & 16;
        x = (up ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[1], 16);
    } else {
        x = v[0];
    }
#pragma unroll
    for (int o = SPAN / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (!WIDE && g.gw == 1) {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = __shfl_sync(0xffffffffu, x, SPAN * n);
        return;
    }
    float* p = g.part + g.buf * (WIDE ? 128 : 32);
    if constexpr (WIDE) {
        if (g.lane % SPAN == 0) {
            const uint32_t mine = smem_u32(p + (g.rank * g.gw + g.wi) * N + g.lane / SPAN);
            for (int r = 0; r < g.ranks; ++r)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(mine, r)), "f"(x) : "memory");
        }
        row_barrier<true>(g);
        x = 0.f;
        for (int i = g.lane; i < g.ranks * g.gw * N; i += 32) x += p[i];
#pragma unroll
        for (int o = N; o < 32; o *= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    } else {
        if (g.lane % SPAN == 0) p[g.wi * N + g.lane / SPAN] = x;
        row_barrier<false>(g);
        x = p[g.lane];
        constexpr int MOST = N == 1 ? 32 : 8 * N;   // (8 warps to a row, but where one sum at a time is formed)
#pragma unroll
        for (int o = N; o < MOST; o *= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __shfl_sync(0xffffffffu, x, n);
    g.buf ^= 1;
}

// Of each of the rows x: mean (0 for an RMS norm) and 1 / sqrt(mean square about it + eps); the rows
// are left less their mean (columns behind a row's end, which are zeros here: anything).
template <int ROWS>
__device__ __forceinline__ void row_stats(RowGroup& g, P8 (&x)[ROWS], bool act, int kind, float inv_d, float eps,
                                          float2 (&st)[ROWS]) {
    float s[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) st[k].x = 0.f;
    if (kind == MOEVIE_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) s[k] = p8_sum(x[k]);
        row_sum<false>(g, s);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            st[k].x = s[k] * inv_d;
            const uint64_t m = f2_of(-st[k].x);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[k].p[i] = f2_add(x[k].p[i], m);
        }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) s[k] = act ? p8_dot(x[k], x[k]) : 0.f;
    row_sum<false>(g, s);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) st[k].y = rsqrtf(fmaf(s[k], inv_d, eps));
}

// ------------------------------------------------------------ runs of rows

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

// ------------------------------------------------------------ rows under way

// A warp's share of the rows that are read: its 256 columns of each operand, copied ahead into
// shared memory that no other warp touches, so that no barrier of a row's warps stands between a copy
// and its use.  An operand of 2 bytes is one piece of 16 bytes to a lane, its own 8 columns; one of
// fp32 is two pieces, which the lanes copy in the order of memory (every 32-byte sector is asked for
// once; asked for twice, by the lane that uses each half, the forward of 65536 x 1664 took 267 us
// instead of 229 and the backward 534 instead of 369) and read back as their own.  A row's slot is filled anew as soon as its values are in
// registers: SLOTS rows are under way while one or two are worked on.
template <int SLOTS, int PIECES>
struct RowRing {
    uint32_t base;       // shared address of the warp's first piece
    uint32_t own;        // this lane's 16 bytes of a piece
    uint32_t in, lo, hi; // fp32: where the lane copies to in each of the two pieces, and its own columns
    bool ok, ok_a, ok_b; // whether its own columns, and what it copies of the two pieces, lie in the row
    // left: columns of the row from the warp's first on
    __device__ __forceinline__ RowRing(void* smem, int left) {
        const int lane = threadIdx.x & 31;
        base = smem_u32(smem) + (threadIdx.x >> 5) * (512u * SLOTS * PIECES);
        own = lane * 16u;
        // The 64 times 16 bytes of a warp's 256 columns: neighbours are swapped in every second eight,
        // so that eight lanes which read every second one meet eight different banks.
        in = (lane ^ ((lane >> 3) & 1)) * 16u;
        lo = (2 * lane + ((lane >> 2) & 1)) * 16u;
        hi = lo ^ 16u;
        ok = lane * 8 < left;
        ok_a = lane * 4 < left;
        ok_b = lane * 4 + 128 < left;
    }
    __device__ __forceinline__ uint32_t at(int slot, int piece) const {
        return base + (uint32_t)(slot * PIECES + piece) * 512u;
    }
    static __device__ __forceinline__ int next(int slot) { return slot + 1 == SLOTS ? 0 : slot + 1; }
};
__device__ __forceinline__ ulonglong2 ld_shared(uint32_t at) {
    ulonglong2 r;
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(r.x), "=l"(r.y) : "r"(at) : "memory");
    return r;
}

// 8 columns of weights that a thread keeps in words of shared memory of its own rather than in
// registers, where the row in hand needs them.
struct Kept {
    uint32_t at, step;
    __device__ __forceinline__ Kept(void* smem, int which)
        : at(smem_u32(smem) + (which * 2 * blockDim.x + threadIdx.x) * 16u), step(blockDim.x * 16u) {}
    __device__ __forceinline__ void set(const P8& v) const {
        asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(at), "l"(v.p[0]), "l"(v.p[1]) : "memory");
        asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(at + step), "l"(v.p[2]), "l"(v.p[3]) : "memory");
    }
    __device__ __forceinline__ P8 get() const {
        P8 v;
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v.p[0]), "=l"(v.p[1]) : "r"(at) : "memory");
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v.p[2]), "=l"(v.p[3]) : "r"(at + step) : "memory");
        return v;
    }
};
constexpr int KEPT_BYTES = 64;   // two of them, for each thread

// copies of 16, 8 and 4 bytes, of which `bytes` are read and the rest are zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ P8 p8_bf16(const ulonglong2& u) {
    return p8_bf16(make_uint4((uint32_t)u.x, (uint32_t)(u.x >> 32), (uint32_t)u.y, (uint32_t)(u.y >> 32)));
}

// One operand's rows: whole (F32 or bf16), or, where Q8 allows it and q8 says so, 8-bit codes with
// their scales (which the callers copy).
template <bool F32, bool Q8>
struct Operand {
    const void* data;
    const float* scale;
    int q8;
    // the lane's share of a row: its 8 columns begin at element `at`; zeros in place of a row that is
    // not live and of columns behind a row's end
    template <typename Ring>
    __device__ __forceinline__ void copy(const Ring& ring, int slot, int piece, int64_t at, bool live) const {
        const uint32_t dst = ring.at(slot, piece);
        if (Q8 && q8) {
            copy8(dst + ring.own / 2, static_cast<const int8_t*>(data) + at, live && ring.ok ? 8 : 0);
            return;
        }
        if constexpr (F32) {
            const float* p = static_cast<const float*>(data) + at - 4 * (threadIdx.x & 31);
            copy16(dst + ring.in, p, live && ring.ok_a ? 16 : 0);
            copy16(dst + ring.in + 512, p + 128, live && ring.ok_b ? 16 : 0);
        } else {
            copy16(dst + ring.own, static_cast<const __nv_bfloat16*>(data) + at, live && ring.ok ? 16 : 0);
        }
    }
    template <typename Ring>
    __device__ __forceinline__ P8 get(const Ring& ring, int slot, int piece, uint32_t scale_at) const {
        const uint32_t src = ring.at(slot, piece);
        if (Q8 && q8) {
            uint32_t lo, hi;
            float s;
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(lo), "=r"(hi) : "r"(src + ring.own / 2) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s) : "r"(scale_at) : "memory");
            return p8_codes(lo, hi, s);
        }
        if constexpr (F32) {
            const ulonglong2 a = ld_shared(src + ring.lo), b = ld_shared(src + ring.hi);
            P8 r;
            r.p[0] = a.x, r.p[1] = a.y, r.p[2] = b.x, r.p[3] = b.y;
            return r;
        } else {
            return p8_bf16(ld_shared(src + ring.own));
        }
    }
};

// ------------------------------------------------------------ forward

// JOIN: r1 = alpha r + gate * N_post(f), and its norm; otherwise the norm of r alone.  BOTH: a join with
// both norms and their statistics (the others ask as they go).  SAVE: 8-bit checkpoints of what is read.
// BIG: rows of more than 2048 columns, by CTAs of up to 1024 threads of 64 registers, a row at a time (over
// the CTAs of a cluster, as in the backward, its up to four barriers a row cost more: 8192 x 4096 bf16 135 us
// instead of 70).
template <bool F32, bool JOIN, bool BOTH, bool SAVE, bool BIG>
__global__ void __launch_bounds__(BIG ? 1024 : NORM_THREADS, BIG ? 1 : SAVE ? 3 : 2) norm_forward_kernel(const NormArgs a) {
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

// ------------------------------------------------------------ backward

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
// ALL: both norms, dr1 and f; the others ask as they go.  Q8: r1 and f may be checkpoints.  BIAS: db_pre and B
// as well.
template <bool F32, bool DUF32, bool ALL, bool Q8, bool BIAS, bool WIDE>
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

    const bool norm = ALL || a.du != nullptr, has_f = ALL || a.f != nullptr, join = ALL || a.df != nullptr;
    const bool post = ALL || a.post != MOEVIE_NORM_NONE, has_dr = ALL || a.dr1 != nullptr;
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
    // lane 0; the scales of the warp's two blocks of r1 (4, 5) and of f (6, 7), by lanes 0 and 1.
    const float2 *st1_at = a.stats_pre + t0, *st2_at = a.stats_post + t0;   // of the row in hand
    const int block = first_col / 128 + g.wi * 2 + g.lane;
    const bool scaled = Q8 && g.lane < 2 && block < a.nb;
    const int64_t scale_at = t0 * a.nb + block;
    const float* s1_at = Q8 && scaled && a.r_q8 ? a.r1_scale + scale_at : nullptr;
    const float* s2_at = Q8 && scaled && a.f_q8 ? a.f_scale + scale_at : nullptr;
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
        if (Q8 && s1_at) copy4(words + 16 + g.lane * 4, s1_at + on * a.nb, live ? 4 : 0);
    };
    auto copy_second = [&](int to, int i, int on) {
        const bool live = i + on < n;
        if (has_f) Fo.copy(ring, to, 2 * PR + PU, at + on * d, live);
        const uint32_t words = ring.at(to, PIECES - 1);
        if (post && g.lane == 0) copy8(words + 8, st2_at + on, live ? 8 : 0);
        if (Q8 && s2_at) copy4(words + 24 + g.lane * 4, s2_at + on * a.nb, live ? 4 : 0);
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
                if (norm) {
                    x1[k] = R1.get(ring, slot ^ k, PR + PU, words + scale_word);
                    du[k] = Du.get(ring, slot ^ k, PR, 0);
                }
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(st1[k].x), "=f"(st1[k].y) : "r"(words) : "memory");
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
                const uint64_t m = f2_of(-st1[k].x), q = f2_of(st1[k].y);
#pragma unroll
                for (int j = 0; j < 4; ++j) x1[k].p[j] = f2_mul(f2_add(x1[k].p[j], m), q);
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
                if (has_f) x2[k] = Fo.get(ring, slot ^ k, 2 * PR + PU, words + scale_word);
                else x2[k] = p8_of(0.f);
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(st2[k].x), "=f"(st2[k].y) : "r"(words) : "memory");
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
                    const uint64_t m = f2_of(-st2[k].x), q = f2_of(st2[k].y);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x2[k].p[j] = f2_mul(f2_add(x2[k].p[j], m), q);
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

// CTAs that share a row and columns of each, warps of a row in a CTA, row groups of a CTA and the grid.
struct NormPlan {
    int ranks, span, gw, groups, threads, grid;
    int64_t n_groups;   // at most T; the last CTA's groups beyond them have nothing to do
};
// About `threads_sm` threads to an SM.  shared: rows of more than 2048 columns by clusters, of which at most
// `clusters` (0: as many as there is room for).
NormPlan norm_plan(int64_t T, int d, int threads_sm, bool shared, int clusters = 0) {
    NormPlan p;
    p.ranks = shared ? (d + 2047) / 2048 : 1;
    p.span = p.ranks == 1 ? d : ((d + 127) / 128 + p.ranks - 1) / p.ranks * 128;   // whole blocks of a checkpoint
    p.gw = (p.span / 8 + 31) / 32;
    p.groups = p.ranks > 1 ? 1 : p.gw == 1 ? 8 : p.gw == 2 ? 4 : p.gw <= 4 ? 2 : 1;
    p.threads = p.gw * 32 * p.groups;
    int64_t most = (int64_t)GB300_SMS * std::max(1, threads_sm / p.threads) / p.ranks;
    if (clusters > 0) most = std::min<int64_t>(most, clusters);
    const int64_t units = std::max<int64_t>(1, std::min<int64_t>(most, (T + p.groups - 1) / p.groups));
    p.grid = (int)units * p.ranks;
    p.n_groups = std::min<int64_t>(T, units * p.groups);
    return p;
}
// Threads to an SM.  Forward: 512 with 128 registers each (65536 x 1664 in fp32: 204 us, with 768 of 80 each 228),
// but 768 where checkpoints are formed as well, which is bound by instructions, not by bytes.
constexpr int NORM_FWD_THREADS = 512, NORM_SAVE_THREADS = 768, NORM_BIG_THREADS = 1024, NORM_BWD_THREADS = 512;
constexpr int NORM_MAX_SMEM = 112 * 1024, NORM_BIG_SMEM = 208 * 1024;

// Grid of the checkpoint kernels and the step of their walk over the blocks, CTAs_SM to an SM at most.
struct BlockPlan {
    int nb, grid, step_blocks;
    int64_t blocks, step_at;
    BlockPlan(int64_t T, int d, int ctas_sm) : nb((d + 127) / 128), blocks(T * nb) {
        grid = (int)std::min<int64_t>((blocks + 16 * Q8_UNITS - 1) / (16 * Q8_UNITS), (int64_t)GB300_SMS * ctas_sm);
        const int64_t step = (int64_t)grid * 16;
        step_blocks = (int)(step % nb);
        step_at = step / nb * d + step_blocks * 128;
    }
};
template <bool F32>
cudaError_t q8_store(const void* x, int64_t T, int d, int8_t* codes, float* scales, cudaStream_t s) {
    const BlockPlan p(T, d, F32 ? 3 : 4);
    return launch_pdl(q8_store_kernel<F32>, dim3(p.grid), dim3(256), 0, s, x, p.blocks, d, p.nb, p.step_at,
                      p.step_blocks, codes, scales);
}
template <bool F32>
cudaError_t q8_load(const int8_t* codes, const float* scales, int64_t T, int d, void* x, cudaStream_t s) {
    const BlockPlan p(T, d, 6);
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

// What the first launch of a kernel on a device sets up: its shared memory's limit, and, for one of
// clusters, how many of them run at a time.
struct RowsKernel {
    std::atomic<int> ready[64][5][33];   // [device][CTAs of a cluster][warps of a CTA]: 0 not yet, else clusters + 1
};

// Launches kern for the rows of a with smem_thread bytes of dynamic shared memory for each thread, rows of more
// than 2048 columns shared out over clusters or by one BIG CTA each.
template <bool BIG, typename Args>
static cudaError_t launch_rows(void (*kern)(Args), RowsKernel& k, bool shared, int threads_sm, size_t smem_thread,
                               cudaStream_t s, Args& a) {
    constexpr int most_smem = BIG ? NORM_BIG_SMEM : NORM_MAX_SMEM;
    NormPlan p = norm_plan(a.T, a.d, threads_sm, shared);
    const size_t smem = smem_thread * p.threads;
    if (smem > most_smem || p.ranks > 4 || p.threads > (BIG ? 1024 : NORM_THREADS)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cfg.blockDim = dim3(p.threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see launch_pdl
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)p.ranks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    int dev = 0, clusters = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64) {
        std::atomic<int>& ready = k.ready[dev][p.ranks][p.threads / 32];
        int now = ready.load(std::memory_order_acquire);
        if (now == 0) {   // idempotent: no lock needed
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem);
            if (e != cudaSuccess) return e;
            now = 1;
            if (p.ranks > 1) {
                cudaLaunchConfig_t most = cfg;
                most.gridDim = dim3(p.ranks);
                most.attrs = at + 1;
                most.numAttrs = 1;
                int n = 0;
                if (cudaOccupancyMaxActiveClusters(&n, kern, &most) != cudaSuccess || n < 1) {
                    cudaGetLastError();
                    n = GB300_SMS / p.ranks;   // (one to so many SMs)
                }
                now = n + 1;
            }
            ready.store(now, std::memory_order_release);
        }
        clusters = now - 1;
    }
    if (p.ranks > 1) p = norm_plan(a.T, a.d, threads_sm, shared, clusters);
    cfg.gridDim = dim3(p.grid);
    cfg.numAttrs = p.ranks > 1 ? 2 : 1;
    a.gw = p.gw;
    a.groups = p.groups;
    a.ranks = p.ranks;
    a.span = p.span;
    a.n_groups = p.n_groups;
    a.nb = (a.d + 127) / 128;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <bool F32, bool JOIN, bool BOTH, bool SAVE, bool BIG>
static cudaError_t norm_forward(NormArgs& a, cudaStream_t s) {
    static RowsKernel k;
    return launch_rows<BIG>(norm_forward_kernel<F32, JOIN, BOTH, SAVE, BIG>, k, false,
                            BIG ? NORM_BIG_THREADS : SAVE ? NORM_SAVE_THREADS : NORM_FWD_THREADS,
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

int64_t norm_groups(int64_t T, int d) {
    return std::max<int64_t>(1, norm_plan(T, d, NORM_BWD_THREADS, true).n_groups);
}

template <bool F32, bool DUF32, bool ALL, bool Q8, bool BIAS, bool WIDE>
static cudaError_t norm_backward(NormBwdArgs& a, cudaStream_t s) {
    static RowsKernel k;
    return launch_rows<false>(norm_backward_kernel<F32, DUF32, ALL, Q8, BIAS, WIDE>, k, true, NORM_BWD_THREADS,
                              KEPT_BYTES + 16 * BWD_SLOTS * (2 * (F32 ? 2 : 1) + (DUF32 ? 2 : 1) + 2), s, a);
}
template <bool F32, bool DUF32, bool WIDE>
static cudaError_t norm_backward(NormBwdArgs& a, bool bias, cudaStream_t s) {
    if (!a.du || !a.dr1 || !a.df || !a.f || a.post == MOEVIE_NORM_NONE)
        return norm_backward<F32, DUF32, false, true, true, WIDE>(a, s);
    if (a.r_q8 || a.f_q8)
        return bias ? norm_backward<F32, DUF32, true, true, true, WIDE>(a, s)
                    : norm_backward<F32, DUF32, true, true, false, WIDE>(a, s);
    return bias ? norm_backward<F32, DUF32, true, false, true, WIDE>(a, s)
                : norm_backward<F32, DUF32, true, false, false, WIDE>(a, s);
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
