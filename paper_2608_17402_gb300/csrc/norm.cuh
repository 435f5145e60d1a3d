// norm.cuh -- what the kernels of norm.cu and norm_back.cu share: 8 columns of a row as pairs of fp32, 8-bit
// codes, sums over a row's threads, rows copied ahead, and the launch of CTAs that walk over rows.
#pragma once

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
constexpr float Q8_MOST = 0x1.020406p+121f;   // the largest scale: 127 times the next float is no finite one

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
// int8 codes as fp32: a code + 128 as the low byte of 2^23 is a float that is off by 2^23 + 128
__device__ __forceinline__ P8 p8_codes(uint32_t lo, uint32_t hi) {
    const uint32_t w[2] = {lo ^ 0x80808080u, hi ^ 0x80808080u};
    const uint64_t off = f2_of(-8388736.0f);
    P8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = w[i / 2];
        const uint64_t v = f2_bits(__byte_perm(x, 0x4b000000u, 0x7540 + 2 * (i & 1)),
                                   __byte_perm(x, 0x4b000000u, 0x7541 + 2 * (i & 1)));
        r.p[i] = f2_add(v, off);
    }
    return r;
}
__device__ __forceinline__ P8 p8_codes(uint32_t lo, uint32_t hi, float scale) {
    P8 r = p8_codes(lo, hi);
    const uint64_t s = f2_of(scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.p[i] = f2_mul(r.p[i], s);
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
// (off by less than 1.2e-4), is too near to a border to tell.  254 x and (2 n + 1) amax decide, each as a
// rounded product and what it left out (their operands 2^-8 times the values: no overflow; amax >= 2^-110 and
// |x| >= amax / 254 leave every bit in range).  The rounded products differ by 2^-11 of themselves at most,
// so their difference is exact; what they left out are whole multiples of x's last place below 2^17 of it, so
// is theirs; and a rounded sum of the two has the sign of the sum.
__device__ __forceinline__ float q8_border(float x, float y, float amax) {
    const float n = floorf(y), m = fmaf(2.0f, n, 1.0f);
    const float xs = x * 0x1p-8f, as = amax * 0x1p-8f;
    const float q = 254.0f * xs, p = m * as;
    const float t = (q - p) + (fmaf(254.0f, xs, -q) - fmaf(m, as, -p));
    const bool odd = (int)n & 1;
    return (t > 0.0f || (t == 0.0f && odd)) ? n + 1.0f : n;
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
__device__ __forceinline__ float warp_max_nan(float a) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(a));
    return r;
}

// Codes of this thread's 8 columns (zeros behind a row's end) and the scale of the block of 128 that
// 16 threads share, all of them here.  A block that holds an infinity or a NaN gets scale NaN; one
// whose values all lie below 2^-110 is kept as zeros.
__device__ __forceinline__ uint2 q8_block(const P8& v, float& scale) {
    constexpr float ROUND = 12582912.0f;   // 1.5 * 2^23: adding it rounds to a whole number, whose low byte it shows
    // 0.5 less more than y can be off: 127 times 2^-23 (the reciprocal), 2^-22 (see below) and three roundings, 7e-5;
    // from amax 2^126 on, where the reciprocal is subnormal, up to 2^-21 in its place, 1.2e-4
    constexpr float NEAR = 0.49987f;
    constexpr float R127 = 1.0f / 127.0f;
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) f2_unpack(v.p[i], x[2 * i], x[2 * i + 1]);
    float amax = max_nan(max_abs_nan(max_abs_nan(x[0], x[1], x[2]), x[3], x[4]), max_abs_nan(x[5], x[6], x[7]));
    // over each half of the warp, all its lanes in both reductions
    const bool upper = threadIdx.x & 16;
    const float lo = warp_max_nan(upper ? 0.f : amax), hi = warp_max_nan(upper ? amax : 0.f);
    amax = upper ? hi : lo;
    if (!(amax >= Q8_LEAST && amax <= 3.402823466e38f)) {
        scale = amax < Q8_LEAST ? 0.f : __uint_as_float(0x7fffffffu);
        return make_uint2(0u, 0u);
    }
    // 127 / amax, a little more than that (by 2^-22): the one border that whole blocks meet often,
    // 63.5 at x = amax / 2, is then rounded to 64, as it has to be (a subnormal reciprocal may lose as much)
    float inv;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(amax));
    inv *= 127.0f * (1.0f + 0x1p-22f);
    // amax / 127, correctly rounded (Markstein: the remainder of a quotient within one unit corrects it); of the
    // largest float the next one below, that its values come back finite
    const float guess = amax * R127;
    scale = fminf(fmaf(fmaf(-127.0f, guess, amax), R127, guess), Q8_MOST);
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
        const float half = amax < 0x1p126f ? 0.5f * amax : -1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) border |= fabsf(e[i]) > NEAR && fabsf(x[i]) != half;
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
// All of a row's warps, in all CTAs that share it.  (With the barrier's number written out for each group the
// backward of 65536 x 1664 takes 354 us instead of 341, the forward of 16384 x 2048 bf16 65 instead of 55.)
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

// (x - st.x) st.y
__device__ __forceinline__ void normed(P8& x, float2 st) {
    const uint64_t m = f2_of(-st.x), q = f2_of(st.y);
#pragma unroll
    for (int j = 0; j < 4; ++j) x.p[j] = f2_mul(f2_add(x.p[j], m), q);
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
    static __device__ __forceinline__ uint2 codes(const Ring& ring, uint32_t src, uint32_t scale_at, float& s) {
        uint2 c;
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c.x), "=r"(c.y) : "r"(src + ring.own / 2) : "memory");
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s) : "r"(scale_at) : "memory");
        return c;
    }
    // the row normed, (x - st.x) st.y; of codes in one step, c (scale st.y) - st.x st.y, whose rounding is as nothing
    // to theirs
    template <typename Ring>
    __device__ __forceinline__ P8 normed(const Ring& ring, int slot, int piece, uint32_t scale_at, float2 st) const {
        P8 x;
        if (Q8 && q8) {
            float s;
            const uint2 c = codes(ring, ring.at(slot, piece), scale_at, s);
            x = p8_codes(c.x, c.y);
            const uint64_t m = f2_of(-st.x * st.y), q = f2_of(s * st.y);
#pragma unroll
            for (int j = 0; j < 4; ++j) x.p[j] = f2_fma(x.p[j], q, m);
        } else {
            x = get(ring, slot, piece, scale_at);
            mv::normed(x, st);
        }
        return x;
    }
    template <typename Ring>
    __device__ __forceinline__ P8 get(const Ring& ring, int slot, int piece, uint32_t scale_at) const {
        const uint32_t src = ring.at(slot, piece);
        if (Q8 && q8) {
            float s;
            const uint2 c = codes(ring, src, scale_at, s);
            return p8_codes(c.x, c.y, s);
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

// CTAs that share a row and columns of each, warps of a row in a CTA, row groups of a CTA and the grid.
struct NormPlan {
    int ranks, span, gw, groups, threads, grid;
    int64_t n_groups;   // at most T; the last CTA's groups beyond them have nothing to do
};
// Barriers whose number comes from a register count as all 16 that a CTA may have, and an SM has 64.
constexpr int NORM_CTAS_SM = 4;
// About `threads_sm` threads to an SM.  shared: rows of more than 2048 columns by clusters, of which at most
// `clusters` (0: as many as there is room for).
NormPlan norm_plan(int64_t T, int d, int threads_sm, bool shared, int clusters = 0) {
    NormPlan p;
    p.ranks = shared ? (d + 2047) / 2048 : 1;
    p.span = p.ranks == 1 ? d : ((d + 127) / 128 + p.ranks - 1) / p.ranks * 128;   // whole blocks of a checkpoint
    p.gw = (p.span / 8 + 31) / 32;
    p.groups = 1;
    if (p.ranks == 1) {   // of CTAs of up to 8 warps the ones of which an SM holds the most warps, large ones first
        int most = 0;
        for (int n = std::max(1, 8 / p.gw); n; --n) {
            const int rows = std::min(NORM_CTAS_SM, threads_sm / (p.gw * 32 * n)) * n;
            if (rows > most) most = rows, p.groups = n;
        }
    }
    p.threads = p.gw * 32 * p.groups;
    int64_t most = (int64_t)GB300_SMS * std::max(1, threads_sm / p.threads) / p.ranks;
    if (clusters > 0) most = std::min<int64_t>(most, clusters);
    const int64_t units = std::max<int64_t>(1, std::min<int64_t>(most, (T + p.groups - 1) / p.groups));
    p.grid = (int)units * p.ranks;
    p.n_groups = std::min<int64_t>(T, units * p.groups);
    return p;
}
// Threads to an SM.  Forward of fp32 rows: 512 with 128 registers each (65536 x 1664: 204 us, with 768 of 80 each
// 228, bound by memory); 768 where rows are bf16 or checkpoints are formed as well, bound by instructions and
// their latency (bf16 16384 x 1536: 40 us, with 640 of 96 each 43, with 512 49).
constexpr int NORM_FWD_THREADS = 512, NORM_MORE_THREADS = 768, NORM_BIG_THREADS = 1024, NORM_BWD_THREADS = 512;
constexpr bool norm_more(bool f32, bool save) { return save || !f32; }
constexpr int NORM_MAX_SMEM = 112 * 1024, NORM_BIG_SMEM = 208 * 1024;

// What the first launch of a kernel on a device sets up: its shared memory's limit, and, for one of
// clusters, how many of them run at a time.
struct RowsKernel {
    std::atomic<int> ready[64][5][33];   // [device][CTAs of a cluster][warps of a CTA]: 0 not yet, else clusters + 1
};

// Launches kern for the rows of a with smem_thread bytes of dynamic shared memory for each thread, rows of more
// than 2048 columns shared out over clusters or by one BIG CTA each.
template <bool BIG, typename Args>
cudaError_t launch_rows(void (*kern)(Args), RowsKernel& k, bool shared, int threads_sm, size_t smem_thread,
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

}  // namespace
}  // namespace mv
