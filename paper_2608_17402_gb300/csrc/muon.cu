// muon.cu -- Newton-Schulz orthogonalisation of stacks of matrices and the optimiser
// step built on it, sm_103a.
//
// For every matrix U [r, c] of a stack, with m = min(r, c):
//   X0 = U / |U|_F   (X0 = 0 for U = 0),
//   A  = X X^T (X^T X when r > c),  B = b A + c A^2,  X <- a X + B X (a X + X B),
// repeated `steps` times with coefficients (a, b, c) per step.  The optimiser step forms
// U from the momentum on the way in and applies the result to the weights on the way out.
//
// Kernels
//   muon_moment_kernel  momentum update (M <- mu M + G) and |U|.
//   muon_scale_kernel   X0 in the working format.  Both are bound by memory: with momentum 20 bytes an
//                       element (G, M, M back; M again, X0's two parts; with Nesterov G again, 24):
//                       256 x 1664 x 416 in 610 us, 5.8 TB/s.  A cluster per matrix that
//                       did both in one launch, its second read from L2, took the same or longer
//                       (256 x 416 x 1664 without momentum, all steps: 2.39 ms against 2.35).
//   ns_kernel           the three products of every step on tcgen05 CTA pairs in one persistent
//                       launch, with the output or the weight update in the last one's epilogue.
//   ns_thin_kernel      all of that for matrices whose smaller side is at most 32, in fp32.
//   ns_small_kernel     the same for few matrices whose smaller side is 33 to 64.
//
// ns_kernel.  Work items are (matrix, stage, tile): a Gram, a polynomial and an apply stage for
// each step.  Only some of the matrices are under way at a time, in buffers that are used again
// for the next ones, so that most of what lies between X0 and the result is still in L2 when it is
// read (all matrices under way at once: the apply stage alone moved 1.4 GB a step, 755 us of a
// 1000 us step on 256 x 416 x 1664).  The matrices under way form NS_LANES groups that are one stage
// apart (one group, if that is the whole stack); in each slot of the schedule every group advances
// by a stage, so that a tile's inputs were finished about a slot of other tiles earlier and its pair
// rarely waits.  A counter per matrix holds the finished tiles of its stages, which follow one
// another; an item waits for the count of all earlier stages.  Items are dealt to the pairs
// round-robin in schedule order and depend on earlier items only; all pairs are co-resident
// (cooperative launch).
//
// Working format.  X is held as hi + lo, two fp16 values (22 significant bits), times 2^10; A and B
// as fp16 times 2^10.  The tensor cores multiply the hi parts (fp16 has three bits more than bf16
// at the same rate; its range suffices as no entry exceeds the largest singular value, which the
// caller's coefficients must keep at 60 or below), accumulate in fp32, and the a X term is added from
// hi and lo in fp32.  That term is what keeps the directions in which U is (nearly) singular clean:
// each step multiplies them by
// a = 3.4, so a rounding of X there would grow by a^steps, several hundred times, while B X is
// small there to begin with.  Against 64 bits the result (default quintic, five steps) is within 2e-3
// (2-norm over 2-norm) for full-rank and for low-rank U alike, as roundings average over the entries;
// where a few entries hold all of U they do not, and a singular value may be off by 2e-2 (the header
// says what to expect of other coefficients).  With X rounded to fp16 alone it would be 4e-2 for a U of
// rank 16.  In the last two steps lo counts 2 and 0 times instead of a, where neither step's a exceeds
// NS_LO_MAX: where singular values have arrived near 1, B lo (which is not formed) takes up most of
// a lo, and leaving both out is nearer (1.6e-3 becomes 1.4e-3 on Gaussian matrices) and saves the
// last step's lo.  The price is a 2e-4 of |X| in the null directions of U: 1.5e-3 instead of 3e-4 for
// rank 1 with a = 3.4, but 8e-3 with a = 20 and a result of half X (1.5e-3 with all of lo).
// For m <= 128 the roundings of a few singular values average less, and time is latency: there (where
// ns_small_kernel does not take them) A and B have lo parts too, and the polynomial and the apply
// product are hi hi + hi lo + lo hi.  The Gram product, whose K is the long side, stays hi hi:
// over five steps the result is then within 0.8e-3 before its rounding to bf16 (all three products
// in one term 2e-3 for 64 singular values, the Gram product in three terms too 1e-5).
//
// What bounds it, measured on one GB300 (five steps; floors are the products of one term, symmetric
// ones counted half, at the measured 1894 TFLOP/s): 256 x 416 x 1664 2.33 ms (floor 0.63), 16 x 768 x 768
// 0.21 ms (0.077), a step on 64 x 1024 x 512 0.56 ms (0.16).  Traffic between L2 and the SMs comes first
// (16 MB per matrix and step of 416 x 1664, 8.8 TB/s in all), not the tensor cores (26 to 36%) or HBM: in
// a copy without the epilogue's arithmetic the first case took 0.97 of the time, without its loads
// 0.93, without the stores 0.85, without all three 0.75; prefetches into L2 ahead of the loads cost 3
// to 20%.  One 1024 x 1024 matrix (124 us) is a chain of 15 dependent stages of 8 us: hand-over between
// CTAs 5 us, 16 K blocks 3 us.  So are stacks of up to about 100 narrow matrices (91 x 505 x 92 152 us).
#include "internal.h"

#include <math.h>

#include <atomic>

#include <cuda_fp16.h>

namespace mv {

namespace {

constexpr float NS_INV_S = 1.0f / NS_S;

// ----------------------------------------------------- element loads (prologue)

// Eight consecutive values of a row; `n` of them exist and no others are touched (zeros in
// their place).  VEC: rows are 16-byte aligned, so whole groups take 16-byte loads.
__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void load_vec8(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    const float4 b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load_vec8(const __nv_bfloat16* p, float (&v)[8]) {
    unpack_bf16x8(*reinterpret_cast<const uint4*>(p), v);
}
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
    if (VEC && n >= 8) {
        load_vec8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? as_f32(p[i]) : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (VEC && n >= 8) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t u) {
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
}

// Splits eight working-format values into hi and lo (see the file comment).
__device__ __forceinline__ void split8(const float (&x)[8], uint4& hi, uint4& lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        h[q] = pack_half2(x[2 * q], x[2 * q + 1]);
        const float2 f = unpack_half2(h[q]);
        l[q] = pack_half2(x[2 * q] - f.x, x[2 * q + 1] - f.y);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// ------------------------------------------------------------------ prologue

// Sums of squares that neither overflow nor vanish: of v, of v 2^-80 (the one used when the
// first overflows) and of v 2^90 (used when the first is below 2^-80, i.e. every |v| < 2^-40).
constexpr float NS_DOWN = 8.271806125530277e-25f;   // 2^-80
constexpr float NS_UP = 1.2379400392853803e+27f;    // 2^90
constexpr float NS_TINY = 8.271806125530277e-25f;   // 2^-80

constexpr int NS_PRO_THREADS = 256;
// Groups of 8 values per CTA: four a thread (with 16 a thread one 1024 x 1024 matrix took 134 us
// instead of 125, 64 x 1024 x 512 574 instead of 557), and more where a matrix would have more than 128
// CTAs, as each reads all their sums.
constexpr int NS_PRO_GROUPS = 1024, NS_PRO_CHUNKS = 128;

// Where the update U comes from.
struct UpdateArgs {
    const void* U;        // the update (or the gradient G) [N] x [r][ld_u]
    int64_t ld_u, st_u;
    int u_bf16, vec;      // bf16 (else fp32); rows 16-byte aligned
    float* M;             // momentum (NULL: U is used as it is), laid out as U
    float mu;
    int nesterov;
    int r, c, gpr;        // gpr: groups of 8 per row
    int groups, chunk, chunks;   // groups of 8 per matrix, per chunk; chunks
    float* part;          // sums of squares [N][chunks][3]
    int32_t* prog;        // progress counters of the matrices, cleared here
};

// Sums of squares of the update over groups [g0, g1) of matrix e, by the whole CTA (threads 0..2
// get them); with a momentum, M is brought up to date on the way.
template <typename T, bool VEC>
__device__ __forceinline__ float update_squares(const UpdateArgs& p, int e, int g0, int g1) {
    const T* U = static_cast<const T*>(p.U) + e * p.st_u;
    float* M = p.M ? p.M + e * p.st_u : nullptr;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
#pragma unroll 2
    for (int g = g0 + (int)threadIdx.x; g < g1; g += (int)blockDim.x) {
        const int row = g / p.gpr, col = (g - row * p.gpr) * 8, n = p.c - col;
        const int64_t at = row * p.ld_u + col;
        float v[8];
        load8<T, VEC>(U + at, n, v);
        if (M) {
            float m[8];
            load8<float, VEC>(M + at, n, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = fmaf(p.mu, m[i], v[i]);
            store8<VEC>(M + at, n, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p.nesterov ? fmaf(p.mu, m[i], v[i]) : m[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s0 = fmaf(v[i], v[i], s0);
            const float d = v[i] * NS_DOWN, u = v[i] * NS_UP;
            s1 = fmaf(d, d, s1);
            s2 = fmaf(u, u, s2);
        }
    }
    __shared__ float red[3][32];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        s0 += __shfl_xor_sync(0xffffffffu, s0, o);
        s1 += __shfl_xor_sync(0xffffffffu, s1, o);
        s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        red[0][warp] = s0;
        red[1][warp] = s1;
        red[2][warp] = s2;
    }
    __syncthreads();
    float s = 0.f;
    if (threadIdx.x < 3)
        for (int w = 0; w < (int)blockDim.x / 32; ++w) s += red[threadIdx.x][w];
    return s;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(NS_PRO_THREADS) muon_moment_kernel(const __grid_constant__ UpdateArgs p) {
    pdl_wait();
    const int e = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.prog[e] = 0;
    const int g0 = blockIdx.x * p.chunk;
    const float s = update_squares<T, VEC>(p, e, g0, min(g0 + p.chunk, p.groups));
    if (threadIdx.x < 3) p.part[((int64_t)e * p.chunks + blockIdx.x) * 3 + threadIdx.x] = s;
}

// The factors of X0 = (v * pre) * post from the three sums of squares of a matrix.
__device__ __forceinline__ void scales_of(float s0, float s1, float s2, float& pre, float& post) {
    float s = s0;
    pre = 1.f;
    if (isinf(s0)) {
        s = s1;
        pre = NS_DOWN;
    } else if (s0 < NS_TINY) {
        s = s2;
        pre = NS_UP;
    }
    post = s == 0.f ? 0.f : 1.0f / sqrtf(s);   // a zero matrix stays zero; NaN stays NaN
}

// X0 = (v * pre) * post from the matrix's partial sums, by one warp (every lane gets the result;
// a fixed order, so that all warps of the grid use the same bits).
__device__ __forceinline__ void norm_scales(const UpdateArgs& u, int e, float& pre, float& post) {
    const float* part = u.part + (int64_t)e * u.chunks * 3;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    for (int i = threadIdx.x & 31; i < u.chunks; i += 32) {
        s0 += __ldg(part + 3 * i);
        s1 += __ldg(part + 3 * i + 1);
        s2 += __ldg(part + 3 * i + 2);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        s0 += __shfl_xor_sync(0xffffffffu, s0, o);
        s1 += __shfl_xor_sync(0xffffffffu, s1, o);
        s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    scales_of(s0, s1, s2, pre, post);
}

// Eight values of the update U of matrix e (n of them exist).
template <typename T, bool VEC>
__device__ __forceinline__ void update8_as(const UpdateArgs& u, int e, int row, int col, int n, float (&v)[8]) {
    const int64_t at = e * u.st_u + row * u.ld_u + col;
    if (u.M && !u.nesterov) {
        load8<float, VEC>(u.M + at, n, v);
        return;
    }
    load8<T, VEC>(static_cast<const T*>(u.U) + at, n, v);
    if (u.M) {
        float m[8];
        load8<float, VEC>(u.M + at, n, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(u.mu, m[i], v[i]);
    }
}
__device__ __forceinline__ void update8(const UpdateArgs& u, int e, int row, int col, int n, float (&v)[8]) {
    if (u.u_bf16) {
        if (u.vec) update8_as<__nv_bfloat16, true>(u, e, row, col, n, v);
        else update8_as<__nv_bfloat16, false>(u, e, row, col, n, v);
    } else {
        if (u.vec) update8_as<float, true>(u, e, row, col, n, v);
        else update8_as<float, false>(u, e, row, col, n, v);
    }
}

// Groups [g0, g1) of X0 = U / |U| in the working format.
__device__ __forceinline__ void scale_groups(const UpdateArgs& u, int e, int g0, int g1, float pre, float post,
                                             __half* xh, __half* xl) {
    const int64_t base = (int64_t)e * u.groups * 8;
#pragma unroll 2
    for (int g = g0 + (int)threadIdx.x; g < g1; g += (int)blockDim.x) {
        const int row = g / u.gpr, col = (g - row * u.gpr) * 8;
        float v[8];
        update8(u, e, row, col, u.c - col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] * pre) * post;
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(xh + base + (int64_t)g * 8) = hi;
        *reinterpret_cast<uint4*>(xl + base + (int64_t)g * 8) = lo;
    }
}

__global__ void __launch_bounds__(NS_PRO_THREADS) muon_scale_kernel(const __grid_constant__ UpdateArgs u, __half* xh,
                                                                    __half* xl) {
    pdl_wait();
    const int e = blockIdx.y;
    float pre, post;
    norm_scales(u, e, pre, post);
    const int g0 = blockIdx.x * u.chunk;
    scale_groups(u, e, g0, min(g0 + u.chunk, u.groups), pre, post * NS_S, xh, xl);
}

// ------------------------------------------------------------------ products

constexpr int NS_BM = 256;            // output rows per tile: a CTA pair, 128 rows (TMEM lanes) each
constexpr int NS_HALF = 128;
constexpr int NS_MAXBN = 256;         // output columns per tile at most (one tcgen05.mma)
constexpr int NS_BK = 64;             // K per ring stage: one 128-byte swizzle row of fp16
constexpr int NS_BOX = 64 * NS_BK * 2;                     // bytes of one 64 x 64 TMA box
// The ring: a stage holds a CTA's A rows and its half of B, three boxes or (256-wide tiles) four; five
// or four stages (five instead of four for the narrow tiles of few matrices: 1024 x 1024 135 -> 134 us).
constexpr int NS_RING_BYTES = 16 * NS_BOX;
constexpr int NS_RING_MAX = 5;        // stages at most
constexpr int NS_EPI_WARPS = 8;       // two per TMEM lane quadrant: 32 of a block's 64 columns each
constexpr int NS_WARP_LOAD = NS_EPI_WARPS;        // operand loads
constexpr int NS_WARP_MMA = NS_EPI_WARPS + 1;
constexpr int NS_WARP_IN = NS_EPI_WARPS + 2;      // loads of what the epilogue reads
constexpr int NS_WARP_OUT = NS_EPI_WARPS + 3;     // stores of what it writes
constexpr int NS_THREADS = (NS_EPI_WARPS + 4) * 32;
// Epilogue blocks: the CTA's 128 rows x 64 columns, in two regions of two boxes (hi and lo, or a
// value and its mirror image; together one fp32 block).
constexpr int NS_REGION = 2 * NS_BOX;
constexpr int NS_SLOTS = 3;
constexpr int NS_SLOT_BYTES = 2 * NS_REGION;
constexpr int NS_BARS = 2 * NS_RING_MAX + 5 + 3 * NS_SLOTS;
constexpr int NS_SMEM = NS_RING_BYTES + NS_SLOTS * NS_SLOT_BYTES + 1024 + 256;
static_assert(NS_SMEM <= 232448 && NS_BARS * 8 + 8 <= 256, "shared memory of one CTA");

constexpr float NS_LO_MAX = 3.5f;     // largest a of the last two steps at which lo may count less
constexpr int NS_LANES = 2;           // groups of matrices under way, a stage apart (three: 256 x 416 x 1664
                                      // 2.38 ms instead of 2.33)
constexpr int NS_MAX_STAGES = 3 * NS_MAX_STEPS;
constexpr int NS_DONE = 2;            // a finished item's contribution to its matrix's counter (both CTAs)

enum NsKind : int { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2 };

struct NsArgs {
    CUtensorMap tX[3][2], tA[2], tB[2];   // [X0, buffer 0, 1][hi, lo]; 3-D maps {inner, rows, matrices
                                          //   (X0) or slots}, boxes 64 x 64
    CUtensorMap tO;                    // the result, where its rows are 16-byte aligned (vec_o)
    CUtensorMap tW;                    // the weights (fp32, plain 64 x 64 boxes), for prefetches
    UpdateArgs u;
    __half *xh[3], *xl[3];             // X0 [N][r][ldx]; X, ping-pong [slots][r][ldx] (lo in place with one term)
    __half *A[2], *B[2];               // hi, lo (lo with three terms only) [slots][m][ldm]
    int N, r, c, m, ldx, ldm, tall, terms;
    int bn, nt_x, mt_x, mt_s, nt_s;    // tile width (64, 128 or 256); tiles of r x c and m x m outputs
    int tiles[3];                      // items of a matrix's stage, by kind
    int n_stages, n_groups, group_max; // stages of a matrix; groups of matrices; their largest size
    int base_size, big_groups;         // the first big_groups of them hold base_size + 1, the others base_size
    int total;                         // items
    int thin_cluster;                  // CTAs per thin matrix
    float* X1;                         // X between segments [N][r][ldx] (thin and few narrow matrices)
    uint8_t restart[NS_MAX_STEPS];     // the step starts a segment (the same)
    uint8_t kind[NS_MAX_STAGES], step[NS_MAX_STAGES];
    int need[NS_MAX_STAGES + 1];       // counter value at which a stage's inputs are complete
    float coef[3 * NS_MAX_STEPS], lo_coef[NS_MAX_STEPS];   // lo_coef: multiplier of lo in a X
    float lo_keep[NS_MAX_STEPS];       // nonzero: the step's X is stored with its lo part
    int steps;
    __nv_bfloat16* O;                  // orthogonalised matrices (or NULL)
    int64_t ld_o, st_o;
    int vec_o;
    float* W;                          // or: weights W <- decay W - rate X, and their bf16 copy
    __nv_bfloat16* Wb;
    int64_t ld_w, st_w;
    float decay, rate;
    DevStatus* status;
    uint64_t limit_ns;
};

// Position of a role in the schedule: the slot that holds items [base, base + count), with the
// group and the stage of each lane (a stage below 0: the lane has not started) and the lane's
// items.
struct NsWalk {
    int base, count;
    int g[NS_LANES], stage[NS_LANES], n[NS_LANES];
};
struct NsItem {
    int e, buf, stage, kind, step, tile;
    int prev;                          // the matrix that used the buffers before, or -1
};

// Groups hold base_size matrices, the first big_groups of them one more.
__device__ __forceinline__ int ns_first(const NsArgs& p, int g) { return g * p.base_size + min(g, p.big_groups); }
__device__ __forceinline__ int ns_size(const NsArgs& p, int g) { return p.base_size + (g < p.big_groups ? 1 : 0); }

__device__ __forceinline__ void ns_count(const NsArgs& p, NsWalk& w) {
    w.count = 0;
#pragma unroll
    for (int l = 0; l < NS_LANES; ++l) {
        w.n[l] = w.stage[l] >= 0 && w.g[l] < p.n_groups ? ns_size(p, w.g[l]) * p.tiles[p.kind[w.stage[l]]] : 0;
        w.count += w.n[l];
    }
}
__device__ __forceinline__ NsWalk ns_walk_start(const NsArgs& p) {
    NsWalk w;
    w.base = 0;
#pragma unroll
    for (int l = 0; l < NS_LANES; ++l) {
        w.g[l] = l;
        w.stage[l] = -l;
    }
    ns_count(p, w);
    return w;
}

// Item `id` (ids only grow from call to call).
__device__ __forceinline__ NsItem ns_item(const NsArgs& p, NsWalk& w, int id) {
    while (id >= w.base + w.count) {
        w.base += w.count;
#pragma unroll
        for (int l = 0; l < NS_LANES; ++l)
            if (++w.stage[l] == p.n_stages) {
                w.stage[l] = 0;
                w.g[l] += NS_LANES;
            }
        ns_count(p, w);
    }
    int pos = id - w.base, l = 0, g = w.g[0], stage = w.stage[0];
#pragma unroll
    for (int i = 1; i < NS_LANES; ++i)
        if (l == i - 1 && pos >= w.n[i - 1]) {
            pos -= w.n[i - 1];
            l = i;
            g = w.g[i];
            stage = w.stage[i];
        }
    NsItem it;
    it.stage = stage;
    it.kind = p.kind[stage];
    it.step = p.step[stage];
    const int tiles = p.tiles[it.kind], i = pos / tiles;
    it.tile = pos - i * tiles;
    it.e = ns_first(p, g) + i;
    it.buf = l * p.group_max + i;
    it.prev = -1;   // the group before on this lane; it has the place, as earlier groups are not smaller
    if (g >= NS_LANES) it.prev = ns_first(p, g - NS_LANES) + i;
    return it;
}

// Where step s reads X (0: X0), and where it writes it (1 or 2).
__device__ __forceinline__ int ns_src(int s) { return s == 0 ? 0 : 2 - (s & 1); }
__device__ __forceinline__ int ns_dst(int s) { return 1 + (s & 1); }

// TWIN below: items are two matrices side by side, a CTA for each; their e and buf then count twos.
struct NsTile {
    int m0, n0, bn, num_kb;            // num_kb: K blocks of one term
    int mma_n;                         // columns that are computed
    int terms;                         // products: hi hi (1), and hi lo + lo hi (3)
    bool mirror;                       // symmetric output: also write its mirror image
    bool same;                         // A's and B's shares of each CTA are the same box: loaded once
    const CUtensorMap *a[2], *b[2];    // operands, hi and lo
    int za, zb;                        // their matrix or slot
    bool a_mn, b_mn;
};

// Operand layouts of a product: an operand whose K runs along the rows of its array is read
// MN-major, one whose K runs along the columns K-major; no array is ever transposed.
//   r <= c:  Gram  X X^T both K-major;   apply B X: B K-major, X MN-major
//   r >  c:  Gram  X^T X both MN-major;  apply X B: both K-major (B is symmetric)
// Symmetric outputs: row tile i has the column tiles from the diagonal on; those past its own
// columns are mirrored.
template <bool TWIN>
__device__ __forceinline__ NsTile ns_tile(const NsArgs& p, const NsItem& it) {
    NsTile t;
    const int src = ns_src(it.step);
    int k = p.m, cols = p.m;
    if (it.kind == NS_APPLY) {
        const int i = it.tile / p.nt_x;
        t.m0 = i * (TWIN ? NS_HALF : NS_BM);
        t.n0 = (it.tile - i * p.nt_x) * p.bn;
        cols = p.c;
        t.mirror = t.same = false;
        t.a_mn = false;
        t.b_mn = !p.tall;
        t.za = p.tall && src == 0 ? it.e : it.buf;
        t.zb = !p.tall && src == 0 ? it.e : it.buf;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            t.a[j] = p.tall ? &p.tX[src][j] : &p.tB[j];
            t.b[j] = p.tall ? &p.tB[j] : &p.tX[src][j];
        }
    } else {
        const int per = NS_BM / p.bn;
        int q = it.tile, i = 0;
        while (i < p.mt_s - 1 && q >= p.nt_s - i * per) {
            q -= p.nt_s - i * per;
            ++i;
        }
        t.m0 = i * NS_BM;
        t.n0 = (i * per + q) * p.bn;
        t.mirror = t.n0 >= t.m0 + NS_BM;
        const bool gram = it.kind == NS_GRAM;
        if (gram) k = p.tall ? p.r : p.c;
        t.a_mn = t.b_mn = gram && p.tall;
        t.za = t.zb = gram && src == 0 ? it.e : it.buf;
#pragma unroll
        for (int j = 0; j < 2; ++j) t.a[j] = t.b[j] = gram ? &p.tX[src][j] : &p.tA[j];
    }
    t.bn = min(p.bn, (cols - t.n0 + 31) & ~31);   // a multiple of 32: each CTA holds half of B
    // A tile on the diagonal: rows and columns of a CTA coincide.  One that the matrix's end trims is
    // computed 256 wide all the same (the products are bound by L2, not by the tensor cores).
    t.terms = it.kind == NS_GRAM ? 1 : p.terms;
    if (it.kind != NS_APPLY) t.same = t.n0 == t.m0 && (p.bn == NS_BM || TWIN) && t.terms == 1;
    t.mma_n = t.same ? NS_BM : TWIN ? 2 * t.bn : t.bn;
    t.num_kb = (k + NS_BK - 1) / NS_BK;
    return t;
}

__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool a_mn_major, bool b_mn_major) {
    return (1u << 4) | (static_cast<uint32_t>(a_mn_major) << 15) | (static_cast<uint32_t>(b_mn_major) << 16) |
           ((static_cast<uint32_t>(N) >> 3) << 17) | ((static_cast<uint32_t>(M) >> 4) << 24);
}

// A CTA's matrix or slot, given an item's; its first row in a tile.
template <bool TWIN>
__device__ __forceinline__ int ns_own(const NsArgs& p, int z, uint32_t rank) { return TWIN ? 2 * z + (int)rank : z; }
template <bool TWIN>
__device__ __forceinline__ int ns_row(const NsArgs& p, const NsTile& t, uint32_t rank) {
    return t.m0 + (TWIN ? 0 : (int)rank * NS_HALF);
}

struct NsSmem {
    uint32_t ring, slots;
    uint32_t full, empty, tfull, tempty, drain;
    int stages, stage_bytes;    // of the ring
    uint32_t in, done, free_;   // per epilogue slot: inputs landed; results written; stores have read it
    uint8_t* slot_ptr;
    uint32_t rank;
    int pair, npairs;
};

__device__ __forceinline__ void ns_abort(volatile int* flag, DevStatus* st, int site, int a) {
    *flag = 1;
    report(st, MOEVIE_ERR_TIMEOUT, site, (int)blockIdx.x, a);
}

// Waits until matrix e's counter has reached `want` (its writers' stores are then visible).
__device__ __forceinline__ bool ns_wait(const NsArgs& p, int e, int want, volatile int* abort_flag, int site) {
    const int32_t* c = p.u.prog + e;
    if (ld_acquire(c) >= want) return true;
    const uint64_t t0 = globaltimer_ns();
    for (uint32_t i = 1; ld_acquire(c) < want; ++i) {
        __nanosleep(100);
        if ((i & 15u) == 0u && (*abort_flag || globaltimer_ns() - t0 > p.limit_ns)) {
            ns_abort(abort_flag, p.status, site, e);
            return false;
        }
    }
    return true;
}

// TMA producer (one thread per CTA): the CTA's 128 rows of A and its half of B's columns; the
// leader posts the byte count of both CTAs on its full barrier.
template <bool TWIN>
__device__ void ns_producer(const NsArgs& p, const NsSmem& sm, volatile int* abort_flag) {
    const uint32_t full_leader = peer_addr(sm.full, 0);
    int s = 0;
    uint32_t ph = 0;
    NsWalk w = ns_walk_start(p);
    for (int id = sm.pair; id < p.total; id += sm.npairs) {
        const NsItem it = ns_item(p, w, id);
        const NsTile t = ns_tile<TWIN>(p, it);
        // the matrix's earlier stages; before its first, the last user of its buffers
        if (it.stage > 0 ? !ns_wait(p, it.e, p.need[it.stage], abort_flag, SITE_NS_WAIT_INPUT)
                         : it.prev >= 0 && !ns_wait(p, it.prev, p.need[p.n_stages], abort_flag, SITE_NS_WAIT_BUFFER))
            return;
        fence_proxy_async_all();   // the inputs were written by ordinary stores
        const int nbox = t.same ? 0 : ((TWIN ? t.bn : t.bn / 2) + 63) / 64;
        const uint32_t bytes = 2u * (uint32_t)(2 + nbox) * NS_BOX;
        const int mm = ns_row<TWIN>(p, t, sm.rank), nn = t.n0 + (TWIN ? 0 : (int)sm.rank * (t.bn / 2));
        const int za = ns_own<TWIN>(p, t.za, sm.rank), zb = ns_own<TWIN>(p, t.zb, sm.rank);   // (past the last: zeros)
        for (int term = 0; term < t.terms; ++term) {
            const CUtensorMap *ma = t.a[term == 2], *mb = t.b[term == 1];   // hi hi, hi lo, lo hi
            for (int kb = 0; kb < t.num_kb; ++kb) {
                if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                    ns_abort(abort_flag, p.status, SITE_NS_WAIT_EMPTY, id);
                    return;
                }
                const uint32_t bar = full_leader + 8 * s, dst = sm.ring + s * sm.stage_bytes;
                if (sm.rank == 0) mbar_arrive_expect_tx(sm.full + 8 * s, bytes);
                const int kk = kb * NS_BK;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    tma_load_3d_pair(dst + j * NS_BOX, ma, bar, t.a_mn ? mm + 64 * j : kk, t.a_mn ? kk : mm + 64 * j,
                                     za);
                for (int j = 0; j < nbox; ++j)
                    tma_load_3d_pair(dst + (2 + j) * NS_BOX, mb, bar, t.b_mn ? nn + 64 * j : kk,
                                     t.b_mn ? kk : nn + 64 * j, zb);
                if (++s == sm.stages) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
    }
}

// MMA issuer: one thread of the leader CTA.
template <bool TWIN>
__device__ __forceinline__ void ns_mma(const NsArgs& p, const NsSmem& sm, uint32_t tmem, volatile int* abort_flag) {
    int s = 0, n = 0;
    uint32_t ph = 0;
    bool issued = false;
    NsWalk w = ns_walk_start(p);
    for (int id = sm.pair; id < p.total; id += sm.npairs) {
        const NsItem it = ns_item(p, w, id);
        const NsTile t = ns_tile<TWIN>(p, it);
        const uint32_t idesc = idesc_f16_f32(NS_BM, t.mma_n, t.a_mn, t.b_mn);
        const uint64_t ad0 = smem_desc_sw128(sm.ring, t.a_mn ? NS_BOX : 16, 1024);
        const uint64_t bd0 = smem_desc_sw128(sm.ring + (t.same ? 0 : 2 * NS_BOX), t.b_mn ? NS_BOX : 16, 1024);
        const uint32_t as = (t.a_mn ? 2048 : 32) >> 4, bs = (t.b_mn ? 2048 : 32) >> 4;
        const int acc = n & 1;
        if (!mbar_wait(sm.tempty + 8 * acc, ((uint32_t)(n >> 1) & 1u) ^ 1u, p.limit_ns, abort_flag)) {
            ns_abort(abort_flag, p.status, SITE_NS_WAIT_TEMPTY, id);
            break;
        }
        ++n;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)acc * NS_MAXBN;
        const int kbs = t.num_kb * t.terms;
        bool ok = true;
        for (int kb = 0; kb < kbs; ++kb) {
            if (!mbar_wait(sm.full + 8 * s, ph, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_FULL, id);
                ok = false;
                break;
            }
            const uint64_t ad = ad0 + (uint64_t)((s * sm.stage_bytes) >> 4);
            const uint64_t bd = bd0 + (uint64_t)((s * sm.stage_bytes) >> 4);
#pragma unroll
            for (int q = 0; q < NS_BK / 16; ++q)
                tc_mma_bf16_pair(d, ad + q * as, bd + q * bs, idesc, (kb | q) != 0 ? 1u : 0u);
            issued = true;
            tc_commit_pair(sm.empty + 8 * s);
            if (++s == sm.stages) {
                s = 0;
                ph ^= 1u;
            }
        }
        if (!ok) break;
        tc_commit_pair(sm.tfull + 8 * acc);
    }
    if (issued) {   // every tcgen05.mma is complete before TMEM is released
        tc_commit_pair(sm.drain);
        if (!mbar_wait(sm.drain, 0, p.limit_ns, nullptr))
            report(p.status, MOEVIE_ERR_TIMEOUT, SITE_NS_DRAIN, (int)blockIdx.x, 0);
    }
}

__device__ __forceinline__ void unpack_half8(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 f = unpack_half2(w[q]);
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
    }
}

// Which regions of an epilogue block a tile reads and writes.
//   GRAM: A = D (a step with c = 0 has no polynomial stage: B = b D);  POLY: B = b A + c D;
//   X: X = a X + D in the working format;  O, W: the same of the last step, to the outputs.
enum NsMode : int { NS_M_GRAM, NS_M_POLY, NS_M_X, NS_M_O, NS_M_W };
__device__ __forceinline__ int ns_mode(const NsArgs& p, const NsItem& it) {
    if (it.kind != NS_APPLY) return it.kind == NS_GRAM ? NS_M_GRAM : NS_M_POLY;
    return it.step < p.steps - 1 ? NS_M_X : p.O ? NS_M_O : NS_M_W;
}

// Whether a tile stores lo parts.
__device__ __forceinline__ bool ns_lo_out(const NsArgs& p, int mode, int step) {
    return mode == NS_M_X ? p.lo_keep[step] != 0.f : mode < NS_M_X && p.terms == 3;
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(tm),
                 "r"(c0), "r"(c1), "r"(c2), "r"(src)
                 : "memory");
}

__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* tm, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(tm), "r"(c0), "r"(c1),
                 "r"(c2)
                 : "memory");
}

// What the epilogue reads of A (polynomial) or X (apply), block by block into its slots: one
// thread.  Gram blocks read nothing; their slots are handed on as they become free.
template <bool TWIN>
__device__ void ns_inputs(const NsArgs& p, const NsSmem& sm, volatile int* abort_flag) {
    int s = 0;
    uint32_t ph = 0;
    NsWalk w = ns_walk_start(p);
    for (int id = sm.pair; id < p.total; id += sm.npairs) {
        const NsItem it = ns_item(p, w, id);
        const NsTile t = ns_tile<TWIN>(p, it);
        const int mode = ns_mode(p, it), src = ns_src(it.step);
        const bool lo = mode >= NS_M_X ? p.lo_coef[it.step] != 0.f : mode == NS_M_POLY && p.terms == 3;
        const int row = ns_row<TWIN>(p, t, sm.rank), e = ns_own<TWIN>(p, it.e, sm.rank);
        const int z = mode >= NS_M_X && src == 0 ? e : ns_own<TWIN>(p, it.buf, sm.rank);
        const CUtensorMap* mh = mode >= NS_M_X ? &p.tX[src][0] : &p.tA[0];
        const CUtensorMap* ml = mode >= NS_M_X ? &p.tX[src][1] : &p.tA[1];
        if (mode != NS_M_GRAM) {
            if (!ns_wait(p, it.e, p.need[it.stage], abort_flag, SITE_NS_WAIT_INPUT)) return;
            fence_proxy_async_all();
        }
        for (int c0 = 0; c0 < t.bn; c0 += 64) {
            if (!mbar_wait(sm.free_ + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_SLOT, id);
                return;
            }
            const uint32_t bar = sm.in + 8 * s, at = sm.slots + s * NS_SLOT_BYTES;
            if (mode == NS_M_W) {   // the weights on their way to L2, blocks ahead of their use
                for (int c = c0 == 0 ? 0 : c0 + 128; c < (c0 == 0 ? min(t.bn, 192) : min(t.bn, c0 + 192)); c += 64)
                    if (t.n0 + c < p.c && e < p.N) {
                        tma_prefetch_3d(&p.tW, t.n0 + c, row, e);
                        tma_prefetch_3d(&p.tW, t.n0 + c, row + 64, e);
                    }
            }
            if (mode == NS_M_GRAM) {
                mbar_arrive(bar);
            } else {
                mbar_arrive_expect_tx(bar, lo ? 2 * NS_REGION : NS_REGION);
                tma_load_3d(at, mh, bar, t.n0 + c0, row, z);
                tma_load_3d(at + NS_BOX, mh, bar, t.n0 + c0, row + 64, z);
                if (lo) {
                    tma_load_3d(at + NS_REGION, ml, bar, t.n0 + c0, row, z);
                    tma_load_3d(at + NS_REGION + NS_BOX, ml, bar, t.n0 + c0, row + 64, z);
                }
            }
            if (++s == NS_SLOTS) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

// Stores the epilogue's finished blocks, hands their slots back and counts finished tiles: one
// thread.
template <bool TWIN>
__device__ void ns_outputs(const NsArgs& p, const NsSmem& sm, volatile int* abort_flag) {
    int s = 0;
    uint32_t ph = 0;
    NsWalk w = ns_walk_start(p);
    for (int id = sm.pair; id < p.total; id += sm.npairs) {
        const NsItem it = ns_item(p, w, id);
        const NsTile t = ns_tile<TWIN>(p, it);
        const int mode = ns_mode(p, it), row = ns_row<TWIN>(p, t, sm.rank), e = ns_own<TWIN>(p, it.e, sm.rank);
        const int rows = mode >= NS_M_X ? p.r : p.m, cols = mode >= NS_M_X ? p.c : p.m;
        const bool to_b = mode == NS_M_POLY || (mode == NS_M_GRAM && p.coef[3 * it.step + 2] == 0.f);
        const bool lo = ns_lo_out(p, mode, it.step);
        const int dst = ns_dst(it.step), z = mode == NS_M_O ? e : ns_own<TWIN>(p, it.buf, sm.rank);
        const CUtensorMap* mh = mode == NS_M_O ? &p.tO : mode == NS_M_X ? &p.tX[dst][0] : to_b ? &p.tB[0] : &p.tA[0];
        const CUtensorMap* ml = mode == NS_M_X ? &p.tX[dst][1] : to_b ? &p.tB[1] : &p.tA[1];
        const bool store = mode != NS_M_W && (mode != NS_M_O || (p.vec_o && e < p.N));
        for (int c0 = 0; c0 < t.bn; c0 += 64) {
            if (!mbar_wait(sm.done + 8 * s, ph, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_SLOT, -id);
                break;
            }
            const uint32_t at = sm.slots + s * NS_SLOT_BYTES;
            const int col = t.n0 + c0;
            if (store && col < cols) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {   // boxes that start past the array's end are not stored
                    if (row + 64 * q >= rows) continue;
                    tma_store_3d(mh, at + q * NS_BOX, col, row + 64 * q, z);
                    if (lo) tma_store_3d(ml, at + NS_REGION + q * NS_BOX, col, row + 64 * q, z);
                    else if (t.mirror) tma_store_3d(mh, at + NS_REGION + q * NS_BOX, row + 64 * q, col, z);
                }
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            mbar_arrive(sm.free_ + 8 * s);
            if (++s == NS_SLOTS) {
                s = 0;
                ph ^= 1u;
            }
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // (bounded by the copies themselves)
        if (*abort_flag) return;
        fence_proxy_async_all();
        add_release(p.u.prog + it.e, 1);
    }
}

// 16-byte chunk c (8 fp16) of row r of a region: the TMA boxes' 128-byte swizzle.
__device__ __forceinline__ uint8_t* ns_cell(uint8_t* region, int r, int c) {
    return region + r * 128 + ((c ^ (r & 7)) << 4);
}
// 16-byte chunk c (4 fp32 of 16) of row r of an fp32 block.
__device__ __forceinline__ float4* ns_cell32(uint8_t* slot, int r, int c) {
    return reinterpret_cast<float4*>(slot + r * 256 + ((c ^ (r & 15)) << 4));
}

// Barrier of the epilogue warps.
__device__ __forceinline__ void ns_epi_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// A warp's 32 columns (half of the block) of one block: thread = row.  One instance per MODE, so
// that each holds only the code that its tiles run.
template <int MODE>
__device__ __forceinline__ void ns_block(const NsArgs& p, const NsItem& it, const NsTile& t, uint8_t* slot, int row,
                                         int half, int rank, int c0, bool live, const uint32_t (&v)[32],
                                         const float4 (&wv)[8]) {
    constexpr bool APPLY = MODE >= NS_M_X;
    const float cc = p.coef[3 * it.step + 2], cb = p.coef[3 * it.step + 1];
    const float fd = MODE == NS_M_GRAM ? (cc == 0.f ? cb * NS_INV_S : NS_INV_S) : MODE == NS_M_POLY ? cc * NS_INV_S : NS_INV_S;
    const float fh = APPLY ? p.coef[3 * it.step] : cb, fl = APPLY ? p.lo_coef[it.step] : cb;
    const bool lo_in = APPLY ? fl != 0.f : p.terms == 3;
    const bool lo_out = ns_lo_out(p, MODE, it.step);
    float keep[MODE == NS_M_W ? 32 : 1];
    uint4 hin[4], lin[4];   // all inputs before the first output (in place: no load passes a store)
    if (MODE != NS_M_GRAM) {
#pragma unroll
        for (int g = 0; g < 4; ++g) hin[g] = *reinterpret_cast<const uint4*>(ns_cell(slot, row, half * 4 + g));
#pragma unroll
        for (int g = 0; g < 4; ++g)
            lin[g] = lo_in ? *reinterpret_cast<const uint4*>(ns_cell(slot + NS_REGION, row, half * 4 + g))
                           : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = half * 4 + g;
        uint4* ch = reinterpret_cast<uint4*>(ns_cell(slot, row, c));
        uint4* cl = reinterpret_cast<uint4*>(ns_cell(slot + NS_REGION, row, c));
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fd * __uint_as_float(v[8 * g + j]);
        if (MODE != NS_M_GRAM) {
            float h[8];
            unpack_half8(hin[g], h);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(fh, h[j], x[j]);
            unpack_half8(lin[g], h);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(fl, h[j], x[j]);
        }
        if (MODE == NS_M_W) {
#pragma unroll
            for (int j = 0; j < 8; ++j) keep[(8 * g + j) % (MODE == NS_M_W ? 32 : 1)] = x[j];
        } else if (MODE == NS_M_O) {
            *ch = make_uint4(pack_bf16x2(x[0] * NS_INV_S, x[1] * NS_INV_S), pack_bf16x2(x[2] * NS_INV_S, x[3] * NS_INV_S),
                             pack_bf16x2(x[4] * NS_INV_S, x[5] * NS_INV_S), pack_bf16x2(x[6] * NS_INV_S, x[7] * NS_INV_S));
        } else {
            uint4 hi, lo;
            split8(x, hi, lo);
            *ch = hi;
            if (lo_out) {
                *cl = lo;
            } else if (t.mirror) {   // column j of the block is row j of the mirror boxes
                const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w};
                uint8_t* box = slot + NS_REGION + (row >> 6) * NS_BOX;
                const int rr = row & 63;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint16_t*>(ns_cell(box, c * 8 + j, rr >> 3) + (rr & 7) * 2) =
                        (uint16_t)(j & 1 ? hw[j >> 1] >> 16 : hw[j >> 1] & 0xffffu);
            }
        }
    }
    if (MODE == NS_M_W) {
        // the block in fp32 where its inputs were, then rows of W in whole 256-byte pieces
        ns_epi_sync();
#pragma unroll
        for (int g = 0; g < 8; ++g)
            *ns_cell32(slot, row, half * 8 + g) =
                make_float4(keep[(4 * g) % (MODE == NS_M_W ? 32 : 1)], keep[(4 * g + 1) % (MODE == NS_M_W ? 32 : 1)],
                            keep[(4 * g + 2) % (MODE == NS_M_W ? 32 : 1)], keep[(4 * g + 3) % (MODE == NS_M_W ? 32 : 1)]);
        ns_epi_sync();
        const float rate = p.rate * NS_INV_S;
        const int q = threadIdx.x & 15, col = t.n0 + c0 + 4 * q, nc = p.c - col;
        const int64_t base = it.e * p.st_w + col;
        if (live && 4 * q < t.bn - c0 && nc > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = (int)(threadIdx.x >> 4) + 16 * i, gr = t.m0 + rank * NS_HALF + r;
                if (gr >= p.r) break;
                const int64_t at = base + gr * p.ld_w;
                const float4 x = *ns_cell32(slot, r, q);
                if (nc >= 4) {
                    float4 o = wv[i];
                    o.x = fmaf(-rate, x.x, p.decay * o.x);
                    o.y = fmaf(-rate, x.y, p.decay * o.y);
                    o.z = fmaf(-rate, x.z, p.decay * o.z);
                    o.w = fmaf(-rate, x.w, p.decay * o.w);
                    *reinterpret_cast<float4*>(p.W + at) = o;
                    if (p.Wb)
                        *reinterpret_cast<uint2*>(p.Wb + at) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
                } else {
                    const float xs[3] = {x.x, x.y, x.z};
#pragma unroll
                    for (int j = 0; j < 3; ++j)
                        if (j < nc) {
                            const float o = fmaf(-rate, xs[j], p.decay * p.W[at + j]);
                            p.W[at + j] = o;
                            if (p.Wb) p.Wb[at + j] = __float2bfloat16_rn(o);
                        }
                }
            }
        }
    } else if (MODE == NS_M_O) {
        if (!p.vec_o) {   // rows off 16-byte bounds: no TMA store; columns in turn over the threads
            ns_epi_sync();
            const int q = threadIdx.x & 63, col = t.n0 + c0 + q;
            if (live && q < t.bn - c0 && col < p.c)
                for (int r = threadIdx.x >> 6; r < NS_HALF; r += 4) {
                    const int gr = t.m0 + rank * NS_HALF + r;
                    if (gr >= p.r) break;
                    p.O[it.e * p.st_o + gr * p.ld_o + col] =
                        *reinterpret_cast<const __nv_bfloat16*>(ns_cell(slot, r, q >> 3) + (q & 7) * 2);
                }
        }
    }
}

// Eight warps: warp w reads TMEM lanes 32 (w % 4) .. and half w / 4 of each 64-column block.  A
// thread's values are consecutive in its row, as they are in the blocks' swizzled rows, so what
// the tile reads and writes in fp16 goes through shared memory in place, 16 bytes at a time, and
// between there and L2 by TMA.  The warps go through the blocks each at its own pace (in step, by a
// barrier per block, they all waited for each other's latencies).  A wait that gives up is recorded
// and the warp goes on without writing results: some modes meet at barriers within a block, which
// every warp must reach.
template <bool TWIN>
__device__ void ns_epilogue(const NsArgs& p, const NsSmem& sm, uint32_t tmem, volatile int* abort_flag) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
    int n = 0, s = 0;
    uint32_t ph = 0;
    bool live = true;
    NsWalk w = ns_walk_start(p);
    for (int id = sm.pair; id < p.total; id += sm.npairs, ++n) {
        NsItem it = ns_item(p, w, id);
        const NsTile t = ns_tile<TWIN>(p, it);
        const int mode = ns_mode(p, it), acc = n & 1, rank = TWIN ? 0 : (int)sm.rank;
        it.e = ns_own<TWIN>(p, it.e, sm.rank);
        const bool real = it.e < p.N;   // (an odd stack's last item has one matrix)
        if (!mbar_wait(sm.tfull + 8 * acc, (uint32_t)(n >> 1) & 1u, p.limit_ns, abort_flag)) {
            ns_abort(abort_flag, p.status, SITE_NS_WAIT_TFULL, id);
            live = false;
        }
        tc_fence_after();
        const uint32_t tbase = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)acc * NS_MAXBN +
                               (TWIN ? sm.rank * (uint32_t)(t.mma_n / 2) : 0u);
        const uint32_t tempty = peer_addr(sm.tempty, 0) + 8 * acc;
#pragma unroll 1
        for (int c0 = 0; c0 < t.bn; c0 += 64) {
            uint8_t* slot = sm.slot_ptr + s * NS_SLOT_BYTES;
            uint32_t v[32];
            tmem_ld_32x32b_x32(tbase + c0 + half * 32, v);   // (past a 32-wide last block: not used)
            float4 wv[8];   // the weights of this thread's piece of the block, while its inputs arrive
            if (mode == NS_M_W) {
                const int q = threadIdx.x & 15, col = t.n0 + c0 + 4 * q;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int gr = t.m0 + rank * NS_HALF + (int)(threadIdx.x >> 4) + 16 * i;
                    wv[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (real && 4 * q < t.bn - c0 && col + 4 <= p.c && gr < p.r)
                        wv[i] = *reinterpret_cast<const float4*>(p.W + it.e * p.st_w + gr * p.ld_w + col);
                }
            }
            if (!mbar_wait(sm.in + 8 * s, ph, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_SLOT, id);
                live = false;
            }
            tmem_wait_ld();
            if (c0 + 64 >= t.bn) {   // this warp's last read of the accumulator
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(tempty);
            }
            if (mode == NS_M_GRAM) ns_block<NS_M_GRAM>(p, it, t, slot, row, half, rank, c0, live && real, v, wv);
            else if (mode == NS_M_POLY) ns_block<NS_M_POLY>(p, it, t, slot, row, half, rank, c0, live && real, v, wv);
            else if (mode == NS_M_X) ns_block<NS_M_X>(p, it, t, slot, row, half, rank, c0, live && real, v, wv);
            else if (mode == NS_M_O) ns_block<NS_M_O>(p, it, t, slot, row, half, rank, c0, live && real, v, wv);
            else ns_block<NS_M_W>(p, it, t, slot, row, half, rank, c0, live && real, v, wv);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.done + 8 * s);
            if (++s == NS_SLOTS) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

template <bool TWIN>
__global__ void __launch_bounds__(NS_THREADS, 1) ns_kernel(const __grid_constant__ NsArgs p) {
    extern __shared__ uint8_t ns_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ns_smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    uint8_t* after = smem + NS_RING_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(after + NS_SLOTS * NS_SLOT_BYTES);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + NS_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    NsSmem sm;
    sm.ring = smem_u32(smem);
    sm.slot_ptr = after;
    sm.slots = smem_u32(after);
    sm.full = smem_u32(bars);
    sm.empty = sm.full + 8 * NS_RING_MAX;
    sm.tfull = sm.empty + 8 * NS_RING_MAX;
    sm.tempty = sm.tfull + 16;
    sm.drain = sm.tempty + 16;
    sm.in = sm.drain + 8;
    sm.done = sm.in + 8 * NS_SLOTS;
    sm.free_ = sm.done + 8 * NS_SLOTS;
    const bool four = p.bn == NS_MAXBN || TWIN;
    sm.stage_bytes = (four ? 4 : 3) * NS_BOX;
    sm.stages = four ? 4 : NS_RING_MAX;
    sm.rank = cluster_rank();
    sm.pair = blockIdx.x >> 1;
    sm.npairs = gridDim.x >> 1;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < sm.stages; ++s) {
            mbar_init(sm.full + 8 * s, 1);
            mbar_init(sm.empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sm.tfull + 8 * a, 1);
            mbar_init(sm.tempty + 8 * a, 2 * NS_EPI_WARPS);
        }
        mbar_init(sm.drain, 1);
        for (int s = 0; s < NS_SLOTS; ++s) {
            mbar_init(sm.in + 8 * s, 1);
            mbar_init(sm.done + 8 * s, NS_EPI_WARPS);
            mbar_init(sm.free_ + 8 * s, 1);
        }
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == NS_WARP_MMA) {
        tmem_alloc_pair(smem_u32(tmem_slot), 2 * NS_MAXBN);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // barriers of both CTAs initialised before any remote arrival
    tc_fence_after();
    pdl_wait();
    const uint32_t tmem = *tmem_slot;
    if (warp < NS_EPI_WARPS) {
        ns_epilogue<TWIN>(p, sm, tmem, abort_flag);
    } else if (warp == NS_WARP_LOAD) {
        if (elect_one()) ns_producer<TWIN>(p, sm, abort_flag);
    } else if (warp == NS_WARP_MMA) {
        if (sm.rank == 0 && elect_one()) ns_mma<TWIN>(p, sm, tmem, abort_flag);
    } else if (warp == NS_WARP_IN) {
        if (elect_one()) ns_inputs<TWIN>(p, sm, abort_flag);
    } else if (warp == NS_WARP_OUT) {
        if (elect_one()) ns_outputs<TWIN>(p, sm, abort_flag);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == NS_WARP_MMA) settle_copies(abort_flag);
    cluster_sync();   // the leader's MMAs have drained; both CTAs are done with TMEM
    if (warp == NS_WARP_MMA) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 2 * NS_MAXBN);
    }
}

// ------------------------------------------------------------- thin matrices

// m <= NS_THIN: fp32 throughout.  All factors of the step polynomials are polynomials of
// A = X0 X0^T and commute, so the iteration runs on symmetric 32 x 32 matrices in shared memory
// (P = a I + b A + c A^2, Q <- P Q, A <- P A P; zeros past m) and X is read twice: for A and for
// Q X0.  But each A <- P A P multiplies the roundings of A between its null directions by up to
// the square of the polynomial's largest gain (a^2 = 12 for the default quintic), where the iteration
// on X multiplies X's by the gain.  So the steps are cut into segments: a new one, which forms A from X
// again, begins before a step for which that growth would pass NS_GROWTH (the default quintic: after
// three steps).  Errors on X0 of rank 1: five steps 4e-5 (in one segment 2e-3), seven 5e-4 (0.25), ten
// 1e-2 (NaN), as the iteration on X in fp32 has them; cut after two steps they are the same.
// Q X0.  Thin matrices are kept off the tensor cores for accuracy as much as for time: with few
// singular values the fp16 roundings do not average out over the entries (a 1 x n matrix is one
// number per step, and its result was 5e-3 off), and their tiles would be mostly empty.
//
// A cluster of up to 8 CTAs per matrix, each with every so many 128 columns of the long side; the
// parts of A are added in CTA order over distributed shared memory, and every CTA iterates for
// itself.  Bound by latency (loads of a chunk 3 us, the iteration 8 us): 32 x 2048 34 us, a stack of 256
// of them 255 us, of which the second segment's passes over X are 10 and 97.
constexpr int NS_THIN_THREADS = 256;
constexpr double NS_GROWTH = 150.0;   // of roundings in A within a segment
constexpr int NS_THIN_K = 128;
constexpr int NS_THIN_LD = NS_THIN + 4;
constexpr int NS_THIN_CLUSTER = 8;

// A thread's elements of a chunk of S x K of the m x n orientation, in memory order over the
// threads: (i0 + di u, kk0 + dk u).
template <int S, int K>
struct NsPlace {
    int i0, di, kk0, dk;
    static constexpr int PER = S * K / NS_THIN_THREADS;
    __device__ __forceinline__ explicit NsPlace(bool tall) {
        const int t = threadIdx.x;
        i0 = tall ? t % S : t / K;
        kk0 = tall ? t / S : t % K;
        di = tall ? 0 : NS_THIN_THREADS / K;
        dk = tall ? NS_THIN_THREADS / S : 0;
    }
};
// xs[i][kk] = X (i, k0 + kk), zeros outside, by the whole CTA: X0 from the update (`first`), or X as the
// segment before left it.
template <int S, int K>
__device__ __forceinline__ void ns_stage(const NsArgs& p, int e, int k0, bool first, float pre, float post,
                                         float (*xs)[K + 4]) {
    const NsPlace<S, K> w(p.tall);
    const int m = p.m, n = p.tall ? p.r : p.c;
    const int64_t ld = first ? p.u.ld_u : p.ldx, d = (p.tall ? w.dk : w.di) * ld;
    const int64_t at = e * (first ? p.u.st_u : (int64_t)p.r * p.ldx) +
                       (p.tall ? (k0 + w.kk0) * ld + w.i0 : w.i0 * ld + k0 + w.kk0);
    auto load = [&](auto get, float pre, float post) {
        float v[w.PER];
#pragma unroll
        for (int u = 0; u < w.PER; ++u)
            v[u] = w.i0 + w.di * u < m && k0 + w.kk0 + w.dk * u < n ? get(at + u * d) : 0.f;
#pragma unroll
        for (int u = 0; u < w.PER; ++u) xs[w.i0 + w.di * u][w.kk0 + w.dk * u] = (v[u] * pre) * post;
    };
    const float* M = p.u.M;
    const float* U = static_cast<const float*>(p.u.U);
    const __nv_bfloat16* B = static_cast<const __nv_bfloat16*>(p.u.U);
    const float* X = p.X1;
    const float mu = p.u.mu;
    if (!first) load([=](int64_t a) { return X[a]; }, 1.f, 1.f);
    else if (M && !p.u.nesterov) load([=](int64_t a) { return M[a]; }, pre, post);
    else if (M) load([=](int64_t a) { return fmaf(mu, M[a], U[a]); }, pre, post);   // (with a momentum, U is fp32)
    else if (p.u.u_bf16) load([=](int64_t a) { return as_f32(B[a]); }, pre, post);
    else load([=](int64_t a) { return U[a]; }, pre, post);
    __syncthreads();
}
// The chunk's results from xs to O or into the weights (`last`), or for the next segment, in which the
// same thread reads each element again.
template <int S, int K>
__device__ __forceinline__ void ns_store(const NsArgs& p, int e, int k0, bool last, const float (*xs)[K + 4]) {
    const NsPlace<S, K> w(p.tall);
    const int m = p.m, n = p.tall ? p.r : p.c;
    const int64_t ld = !last ? p.ldx : p.O ? p.ld_o : p.ld_w, d = (p.tall ? w.dk : w.di) * ld;
    const int64_t at = e * (!last ? (int64_t)p.r * p.ldx : p.O ? p.st_o : p.st_w) +
                       (p.tall ? (k0 + w.kk0) * ld + w.i0 : w.i0 * ld + k0 + w.kk0);
    auto inside = [&](int u) { return w.i0 + w.di * u < m && k0 + w.kk0 + w.dk * u < n; };
    if (!last) {
#pragma unroll
        for (int u = 0; u < w.PER; ++u)
            if (inside(u)) p.X1[at + u * d] = xs[w.i0 + w.di * u][w.kk0 + w.dk * u];
        return;
    }
    if (p.O) {
#pragma unroll
        for (int u = 0; u < w.PER; ++u)
            if (inside(u)) p.O[at + u * d] = __float2bfloat16_rn(xs[w.i0 + w.di * u][w.kk0 + w.dk * u]);
        return;
    }
    float v[w.PER];
#pragma unroll
    for (int u = 0; u < w.PER; ++u) v[u] = inside(u) ? p.W[at + u * d] : 0.f;
#pragma unroll
    for (int u = 0; u < w.PER; ++u)
        if (inside(u)) {
            const float o = fmaf(-p.rate, xs[w.i0 + w.di * u][w.kk0 + w.dk * u], p.decay * v[u]);
            p.W[at + u * d] = o;
            if (p.Wb) p.Wb[at + u * d] = __float2bfloat16_rn(o);
        }
}

__global__ void __launch_bounds__(NS_THIN_THREADS, 3) ns_thin_kernel(const __grid_constant__ NsArgs p) {
    pdl_wait();
    typedef float Square[NS_THIN][NS_THIN_LD];
    __shared__ __align__(16) Square sq[4];
    __shared__ __align__(16) float xs[NS_THIN][NS_THIN_K + 4];
    const int tid = threadIdx.x, m = p.m, n = p.tall ? p.r : p.c;
    const int C = p.thin_cluster, e = blockIdx.x / C, rank = blockIdx.x % C;
    const int chunks = (n + NS_THIN_K - 1) / NS_THIN_K;
    float pre, post;
    norm_scales(p.u, e, pre, post);
    // A: four groups of 64 threads share a chunk's columns, a thread has rows ti + 8 u, columns tj + 8 v
    const int g = tid >> 6, ti = tid >> 3 & 7, tj = tid & 7;
    float acc[4][4] = {};
    auto gram = [&]() {   // of the chunk in xs
#pragma unroll 2
        for (int q = 0; q < NS_THIN_K / 16; ++q) {
            const int kk = (g * (NS_THIN_K / 16) + q) * 4;
            float4 a[4], b[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                a[u] = *reinterpret_cast<const float4*>(&xs[ti + 8 * u][kk]);
                b[u] = *reinterpret_cast<const float4*>(&xs[tj + 8 * u][kk]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float lo = fmaf(a[u].y, b[v].y, fmaf(a[u].x, b[v].x, acc[u][v]));
                    acc[u][v] = fmaf(a[u].w, b[v].w, fmaf(a[u].z, b[v].z, lo));
                }
        }
        if (chunks > C) __syncthreads();   // (one chunk a CTA: it stays in xs)
    };
    for (int ch = rank; ch < chunks; ch += C) {
        ns_stage<NS_THIN, NS_THIN_K>(p, e, ch * NS_THIN_K, true, pre, post, xs);
        gram();
    }
    for (int s0 = 0, s1; s0 < p.steps; s0 = s1) {   // segments [s0, s1)
        for (s1 = s0 + 1; s1 < p.steps && !p.restart[s1]; ++s1) {}
        const bool last = s1 == p.steps;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                sq[g][ti + 8 * u][tj + 8 * v] = acc[u][v];
                acc[u][v] = 0.f;
            }
        __syncthreads();
        // a thread's four elements of a square: row tid / 8, columns 4 (tid % 8) ..
        const int er = tid >> 3, ec = (tid & 7) * 4;
        auto at4 = [&](Square& S) { return reinterpret_cast<float4*>(&S[er][ec]); };
        float4 sum = *at4(sq[0]);
        for (int g = 1; g < 4; ++g) {
            const float4 v = *at4(sq[g]);
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        *at4(sq[0]) = sum;   // (read by this thread alone so far)
        if (C > 1) {
            const uint32_t mine = smem_u32(at4(sq[0]));
            cluster_sync();
            sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int r = 0; r < C; ++r) {
                float4 v;
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                             : "r"(peer_addr(mine, r)));
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            cluster_sync();   // every CTA has read the parts
            *at4(sq[0]) = sum;
        }
        __syncthreads();
        // out = L R for symmetric operands, `out` none of them; 2 x 2 elements a thread
        auto product = [&](Square& out, const Square& L, const Square& R) {
            const int i = (tid >> 4) * 2, j = (tid & 15) * 2;
            float2 r0 = make_float2(0.f, 0.f), r1 = r0;
#pragma unroll 8
            for (int k = 0; k < NS_THIN; ++k) {
                const float2 l = *reinterpret_cast<const float2*>(&L[k][i]), r = *reinterpret_cast<const float2*>(&R[k][j]);
                r0 = make_float2(fmaf(l.x, r.x, r0.x), fmaf(l.x, r.y, r0.y));
                r1 = make_float2(fmaf(l.y, r.x, r1.x), fmaf(l.y, r.y, r1.y));
            }
            *reinterpret_cast<float2*>(&out[i][j]) = r0;
            *reinterpret_cast<float2*>(&out[i + 1][j]) = r1;
            __syncthreads();
        };
        Square& A = sq[0];
        Square& P = sq[1];
        int iq = 2, it2 = 3;   // where Q and the scratch matrix are
        for (int it = s0; it < s1; ++it) {
            const float ca = p.coef[3 * it], cb = p.coef[3 * it + 1], cc = p.coef[3 * it + 2];
            product(sq[it2], A, A);
            const float4 a = *at4(A), t = *at4(sq[it2]);
            float4 v = make_float4(fmaf(cc, t.x, cb * a.x), fmaf(cc, t.y, cb * a.y), fmaf(cc, t.z, cb * a.z), fmaf(cc, t.w, cb * a.w));
            v.x += er == ec ? ca : 0.f;
            v.y += er == ec + 1 ? ca : 0.f;
            v.z += er == ec + 2 ? ca : 0.f;
            v.w += er == ec + 3 ? ca : 0.f;
            *at4(P) = v;
            if (it == s0) *at4(sq[iq]) = v;
            __syncthreads();
            if (it > s0) {
                product(sq[it2], P, sq[iq]);
                iq ^= 1;   // 2 and 3 change places
                it2 ^= 1;
            }
            if (it + 1 < s1) {
                product(sq[it2], P, A);
                product(A, sq[it2], P);
            }
        }
        // Q is the product of the steps' P, the last one leftmost: in that order a rounding in one of them is
        // multiplied by those after it, as in the iteration on X itself.  (In the other order, that of the
        // transpose, the last P's roundings go through all earlier ones: on X0 of rank 1 the result was off
        // by 0.8.)  Transposed, so that a row's factors lie side by side.
        {
            const float4 v = *at4(sq[iq]);
            sq[it2][ec][er] = v.x;
            sq[it2][ec + 1][er] = v.y;
            sq[it2][ec + 2][er] = v.z;
            sq[it2][ec + 3][er] = v.w;
            __syncthreads();
        }
        // Q X: 4 rows x 4 columns a thread, through xs to memory order; the next segment's A on the way
        const Square& QT = sq[it2];
        for (int ch = rank; ch < chunks; ch += C) {
            const int k0 = ch * NS_THIN_K, c4 = (tid & 31) * 4, r4 = (tid >> 5) * 4;
            if (chunks > C) ns_stage<NS_THIN, NS_THIN_K>(p, e, k0, s0 == 0, pre, post, xs);
            float4 o[4] = {};
#pragma unroll 4
            for (int j = 0; j < m; ++j) {
                const float4 x = *reinterpret_cast<const float4*>(&xs[j][c4]), q = *reinterpret_cast<const float4*>(&QT[j][r4]);
                const float qs[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    o[u] = make_float4(fmaf(qs[u], x.x, o[u].x), fmaf(qs[u], x.y, o[u].y), fmaf(qs[u], x.z, o[u].z),
                                       fmaf(qs[u], x.w, o[u].w));
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 4; ++u) *reinterpret_cast<float4*>(&xs[r4 + u][c4]) = o[u];
            __syncthreads();
            if (last || chunks > C) ns_store<NS_THIN, NS_THIN_K>(p, e, k0, last, xs);
            if (last) __syncthreads();
            else gram();
        }
    }
}

// ---------------------------------------------------- few narrow matrices

// NS_THIN < m <= NS_SMALL, the same iteration in fp32 by a cluster of 8 CTAs per matrix: each forms
// the part of A from its columns of X and then has 8 rows of every product, one a warp.  All factors
// being symmetric and commuting, rows of Q P, A P and (A P) P need only the CTA's own rows of the
// left factor, so P and A alone are shared, in every CTA's memory.  For few matrices: on the tensor
// cores the Gram product of one such matrix is a single tile, n / 64 K blocks one after the other,
// and every step three dependent launches' worth of hand-over.
// Bound by shared memory and the fp32 units of its 8 SMs: 64 x 512 in 37 us, 64 x 2048 in 73, 12 for each
// pass over X.  (128 x 2048 in the same way took 200 us, 115 on the tensor cores; 256 x 100, the best
// of those above 64, 104 and 100.)
constexpr int NS_SMALL = 64;
constexpr int NS_SMALL_K = 64;
constexpr int NS_SMALL_ROWS = NS_SMALL / 8;   // of a CTA
constexpr int NS_SMALL_LD = NS_SMALL + 4;
constexpr int NS_SMALL_SMEM = 4 * ((2 * NS_SMALL + 2 * NS_SMALL_ROWS) * NS_SMALL_LD + NS_SMALL * (NS_SMALL_K + 4));

// Writes two consecutive floats at the same place of every CTA of the cluster.
__device__ __forceinline__ void ns_share(const float* at, const float (&v)[2]) {
    const uint32_t mine = smem_u32(at);
#pragma unroll
    for (int r = 0; r < 8; ++r)
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(peer_addr(mine, r)), "f"(v[0]), "f"(v[1]) : "memory");
}

// out[i] = rows[i] . R; a lane has two consecutive columns.
template <int NR>
__device__ __forceinline__ void ns_rows(float (&out)[NR][2], const float* const (&rows)[NR], const float (*Rm)[NS_SMALL_LD]) {
    const int c = (threadIdx.x & 31) * 2;
#pragma unroll
    for (int i = 0; i < NR; ++i) out[i][0] = out[i][1] = 0.f;
#pragma unroll 2
    for (int k = 0; k < NS_SMALL; k += 4) {
        float l[NR][4];
#pragma unroll
        for (int i = 0; i < NR; ++i) *reinterpret_cast<float4*>(l[i]) = *reinterpret_cast<const float4*>(rows[i] + k);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 r = *reinterpret_cast<const float2*>(&Rm[k + q][c]);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                out[i][0] = fmaf(l[i][q], r.x, out[i][0]);
                out[i][1] = fmaf(l[i][q], r.y, out[i][1]);
            }
        }
    }
}

__global__ void __launch_bounds__(NS_THIN_THREADS, 2) ns_small_kernel(const __grid_constant__ NsArgs p) {
    constexpr int S = NS_SMALL, K = NS_SMALL_K, TI = S / 16;
    extern __shared__ __align__(16) float ns_small_mem[];
    typedef float Row[NS_SMALL_LD];
    Row* A = reinterpret_cast<Row*>(ns_small_mem);
    Row* P = A + S;
    Row* Qs = P + S;   // this CTA's rows of Q and of A P
    Row* Ts = Qs + NS_SMALL_ROWS;
    typedef float XRow[K + 4];
    XRow* xs = reinterpret_cast<XRow*>(Ts + NS_SMALL_ROWS);
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, m = p.m, n = p.tall ? p.r : p.c;
    const int e = blockIdx.x / 8, rank = (int)cluster_rank(), chunks = (n + K - 1) / K;
    float pre, post;
    norm_scales(p.u, e, pre, post);
    // this CTA's part of A: rows ti + 16 u, columns tj + 16 v
    const int ti = tid >> 4, tj = tid & 15;
    float acc[TI][TI] = {};
    auto gram = [&]() {   // of the chunk in xs
#pragma unroll 1
        for (int kk = 0; kk < K; kk += 4) {
            float4 b[TI];
#pragma unroll
            for (int v = 0; v < TI; ++v) b[v] = *reinterpret_cast<const float4*>(&xs[tj + 16 * v][kk]);
#pragma unroll
            for (int u = 0; u < TI; ++u) {
                const float4 a = *reinterpret_cast<const float4*>(&xs[ti + 16 * u][kk]);
#pragma unroll
                for (int v = 0; v < TI; ++v)
                    acc[u][v] = fmaf(a.w, b[v].w, fmaf(a.z, b[v].z, fmaf(a.y, b[v].y, fmaf(a.x, b[v].x, acc[u][v]))));
            }
        }
        if (chunks > 8) __syncthreads();   // (one chunk a CTA: it stays in xs)
    };
    for (int ch = rank; ch < chunks; ch += 8) {
        ns_stage<S, K>(p, e, ch * K, true, pre, post, xs);
        gram();
    }
    for (int s0 = 0, s1; s0 < p.steps; s0 = s1) {   // segments [s0, s1)
        for (s1 = s0 + 1; s1 < p.steps && !p.restart[s1]; ++s1) {}
        const bool final = s1 == p.steps;
#pragma unroll
        for (int u = 0; u < TI; ++u)
#pragma unroll
            for (int v = 0; v < TI; ++v) {
                A[ti + 16 * u][tj + 16 * v] = acc[u][v];
                acc[u][v] = 0.f;
            }
        // the sum of the parts, this CTA's rows first, then everyone's
        const int row = rank * NS_SMALL_ROWS + warp, col = lane * 2;   // a warp's row, a lane's columns
        float t[1][2] = {};
        cluster_sync();
        const uint32_t mine = smem_u32(&A[row][col]);
        for (int r = 0; r < 8; ++r) {
            float x, y;
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x), "=f"(y) : "r"(peer_addr(mine, r)));
            t[0][0] += x;
            t[0][1] += y;
        }
        cluster_sync();
        ns_share(&A[row][col], t[0]);
        cluster_sync();
        for (int it = s0; it < s1; ++it) {
            const float ca = p.coef[3 * it], cb = p.coef[3 * it + 1], cc = p.coef[3 * it + 2];
            const float* const a_row[1] = {A[row]};
            ns_rows<1>(t, a_row, A);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                t[0][j] = fmaf(cc, t[0][j], cb * A[row][col + j]) + (row == col + j ? ca : 0.f);
                if (it == s0) Qs[warp][col + j] = t[0][j];
            }
            ns_share(&P[row][col], t[0]);
            cluster_sync();   // P is complete
            // rows of Q P and of A P, then of (A P) P; a warp's rows of Q and A P are its own
            float o[2][2];
            const float* const rows[2] = {Qs[warp], A[row]};
            ns_rows<2>(o, rows, P);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (it > s0) Qs[warp][col + j] = o[0][j];
                Ts[warp][col + j] = o[1][j];
            }
            __syncwarp();
            if (it + 1 == s1) break;
            const float* const t_row[1] = {Ts[warp]};
            ns_rows<1>(t, t_row, P);
            ns_share(&A[row][col], t[0]);
            cluster_sync();   // A is complete, and P free
        }
        cluster_sync();   // P free
        const float q2[2] = {Qs[warp][col], Qs[warp][col + 1]};
        ns_share(&P[row][col], q2);
        cluster_sync();
        // Q X: 4 rows x 4 columns a thread, through xs to memory order; the next segment's A on the way
        for (int ch = rank; ch < chunks; ch += 8) {
            const int c4 = (tid & 15) * 4, r0 = (tid >> 4) * TI;
            if (chunks > 8) ns_stage<S, K>(p, e, ch * K, s0 == 0, pre, post, xs);
            float4 o[TI] = {};
#pragma unroll 2
            for (int j = 0; j < m; ++j) {
                const float4 x = *reinterpret_cast<const float4*>(&xs[j][c4]);
                float q[TI];
#pragma unroll
                for (int u = 0; u < TI; u += 4) *reinterpret_cast<float4*>(q + u) = *reinterpret_cast<const float4*>(&P[j][r0 + u]);
#pragma unroll
                for (int u = 0; u < TI; ++u)
                    o[u] = make_float4(fmaf(q[u], x.x, o[u].x), fmaf(q[u], x.y, o[u].y), fmaf(q[u], x.z, o[u].z),
                                       fmaf(q[u], x.w, o[u].w));
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < TI; ++u) *reinterpret_cast<float4*>(&xs[r0 + u][c4]) = o[u];
            __syncthreads();
            if (final || chunks > 8) ns_store<S, K>(p, e, ch * K, final, xs);
            if (final) __syncthreads();
            else gram();
        }
    }
}

inline int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

// Matrices under way: as many as keep the working arrays within this, in NS_LANES groups.  Fewer
// keep more of them in L2, but a slot of the schedule must hold several tiles for every pair, as a
// tile's inputs are about 12 us old before the next can start on them.  Measured on 256 x 416 x 1664:
// 48 MB 5.2 ms, 72 MB 3.8, 100 MB 3.3, 140 MB 2.8, 220 MB 2.5, 400 MB 2.4.  A stack that is under way as a
// whole forms one group: with two, its schedule is one stage longer and its tiles wait as much
// (16 x 768 x 768 212 us instead of 224, 13 x 1889 x 354 263 instead of 297).
constexpr int64_t NS_UNDER_WAY_BYTES = 384ll << 20;
// Stacks of at least so many wide matrices of m <= 128 go through the tiles two by two, a CTA of the
// pair for each: rows 0 .. 127 of a tile and the first half of its columns belong to the one, the
// rest to the other (what the MMA forms of one's rows and the other's columns is not read).  One by
// one, every tile left a CTA without rows: 147 of 90 x 770 390 us instead of 266, 128 of 128 x 2048 574
// instead of 471.  Tall matrices fill both CTAs in the apply stage and lose (64 of 2048 x 100 345 us
// instead of 365 two by two), as do squares (64 of 128 x 128 100 and 109).
constexpr int NS_TWIN_MIN = 64;

struct NsLayout {
    size_t prog, part, x0h, x0l, xh0, xh1, xl0, xl1, A, Al, B, Bl, total;
    int chunk, chunks, groups, n_groups, group_max, slots, terms, twin, units;
};
int ns_terms(int64_t m) { return m <= 128 ? 3 : 1; }
// Whether stacks of N matrices go through the tiles two by two.
bool ns_twin(int64_t N, int64_t r, int64_t c) { return r > NS_THIN && r <= NS_HALF && r < c && N >= NS_TWIN_MIN; }
// Units (matrices, or twos) of a group at most.
int64_t ns_group_most(int64_t r, int64_t c, bool twin) {
    const int64_t m = r < c ? r : c, x = r * up8(c), a = m * up8(m);
    const int64_t each = ns_terms(m) == 3 ? 8 * x + 8 * a : 6 * x + 4 * a, most = NS_UNDER_WAY_BYTES / (each * (twin ? 2 : 1) * NS_LANES);
    return most > 1 ? most : 1;
}
// Matrices under way at most in any stack of up to N: all of a stack that fits in one round, which
// more matrices, as they take more rounds of even size, fall short of.
int64_t ns_most_slots(int64_t N, int64_t r, int64_t c) {
    auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
    if (!ns_twin(N, r, c)) return least(N, ns_group_most(r, c, false) * NS_LANES);
    const int64_t single = least(NS_TWIN_MIN - 1, ns_group_most(r, c, false) * NS_LANES);
    const int64_t twos = 2 * least((N + 1) / 2, ns_group_most(r, c, true) * NS_LANES);
    return single > twos ? single : twos;
}

// The schedule's groups and the places of the buffers in the workspace; total: for any stack of up to N.
NsLayout ns_layout(int64_t N, int64_t r, int64_t c) {
    NsLayout L;
    const int64_t m = r < c ? r : c, ldx = up8(c), ldm = up8(m);
    L.groups = (int)(r * ldx / 8);
    L.chunk = (L.groups + NS_PRO_CHUNKS - 1) / NS_PRO_CHUNKS;
    if (L.chunk < NS_PRO_GROUPS) L.chunk = NS_PRO_GROUPS;
    L.chunks = (L.groups + L.chunk - 1) / L.chunk;
    L.terms = ns_terms(m);
    L.twin = ns_twin(N, r, c);
    const int64_t units = L.twin ? (N + 1) / 2 : N;          // what items are made of
    L.units = (int)units;
    const int64_t most = ns_group_most(r, c, L.twin);
    const int64_t rounds = (units + most * NS_LANES - 1) / (most * NS_LANES);
    L.n_groups = (int)(rounds * NS_LANES < units ? rounds * NS_LANES : units);   // sizes then differ by one at most
    if (rounds <= 1) L.n_groups = 1;
    L.group_max = (int)((units + L.n_groups - 1) / L.n_groups);
    L.slots = L.group_max * (L.n_groups < NS_LANES ? L.n_groups : NS_LANES) * (L.twin ? 2 : 1);
    const size_t room = (size_t)ns_most_slots(N, r, c);      // at least `slots`
    size_t o = up256(sizeof(DevStatus));
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    L.prog = take((size_t)N * 4);
    L.part = take((size_t)N * L.chunks * 3 * sizeof(float));
    const size_t x = room * r * ldx * 2, a = room * m * ldm * 2;
    const bool thin = m <= NS_THIN;
    L.x0h = take((size_t)N * r * ldx * (thin ? 4 : 2));   // (thin, and few narrow matrices from here on: X in fp32)
    L.x0l = take(thin ? 0 : (size_t)N * r * ldx * 2);
    L.xh0 = take(thin ? 0 : x);
    L.xh1 = take(thin ? 0 : x);
    L.xl0 = take(thin ? 0 : x);
    L.xl1 = L.terms == 3 ? take(thin ? 0 : x) : L.xl0;
    L.A = take(thin ? 0 : a);
    L.B = take(thin ? 0 : a);
    L.Al = L.terms == 3 ? take(thin ? 0 : a) : L.A;
    L.Bl = L.terms == 3 ? take(thin ? 0 : a) : L.B;
    L.total = o;
    return L;
}

// The update's norms (and momentum), and X0 unless the matrices are thin.
template <typename T, bool VEC>
cudaError_t launch_prologue(const UpdateArgs& p, int N, bool thin, __half* xh, __half* xl, cudaStream_t s) {
    const dim3 grid((unsigned)p.chunks, (unsigned)N);
    cudaError_t e = launch_pdl(muon_moment_kernel<T, VEC>, grid, dim3(NS_PRO_THREADS), 0, s, p);
    count_launches(1);
    if (e != cudaSuccess || thin) return e;
    count_launches(1);
    return launch_pdl(muon_scale_kernel, grid, dim3(NS_PRO_THREADS), 0, s, p, xh, xl);
}

}  // namespace

// Monotone in N, as each buffer's size is.
size_t ns_workspace_bytes(int64_t N, int64_t r, int64_t c) { return ns_layout(N, r, c).total; }

namespace {
// Launch attributes of a kernel with a cluster per matrix.
struct NsClusterLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    NsClusterLaunch(int N, int ctas, int smem, cudaStream_t s) {
        cfg.gridDim = dim3((unsigned)(N * ctas));
        cfg.blockDim = dim3(NS_THIN_THREADS);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.stream = s;
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)ctas;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see launch_pdl
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at;
        cfg.numAttrs = 2;
    }
};
// Clusters of `ctas` CTAs of a kernel that run at a time on the current device (0: none), its shared
// memory attribute set on the way; `cache`: per device, count + 1.
int clusters_at_once(std::atomic<int> (&cache)[64], void (*kern)(NsArgs), int ctas, int threads, int smem) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = cache[dev].load(std::memory_order_acquire) - 1;
    if (n >= 0) return n;
    n = 0;
    NsClusterLaunch l(1, ctas, smem, nullptr);
    l.cfg.blockDim = dim3((unsigned)threads);
    l.cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &l.cfg) != cudaSuccess || n < 0) {
        cudaGetLastError();
        n = 0;
    }
    cache[dev].store(n + 1, std::memory_order_release);
    return n;
}
int ns_small_clusters() {
    static std::atomic<int> cache[64];
    return clusters_at_once(cache, ns_small_kernel, 8, NS_THIN_THREADS, NS_SMALL_SMEM);
}
template <bool TWIN>
int ns_pairs() {
    static std::atomic<int> cache[64];
    return clusters_at_once(cache, ns_kernel<TWIN>, 2, NS_THREADS, NS_SMEM);
}
// Whether the cluster kernel is the faster one for N matrices m x n: times (us, five steps of the default
// quintic) of both, fitted to measurements at m of 40 and 64, n of 64 to 4096, N of 1 to 100.  Cluster
// kernel and tensor cores: one 64 x 64 37 and 69, one 64 x 2048 73 and 104, 32 of them 120 and 180, 64
// 232 and 213; 64 of 64 x 64 96 and 77; 18 of 4096 x 64 201 and 191.
bool ns_small_pays(int N, int m, int n, bool tall) {
    if (m <= NS_THIN || m > NS_SMALL) return false;
    const int at_once = ns_small_clusters();
    if (at_once <= 0) return false;
    // two CTAs per SM; up to a quarter as many clusters have an SM per CTA; up to 512 columns stay on chip
    const int full = N / at_once, rest = N - full * at_once;
    const float here = 5.0f + full * (48.0f + 0.041f * fmaxf(0.f, n - 450.0f)) +
                       (rest == 0 ? 0.f : 4 * rest <= at_once ? 32.0f + 0.0227f * fmaxf(0.f, n - 430.0f)
                                                               : 48.0f + 0.041f * fmaxf(0.f, n - 450.0f));
    const float tensor = tall ? 68.0f + 0.016f * n + N * (0.08f + 0.00072f * n)
                              : 68.0f + 0.017f * n + (N >= NS_TWIN_MIN ? 0.7f : 1.0f) * N * (0.12f + 0.00115f * n);
    return here < tensor;
}
}  // namespace

// Largest values over a step's singular values in [0, s]: each lies at the end of the interval or where
// the derivative is zero.
NsBounds ns_bounds(const float* coef, double s) {
    const double a = coef[0], b = coef[1], c = coef[2], t = s * s;
    NsBounds r;
    auto b_of = [&](double u) { return fabs(b * u + c * u * u); };
    auto gain_of = [&](double u) { return fabs(a + b * u + c * u * u); };
    const double v = c != 0.0 ? -b / (2.0 * c) : -1.0;
    r.b = b_of(t);
    r.gain = fmax(gain_of(0.0), gain_of(t));
    if (v > 0.0 && v < t) {
        r.b = fmax(r.b, b_of(v));
        r.gain = fmax(r.gain, gain_of(v));
    }
    r.largest = s * gain_of(t);
    // (a + 3 b u + 5 c u^2 = 0; one root by a quotient that c = 0 leaves finite)
    const double disc = 9.0 * b * b - 20.0 * a * c;
    if (disc >= 0.0) {
        const double q = -0.5 * (3.0 * b + copysign(sqrt(disc), b));
        for (const double u : {q != 0.0 ? a / q : -1.0, c != 0.0 ? q / (5.0 * c) : -1.0})
            if (u > 0.0 && u < t) r.largest = fmax(r.largest, sqrt(u) * gain_of(u));
    }
    return r;
}

cudaError_t launch_newton_schulz(const NsCall& q, uint8_t* ws, int sms, uint64_t limit_ns, cudaStream_t s) {
    const NsLayout L = ns_layout(q.N, q.r, q.c);
    NsArgs a = {};
    a.N = q.N;
    a.r = q.r;
    a.c = q.c;
    a.tall = q.r > q.c;
    a.m = a.tall ? q.c : q.r;
    a.ldx = (int)up8(q.c);
    a.ldm = (int)up8(a.m);
    a.terms = L.terms;
    a.u.U = q.U;
    a.u.ld_u = q.ld_u;
    a.u.st_u = q.st_u;
    a.u.u_bf16 = q.u_bf16;
    a.u.vec = q.ld_u % 8 == 0 && q.st_u % 8 == 0 && (reinterpret_cast<uintptr_t>(q.U) & 15u) == 0;
    a.u.M = q.M;
    a.u.mu = q.momentum;
    a.u.nesterov = q.nesterov;
    a.u.r = q.r;
    a.u.c = q.c;
    a.u.gpr = a.ldx / 8;
    a.u.groups = L.groups;
    a.u.chunk = L.chunk;
    a.u.chunks = L.chunks;
    a.u.part = reinterpret_cast<float*>(ws + L.part);
    a.u.prog = reinterpret_cast<int32_t*>(ws + L.prog);
    a.xh[0] = reinterpret_cast<__half*>(ws + L.x0h);
    a.xl[0] = reinterpret_cast<__half*>(ws + L.x0l);
    a.X1 = reinterpret_cast<float*>(ws + L.x0h);
    const bool thin = a.m <= NS_THIN, small = ns_small_pays(a.N, a.m, a.tall ? a.r : a.c, a.tall);

    a.steps = q.steps;
    int stage = 0;
    for (int it = 0; it < q.steps; ++it) {
        for (int j = 0; j < 3; ++j) a.coef[3 * it + j] = q.coef[3 * it + j];
        // lo in the last two steps: see the file comment
        const float ca = q.coef[3 * it], last = fabsf(q.coef[3 * (q.steps - 1)]), lim = it == q.steps - 1 ? 0.0f : 2.0f;
        const bool less = a.terms == 1 && it >= q.steps - 2 && it > 0 && fabsf(ca) <= NS_LO_MAX && last <= NS_LO_MAX;
        a.lo_coef[it] = less && fabsf(ca) > lim ? copysignf(lim, ca) : ca;
        for (int kind = NS_GRAM; kind <= NS_APPLY; ++kind) {
            if (kind == NS_POLY && a.coef[3 * it + 2] == 0.f) continue;
            a.kind[stage] = (uint8_t)kind;
            a.step[stage++] = (uint8_t)it;
        }
    }
    a.n_stages = stage;
    double largest = 1.0, growth = 1.0;   // singular value of X; of roundings in A since the segment began
    for (int it = 0; it < q.steps; ++it) {
        const NsBounds b = ns_bounds(q.coef + 3 * it, largest);
        a.restart[it] = it > 0 && !(growth <= NS_GROWTH);
        if (a.restart[it]) growth = 1.0;
        growth *= b.gain > 1.0 ? b.gain * b.gain : 1.0;
        largest = b.largest;
    }
    // X's lo part is read by the next step's a X term, unless it counts 0 times there, and, with three
    // terms, by its products whatever a is.
    for (int it = 0; it + 1 < q.steps; ++it) a.lo_keep[it] = a.terms == 3 ? 1.0f : a.lo_coef[it + 1];
    a.O = q.O;
    a.ld_o = q.ld_o;
    a.st_o = q.st_o;
    a.vec_o = q.ld_o % 8 == 0 && q.st_o % 8 == 0 && (reinterpret_cast<uintptr_t>(q.O) & 15u) == 0;
    a.W = q.W;
    a.Wb = q.Wb;
    a.ld_w = q.ld_u;
    a.st_w = q.st_u;
    a.decay = q.decay;
    a.rate = q.rate;
    a.status = reinterpret_cast<DevStatus*>(ws);
    a.limit_ns = limit_ns;
    // The prologue brings M up to date in place, so it is enqueued after all that can fail on the host.
    auto prologue = [&]() {
        const bool alone = thin || small;
        if (q.u_bf16)
            return a.u.vec ? launch_prologue<__nv_bfloat16, true>(a.u, q.N, alone, a.xh[0], a.xl[0], s)
                           : launch_prologue<__nv_bfloat16, false>(a.u, q.N, alone, a.xh[0], a.xl[0], s);
        return a.u.vec ? launch_prologue<float, true>(a.u, q.N, alone, a.xh[0], a.xl[0], s)
                       : launch_prologue<float, false>(a.u, q.N, alone, a.xh[0], a.xl[0], s);
    };
    cudaError_t e;
    if (thin || small) {
        if ((e = prologue()) != cudaSuccess) return e;
        if (small) {
            NsClusterLaunch l(a.N, 8, NS_SMALL_SMEM, s);
            e = cudaLaunchKernelEx(&l.cfg, ns_small_kernel, a);
        } else {
            // CTAs of a matrix: one per 128 columns, up to about eight CTAs per SM in all
            const int n = a.tall ? a.r : a.c, room = 8 * sms / a.N;
            a.thin_cluster = (n + NS_THIN_K - 1) / NS_THIN_K;
            if (a.thin_cluster > NS_THIN_CLUSTER) a.thin_cluster = NS_THIN_CLUSTER;
            if (a.thin_cluster > room) a.thin_cluster = room > 1 ? room : 1;
            NsClusterLaunch l(a.N, a.thin_cluster, 0, s);
            e = cudaLaunchKernelEx(&l.cfg, ns_thin_kernel, a);
        }
        count_launches(1);
        return e != cudaSuccess ? e : cudaGetLastError();
    }
    a.xh[1] = reinterpret_cast<__half*>(ws + L.xh0);
    a.xh[2] = reinterpret_cast<__half*>(ws + L.xh1);
    a.xl[1] = reinterpret_cast<__half*>(ws + L.xl0);
    a.xl[2] = reinterpret_cast<__half*>(ws + L.xl1);
    a.A[0] = reinterpret_cast<__half*>(ws + L.A);
    a.A[1] = reinterpret_cast<__half*>(ws + L.Al);
    a.B[0] = reinterpret_cast<__half*>(ws + L.B);
    a.B[1] = reinterpret_cast<__half*>(ws + L.Bl);
    bool ok = true;
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 2; ++j)
            ok = ok && make_weight_tmap_strided(&a.tX[i][j], j ? a.xl[i] : a.xh[i], a.c, a.r, i ? L.slots : a.N, a.ldx,
                                                (int64_t)a.r * a.ldx);
    for (int i = 0; i < 2; ++i) {
        ok = ok && make_weight_tmap_strided(&a.tA[i], a.A[i], a.m, a.m, L.slots, a.ldm, (int64_t)a.m * a.ldm) &&
             make_weight_tmap_strided(&a.tB[i], a.B[i], a.m, a.m, L.slots, a.ldm, (int64_t)a.m * a.ldm);
    }
    if (a.W) ok = ok && make_f32_tmap(&a.tW, a.W, a.c, a.r, a.N, a.ld_w, a.N > 1 ? a.st_w : (int64_t)a.r * a.ld_w);
    if (a.O && a.vec_o)
        ok = ok && make_weight_tmap_strided(&a.tO, a.O, a.c, a.r, a.N, a.ld_o, a.N > 1 ? a.st_o : (int64_t)a.r * a.ld_o);
    if (!ok) return cudaErrorInvalidValue;
    // 256-column tiles, narrower ones where the matrices under way have fewer than there are pairs
    a.mt_s = (a.m + NS_BM - 1) / NS_BM;
    const int rows = L.twin ? NS_HALF : NS_BM;
    a.mt_x = (a.r + rows - 1) / rows;
    for (a.bn = L.twin ? NS_HALF : NS_MAXBN;; a.bn /= 2) {
        a.nt_s = (a.m + a.bn - 1) / a.bn;
        a.nt_x = (a.c + a.bn - 1) / a.bn;
        if (L.twin || a.bn == 64 || L.slots * a.mt_x * a.nt_x >= sms / 2) break;
    }
    int sym = 0;
    for (int i = 0; i < a.mt_s; ++i) sym += a.nt_s - i * (NS_BM / a.bn);
    a.tiles[NS_GRAM] = a.tiles[NS_POLY] = sym;
    a.tiles[NS_APPLY] = a.mt_x * a.nt_x;
    int64_t items = 0;
    for (int i = 0; i < a.n_stages; ++i) {
        a.need[i] = (int)items * NS_DONE;
        items += a.tiles[a.kind[i]];
    }
    a.need[a.n_stages] = (int)items * NS_DONE;
    items *= L.units;
    if (items >= (int64_t(1) << 31) - 65536) return cudaErrorInvalidValue;
    a.total = (int)items;
    a.n_groups = L.n_groups;
    a.group_max = L.group_max;
    a.base_size = L.units / L.n_groups;
    a.big_groups = L.units % L.n_groups;
    const int most = L.twin ? ns_pairs<true>() : ns_pairs<false>();   // co-resident, as they wait on one another
    if (most <= 0) return cudaErrorCooperativeLaunchTooLarge;
    const int64_t pairs = items < most ? items : most;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(NS_THREADS);
    cfg.dynamicSmemBytes = NS_SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[3];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeCooperative;   // pairs wait on one another: all co-resident
    at[1].val.cooperative = 1;
    at[2].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see launch_pdl
    at[2].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 3;
    if ((e = prologue()) != cudaSuccess) return e;
    e = cudaLaunchKernelEx(&cfg, L.twin ? ns_kernel<true> : ns_kernel<false>, a);
    count_launches(1);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mv
