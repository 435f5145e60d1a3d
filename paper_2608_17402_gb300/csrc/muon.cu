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
//   muon_moment_kernel  one pass over the gradient: momentum update (M <- mu M + G) and, per
//                       chunk, partial sums of squares of U.  Bound by memory.
//   muon_scale_kernel   X0 in the working format from U and the matrix's norm.
//   ns_gemm_kernel      the three products of a step on tcgen05, each with its epilogue.
//   ns_thin_kernel      all steps of a matrix whose smaller side is at most 32, in fp32.
//
// Working format.  X is held as hi + lo / 2048, two fp16 values (22 significant bits), times
// 2^8; A and B as fp16 times 2^8.  The tensor cores multiply the hi parts (fp16 has three
// bits more than bf16 at the same rate, and every entry of X, A and B is bounded by a few
// units, so its range suffices), accumulate in fp32, and the a X term is added from the full
// hi + lo pair in fp32.  That term is what keeps the directions in which U is (nearly)
// singular clean: each step multiplies them by a = 3.4, so a rounding of X there would grow by
// a^steps, several hundred times, while B X is small there to begin with.  Against 64 bits the
// result is within 2e-3 (2-norm over 2-norm) for full-rank and for low-rank U alike; with X
// rounded to fp16 alone it would be 4e-2 for a U of rank 16.
#include "internal.h"

#include <cuda_fp16.h>

namespace mv {

namespace {

constexpr float NS_S = 256.0f;            // scale of X, A, B in the working format
constexpr float NS_INV_S = 1.0f / 256.0f;
constexpr float NS_LO = 2048.0f;          // lo holds (x - hi) * 2^11
constexpr float NS_INV_LO = 1.0f / 2048.0f;

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
        l[q] = pack_half2((x[2 * q] - f.x) * NS_LO, (x[2 * q + 1] - f.y) * NS_LO);
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
constexpr int NS_PRO_GROUPS = 4096;   // groups of 8 values per CTA

struct ProArgs {
    const void* U;        // the update (or the gradient G) [N] x [r][ld_u]
    int64_t ld_u, st_u;
    float* M;             // momentum (NULL: U is used as it is), laid out as U
    float mu;
    int nesterov;
    int r, c, ld;         // ld: row stride of the working arrays (c rounded up to 8)
    int groups, chunks;   // groups of 8 per matrix, chunks of NS_PRO_GROUPS of them
    float* part;          // [N][chunks][3]
    __half* xh;           // [N][r][ld]
    __half* xl;
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(NS_PRO_THREADS) muon_moment_kernel(const __grid_constant__ ProArgs p) {
    pdl_wait();
    const int e = blockIdx.y, gpr = p.ld / 8;
    const int g0 = blockIdx.x * NS_PRO_GROUPS, g1 = min(g0 + NS_PRO_GROUPS, p.groups);
    const T* U = static_cast<const T*>(p.U) + e * p.st_u;
    float* M = p.M ? p.M + e * p.st_u : nullptr;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    for (int g = g0 + (int)threadIdx.x; g < g1; g += NS_PRO_THREADS) {
        const int row = g / gpr, col = (g - row * gpr) * 8, n = p.c - col;
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
    __shared__ float red[3][NS_PRO_THREADS / 32];
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
    if (threadIdx.x < 3) {
        float s = 0.f;
        for (int w = 0; w < NS_PRO_THREADS / 32; ++w) s += red[threadIdx.x][w];
        p.part[((int64_t)e * p.chunks + blockIdx.x) * 3 + threadIdx.x] = s;
    }
}

// x = (v * pre) * post in the working format, from the matrix's partial sums (added in chunk
// order by every thread's CTA, so that all of them use the same bits).
__device__ __forceinline__ void norm_scales(const float* part, int chunks, float& pre, float& post) {
    float s0 = 0.f, s1 = 0.f, s2 = 0.f;
    for (int i = 0; i < chunks; ++i) {
        s0 += part[3 * i];
        s1 += part[3 * i + 1];
        s2 += part[3 * i + 2];
    }
    float s = s0;
    pre = 1.f;
    if (isinf(s0)) {
        s = s1;
        pre = NS_DOWN;
    } else if (s0 < NS_TINY) {
        s = s2;
        pre = NS_UP;
    }
    post = s == 0.f ? 0.f : NS_S / sqrtf(s);   // a zero matrix stays zero; NaN stays NaN
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(NS_PRO_THREADS) muon_scale_kernel(const __grid_constant__ ProArgs p) {
    pdl_wait();
    __shared__ float sc[2];
    const int e = blockIdx.y, gpr = p.ld / 8;
    if (threadIdx.x == 0) norm_scales(p.part + (int64_t)e * p.chunks * 3, p.chunks, sc[0], sc[1]);
    __syncthreads();
    const float pre = sc[0], post = sc[1];
    const int g0 = blockIdx.x * NS_PRO_GROUPS, g1 = min(g0 + NS_PRO_GROUPS, p.groups);
    const T* U = static_cast<const T*>(p.U) + e * p.st_u;
    const float* M = p.M ? p.M + e * p.st_u : nullptr;
    __half* xh = p.xh + (int64_t)e * p.r * p.ld;
    __half* xl = p.xl + (int64_t)e * p.r * p.ld;
    for (int g = g0 + (int)threadIdx.x; g < g1; g += NS_PRO_THREADS) {
        const int row = g / gpr, col = (g - row * gpr) * 8, n = p.c - col;
        const int64_t at = row * p.ld_u + col;
        float v[8];
        if (M && !p.nesterov) {
            load8<float, VEC>(M + at, n, v);
        } else {
            load8<T, VEC>(U + at, n, v);
            if (M) {
                float m[8];
                load8<float, VEC>(M + at, n, m);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf(p.mu, m[i], v[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] * pre) * post;
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(xh + (int64_t)g * 8) = hi;
        *reinterpret_cast<uint4*>(xl + (int64_t)g * 8) = lo;
    }
}

// ------------------------------------------------------------------ products

constexpr int NS_BM = 128;            // output rows per tile: TMEM lanes
constexpr int NS_MAXBN = 256;         // output columns per tile at most (one tcgen05.mma)
constexpr int NS_BK = 64;             // K per stage: one 128-byte swizzle row of fp16
constexpr int NS_STAGES = 4;
constexpr int NS_BOX = 64 * NS_BK * 2;                  // bytes of one 64 x 64 TMA box
constexpr int NS_STAGE_BYTES = (NS_BM + NS_MAXBN) / 64 * NS_BOX;
constexpr int NS_EPI_WARPS = 8;       // two per TMEM lane quadrant, alternate 32-column chunks
constexpr int NS_WARP_LOAD = NS_EPI_WARPS;
constexpr int NS_WARP_MMA = NS_EPI_WARPS + 1;
constexpr int NS_THREADS = (NS_EPI_WARPS + 2) * 32;
constexpr int NS_SMEM = NS_STAGES * NS_STAGE_BYTES + 1024 + 256;
static_assert(NS_SMEM <= 232448, "shared memory of one CTA");

enum NsKind : int { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2 };

struct NsArgs {
    CUtensorMap tmX[2], tmA, tmB;   // 3-D maps {inner, rows, N}, boxes 64 x 64
    __half* xh[2];                  // X hi, ping-pong [N][r][ldx]
    __half* xl;                     // X lo [N][r][ldx]; each element is rewritten by the thread that reads it
    __half* A;                      // [N][m][ldm]
    __half* B;
    int N, r, c, m, ldx, ldm, tall;
    int bn_s, nt_s, mt_s, sym_tiles;   // m x m outputs: tile width, tiles across, down, computed
    int bn_x, nt_x, mt_x;              // r x c outputs
    int kind, src;                     // this launch's product; X buffer it reads
    float ca, cb, cc;                  // the step's coefficients
    int last;                          // NS_APPLY of the last step: write the outputs
    // outputs of the last step
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

struct NsTile {
    int e, m0, n0, num_kb, bn;
};

// First needed tile of row tile i of a symmetric output: tiles left of it lie strictly below
// the diagonal and are written as mirror images.
__device__ __forceinline__ int sym_first(const NsArgs& p, int i) { return i * NS_BM / p.bn_s; }

__device__ __forceinline__ NsTile ns_tile(const NsArgs& p, int w) {
    NsTile t;
    if (p.kind == NS_APPLY) {
        const int per = p.mt_x * p.nt_x;
        t.e = w / per;
        const int q = w - t.e * per;
        t.m0 = q / p.nt_x * NS_BM;
        t.n0 = q % p.nt_x * p.bn_x;
        t.bn = p.bn_x;
        t.num_kb = (p.m + NS_BK - 1) / NS_BK;
    } else {
        t.e = w / p.sym_tiles;
        int q = w - t.e * p.sym_tiles, i = 0;
        for (; i < p.mt_s - 1; ++i) {
            const int n = p.nt_s - sym_first(p, i);
            if (q < n) break;
            q -= n;
        }
        t.m0 = i * NS_BM;
        t.n0 = (sym_first(p, i) + q) * p.bn_s;
        t.bn = p.bn_s;
        const int k = p.kind == NS_GRAM ? (p.tall ? p.r : p.c) : p.m;
        t.num_kb = (k + NS_BK - 1) / NS_BK;
    }
    return t;
}

__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool a_mn_major, bool b_mn_major) {
    return (1u << 4) | (static_cast<uint32_t>(a_mn_major) << 15) | (static_cast<uint32_t>(b_mn_major) << 16) |
           ((static_cast<uint32_t>(N) >> 3) << 17) | ((static_cast<uint32_t>(M) >> 4) << 24);
}

// Operand layouts of a product: an operand whose K runs along the rows of its array is read
// MN-major, one whose K runs along the columns K-major; no array is ever transposed.
//   r <= c:  Gram  X X^T both K-major;   apply B X: B K-major, X MN-major
//   r >  c:  Gram  X^T X both MN-major;  apply X B: both K-major (B is symmetric)
struct NsOperands {
    const CUtensorMap *a, *b;
    bool a_mn, b_mn;
};
__device__ __forceinline__ NsOperands ns_operands(const NsArgs& p) {
    NsOperands o;
    if (p.kind == NS_GRAM) {
        o.a = o.b = &p.tmX[p.src];
        o.a_mn = o.b_mn = p.tall;
    } else if (p.kind == NS_POLY) {
        o.a = o.b = &p.tmA;
        o.a_mn = o.b_mn = false;
    } else {
        o.a = p.tall ? &p.tmX[p.src] : &p.tmB;
        o.b = p.tall ? &p.tmB : &p.tmX[p.src];
        o.a_mn = false;
        o.b_mn = !p.tall;
    }
    return o;
}

struct NsSmem {
    uint32_t ring, full, empty, tfull, tempty, drain;
};

__device__ __forceinline__ void ns_abort(volatile int* flag, DevStatus* st, int site, int a) {
    *flag = 1;
    report(st, MOEVIE_ERR_TIMEOUT, site, (int)blockIdx.x, a);
}

__device__ void ns_producer(const NsArgs& p, const NsSmem& sm, int n_work, volatile int* abort_flag) {
    const NsOperands o = ns_operands(p);
    tma_prefetch_desc(o.a);
    tma_prefetch_desc(o.b);
    int s = 0;
    uint32_t ph = 0;
    for (int w = blockIdx.x; w < n_work; w += gridDim.x) {
        const NsTile t = ns_tile(p, w);
        const int nbox = (t.bn + 63) / 64;
        const uint32_t bytes = (uint32_t)(2 + nbox) * NS_BOX;
        for (int kb = 0; kb < t.num_kb; ++kb) {
            if (!mbar_wait(sm.empty + 8 * s, ph ^ 1u, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_EMPTY, w);
                return;
            }
            const uint32_t bar = sm.full + 8 * s, dst = sm.ring + s * NS_STAGE_BYTES;
            mbar_arrive_expect_tx(bar, bytes);
            const int kk = kb * NS_BK;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int mm = t.m0 + 64 * j;
                tma_load_3d(dst + j * NS_BOX, o.a, bar, o.a_mn ? mm : kk, o.a_mn ? kk : mm, t.e);
            }
            for (int j = 0; j < nbox; ++j) {
                const int nn = t.n0 + 64 * j;
                tma_load_3d(dst + (2 + j) * NS_BOX, o.b, bar, o.b_mn ? nn : kk, o.b_mn ? kk : nn, t.e);
            }
            if (++s == NS_STAGES) {
                s = 0;
                ph ^= 1u;
            }
        }
    }
}

__device__ __forceinline__ void ns_mma(const NsArgs& p, const NsSmem& sm, uint32_t tmem, int n_work,
                                       volatile int* abort_flag) {
    const NsOperands o = ns_operands(p);
    const uint64_t ad0 = smem_desc_sw128(sm.ring, o.a_mn ? NS_BOX : 16, 1024);
    const uint64_t bd0 = smem_desc_sw128(sm.ring + 2 * NS_BOX, o.b_mn ? NS_BOX : 16, 1024);
    const uint32_t as = (o.a_mn ? 2048 : 32) >> 4, bs = (o.b_mn ? 2048 : 32) >> 4;
    int s = 0, it = 0;
    uint32_t ph = 0;
    bool issued = false;
    for (int w = blockIdx.x; w < n_work; w += gridDim.x, ++it) {
        const NsTile t = ns_tile(p, w);
        const uint32_t idesc = idesc_f16_f32(NS_BM, t.bn, o.a_mn, o.b_mn);
        const int acc = it & 1;
        if (!mbar_wait(sm.tempty + 8 * acc, ((it >> 1) & 1) ^ 1u, p.limit_ns, abort_flag)) {
            ns_abort(abort_flag, p.status, SITE_NS_WAIT_TEMPTY, w);
            break;
        }
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)acc * NS_MAXBN;
        bool ok = true;
        for (int kb = 0; kb < t.num_kb; ++kb) {
            if (!mbar_wait(sm.full + 8 * s, ph, p.limit_ns, abort_flag)) {
                ns_abort(abort_flag, p.status, SITE_NS_WAIT_FULL, w);
                ok = false;
                break;
            }
            const uint64_t ad = ad0 + (uint64_t)((s * NS_STAGE_BYTES) >> 4);
            const uint64_t bd = bd0 + (uint64_t)((s * NS_STAGE_BYTES) >> 4);
#pragma unroll
            for (int q = 0; q < NS_BK / 16; ++q)
                tc_mma_bf16(d, ad + q * as, bd + q * bs, idesc, (kb | q) != 0 ? 1u : 0u);
            issued = true;
            tc_commit(sm.empty + 8 * s);
            if (++s == NS_STAGES) {
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
            report(p.status, MOEVIE_ERR_TIMEOUT, SITE_NS_DRAIN, (int)blockIdx.x, 0);
    }
}

// Eight working-format values of a row from L2 (written by other SMs).
__device__ __forceinline__ void load_half8(const __half* p, float (&v)[8]) {
    const uint4 u = __ldcg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 f = unpack_half2(w[q]);
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
    }
}

// One group of eight columns of an output row.
__device__ __forceinline__ void ns_store_sym(const NsArgs& p, const NsTile& t, int row, int col,
                                             const float (&d)[8]) {
    const int64_t base = (int64_t)t.e * p.m * p.ldm;
    float v[8];
    const bool gram = p.kind == NS_GRAM;
    if (gram) {
        // with c = 0 the step has no A^2: B = b A comes straight from the Gram product
        const float sc = p.cc == 0.f ? p.cb * NS_INV_S : NS_INV_S;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = d[i] * sc;
    } else {
        load_half8(p.A + base + (int64_t)row * p.ldm + col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(p.cc * NS_INV_S, d[i], p.cb * v[i]);
    }
    __half* out = (gram && p.cc != 0.f ? p.A : p.B) + base;
    uint4 u;
    u.x = pack_half2(v[0], v[1]);
    u.y = pack_half2(v[2], v[3]);
    u.z = pack_half2(v[4], v[5]);
    u.w = pack_half2(v[6], v[7]);
    *reinterpret_cast<uint4*>(out + (int64_t)row * p.ldm + col) = u;
    // the mirror image, where its own tile is not computed
    const int col_end = (row / p.bn_s + 1) * p.bn_s;   // end of the tile column that holds `row`
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int j = col + i;
        if (j < p.m && col_end <= j / NS_BM * NS_BM) out[(int64_t)j * p.ldm + row] = __float2half_rn(v[i]);
    }
}

__device__ __forceinline__ void ns_store_x(const NsArgs& p, const NsTile& t, int row, int col,
                                           const float (&d)[8]) {
    const int64_t at = ((int64_t)t.e * p.r + row) * p.ldx + col;
    float v[8], l[8];
    load_half8(p.xh[p.src] + at, v);
    load_half8(p.xl + at, l);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(NS_INV_S, d[i], p.ca * fmaf(NS_INV_LO, l[i], v[i]));
    if (!p.last) {
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(p.xh[p.src ^ 1] + at) = hi;
        *reinterpret_cast<uint4*>(p.xl + at) = lo;
        return;
    }
    const int n = p.c - col;   // columns of this group that exist
    if (p.O) {
        __nv_bfloat16* o = p.O + t.e * p.st_o + row * p.ld_o + col;
        if (p.vec_o && n >= 8) {
            uint4 u;
            u.x = pack_bf16x2(v[0] * NS_INV_S, v[1] * NS_INV_S);
            u.y = pack_bf16x2(v[2] * NS_INV_S, v[3] * NS_INV_S);
            u.z = pack_bf16x2(v[4] * NS_INV_S, v[5] * NS_INV_S);
            u.w = pack_bf16x2(v[6] * NS_INV_S, v[7] * NS_INV_S);
            *reinterpret_cast<uint4*>(o) = u;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) o[i] = __float2bfloat16_rn(v[i] * NS_INV_S);
        }
    } else {
        const int64_t wat = t.e * p.st_w + row * p.ld_w + col;
        float w[8];
        load8<float, true>(p.W + wat, n, w);
        const float rate = p.rate * NS_INV_S;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = fmaf(-rate, v[i], p.decay * w[i]);
        store8<true>(p.W + wat, n, w);
        if (p.Wb) {
            if (n >= 8) {
                uint4 u;
                u.x = pack_bf16x2(w[0], w[1]);
                u.y = pack_bf16x2(w[2], w[3]);
                u.z = pack_bf16x2(w[4], w[5]);
                u.w = pack_bf16x2(w[6], w[7]);
                *reinterpret_cast<uint4*>(p.Wb + wat) = u;
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) p.Wb[wat + i] = __float2bfloat16_rn(w[i]);
            }
        }
    }
}

__device__ void ns_epilogue(const NsArgs& p, const NsSmem& sm, uint32_t tmem, int n_work,
                            volatile int* abort_flag) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quad = warp & 3, half = warp >> 2;
    int it = 0;
    for (int w = blockIdx.x; w < n_work; w += gridDim.x, ++it) {
        const NsTile t = ns_tile(p, w);
        const int acc = it & 1, row = t.m0 + quad * 32 + lane;
        const int rows = p.kind == NS_APPLY ? p.r : p.m, cols = p.kind == NS_APPLY ? p.c : p.m;
        const int nchunk = (t.bn + 31) / 32;
        if (!mbar_wait(sm.tfull + 8 * acc, (uint32_t)(it >> 1) & 1u, p.limit_ns, abort_flag)) {
            ns_abort(abort_flag, p.status, SITE_NS_WAIT_TFULL, w);
            return;
        }
        tc_fence_after();
        const uint32_t tbase = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)acc * NS_MAXBN;
        for (int ch = half; ch < nchunk; ch += 2) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(tbase + ch * 32, v);
            tmem_wait_ld();
            if (row >= rows) continue;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int off = ch * 32 + g * 8, col = t.n0 + off;
                if (off >= t.bn || col >= cols) break;
                float d[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = __uint_as_float(v[8 * g + i]);
                if (p.kind == NS_APPLY) ns_store_x(p, t, row, col, d);
                else ns_store_sym(p, t, row, col, d);
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.tempty + 8 * acc);
    }
}

__global__ void __launch_bounds__(NS_THREADS, 1) ns_gemm_kernel(const __grid_constant__ NsArgs p) {
    extern __shared__ uint8_t ns_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ns_smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + NS_STAGES * NS_STAGE_BYTES);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * NS_STAGES + 5);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    NsSmem sm;
    sm.ring = smem_u32(smem);
    sm.full = smem_u32(bars);
    sm.empty = sm.full + 8 * NS_STAGES;
    sm.tfull = sm.empty + 8 * NS_STAGES;
    sm.tempty = sm.tfull + 16;
    sm.drain = sm.tempty + 16;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < NS_STAGES; ++s) {
            mbar_init(sm.full + 8 * s, 1);
            mbar_init(sm.empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(sm.tfull + 8 * a, 1);
            mbar_init(sm.tempty + 8 * a, NS_EPI_WARPS);
        }
        mbar_init(sm.drain, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == NS_WARP_MMA) {
        tmem_alloc(smem_u32(tmem_slot), 2 * NS_MAXBN);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    const uint32_t tmem = *tmem_slot;
    const int n_work = p.N * (p.kind == NS_APPLY ? p.mt_x * p.nt_x : p.sym_tiles);
    if (warp < NS_EPI_WARPS) {
        ns_epilogue(p, sm, tmem, n_work, abort_flag);
    } else if (warp == NS_WARP_LOAD) {
        if ((threadIdx.x & 31) == 0) ns_producer(p, sm, n_work, abort_flag);
    } else {
        if ((threadIdx.x & 31) == 0) ns_mma(p, sm, tmem, n_work, abort_flag);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == NS_WARP_MMA) {
        tc_fence_after();
        tmem_dealloc(tmem, 2 * NS_MAXBN);
    }
}

// ------------------------------------------------------------- thin matrices

// m <= NS_THIN: one CTA per matrix, fp32 throughout.  All factors of the step polynomials are
// polynomials of A = X0 X0^T and commute, so the iteration runs on m x m matrices in shared
// memory (P = a I + b A + c A^2, Q <- P Q, A <- P A P) and X is read twice: for A and for
// Q X0.  Thin matrices are kept off the tensor cores for accuracy as much as for time: with few
// singular values the fp16 roundings do not average out over the entries (a 1 x n matrix is one
// number per step, and its result was 5e-3 off), and their tiles would be mostly empty.
constexpr int NS_THIN = 32;
constexpr int NS_THIN_THREADS = 256;
constexpr int NS_THIN_K = 64;

__device__ __forceinline__ void ns_out1(const NsArgs& p, int e, int row, int col, float v) {
    if (p.O) {
        p.O[e * p.st_o + row * p.ld_o + col] = __float2bfloat16_rn(v);
    } else {
        const int64_t at = e * p.st_w + row * p.ld_w + col;
        const float w = fmaf(-p.rate, v, p.decay * p.W[at]);
        p.W[at] = w;
        if (p.Wb) p.Wb[at] = __float2bfloat16_rn(w);
    }
}

struct NsSteps {
    float coef[3 * NS_MAX_STEPS];
    int steps;
};

__global__ void __launch_bounds__(NS_THIN_THREADS) ns_thin_kernel(const __grid_constant__ NsArgs p,
                                                                  const __grid_constant__ NsSteps st) {
    pdl_wait();
    __shared__ float A[NS_THIN][NS_THIN + 1], P[NS_THIN][NS_THIN + 1], Q[NS_THIN][NS_THIN + 1],
        T[NS_THIN][NS_THIN + 1], xs[NS_THIN][NS_THIN_K + 1];
    const int e = blockIdx.x, m = p.m, n = p.tall ? p.r : p.c, tid = threadIdx.x;
    constexpr int PER = NS_THIN * NS_THIN / NS_THIN_THREADS;
    const __half* xh = p.xh[0] + (int64_t)e * p.r * p.ldx;
    const __half* xl = p.xl + (int64_t)e * p.r * p.ldx;
    auto stage = [&](int k0) {   // xs[i][kk] = X0 (i, k0 + kk) of the m x n orientation
        for (int q = tid; q < m * NS_THIN_K; q += NS_THIN_THREADS) {
            const int i = p.tall ? q % m : q / NS_THIN_K, kk = p.tall ? q / m : q % NS_THIN_K;
            float v = 0.f;
            if (k0 + kk < n) {
                const int64_t at = p.tall ? (int64_t)(k0 + kk) * p.ldx + i : (int64_t)i * p.ldx + k0 + kk;
                v = fmaf(NS_INV_LO, __half2float(xl[at]), __half2float(xh[at])) * NS_INV_S;
            }
            xs[i][kk] = v;
        }
    };
    // out = L R, every operand m x m in shared memory, `out` none of them
    auto product = [&](float (*out)[NS_THIN + 1], const float (*L)[NS_THIN + 1], const float (*R)[NS_THIN + 1]) {
        for (int q = tid; q < m * m; q += NS_THIN_THREADS) {
            const int i = q / m, j = q - i * m;
            float s = 0.f;
            for (int k = 0; k < m; ++k) s = fmaf(L[i][k], R[k][j], s);
            out[i][j] = s;
        }
        __syncthreads();
    };
    float acc[PER] = {};
    for (int k0 = 0; k0 < n; k0 += NS_THIN_K) {
        stage(k0);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int q = tid + u * NS_THIN_THREADS, i = q / m, j = q - i * m;
            if (q < m * m) {
                float s = acc[u];
                for (int kk = 0; kk < NS_THIN_K; ++kk) s = fmaf(xs[i][kk], xs[j][kk], s);
                acc[u] = s;
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int q = tid + u * NS_THIN_THREADS;
        if (q < m * m) A[q / m][q % m] = acc[u];
    }
    __syncthreads();
    for (int it = 0; it < st.steps; ++it) {
        const float ca = st.coef[3 * it], cb = st.coef[3 * it + 1], cc = st.coef[3 * it + 2];
        product(T, A, A);
        for (int q = tid; q < m * m; q += NS_THIN_THREADS) {
            const int i = q / m, j = q - i * m;
            P[i][j] = fmaf(cc, T[i][j], cb * A[i][j]) + (i == j ? ca : 0.f);
            if (it == 0) Q[i][j] = P[i][j];
        }
        __syncthreads();
        if (it > 0) {
            product(T, P, Q);
            for (int q = tid; q < m * m; q += NS_THIN_THREADS) Q[q / m][q % m] = T[q / m][q % m];
            __syncthreads();
        }
        if (it + 1 < st.steps) {
            product(T, P, A);
            product(A, T, P);
        }
    }
    for (int k0 = 0; k0 < n; k0 += NS_THIN_K) {
        stage(k0);
        __syncthreads();
        for (int q = tid; q < m * NS_THIN_K; q += NS_THIN_THREADS) {
            const int i = p.tall ? q % m : q / NS_THIN_K, kk = p.tall ? q / m : q % NS_THIN_K;
            if (k0 + kk < n) {
                float s = 0.f;
                for (int j = 0; j < m; ++j) s = fmaf(Q[i][j], xs[j][kk], s);
                ns_out1(p, e, p.tall ? k0 + kk : i, p.tall ? i : k0 + kk, s);
            }
        }
        __syncthreads();
    }
}

// Width of the n-tiles of an output of n columns: as few tiles as 256-wide MMAs allow, of
// equal width, a multiple of 16.
void ns_tiles(int n, int* bn, int* nt) {
    const int t = (n + NS_MAXBN - 1) / NS_MAXBN;
    *bn = ((n + t - 1) / t + 15) / 16 * 16;
    *nt = (n + *bn - 1) / *bn;
}

inline int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

struct NsLayout {
    size_t part, xh0, xh1, xl, A, B, total;
    int chunks, groups;
};
NsLayout ns_layout(int64_t N, int64_t r, int64_t c) {
    NsLayout L;
    const int64_t m = r < c ? r : c, ldx = up8(c), ldm = up8(m);
    L.groups = (int)(r * ldx / 8);
    L.chunks = (L.groups + NS_PRO_GROUPS - 1) / NS_PRO_GROUPS;
    size_t o = up256(sizeof(DevStatus));
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    L.part = take((size_t)N * L.chunks * 3 * sizeof(float));
    L.xh0 = take((size_t)(N * r * ldx) * 2);
    L.xh1 = take((size_t)(N * r * ldx) * 2);
    L.xl = take((size_t)(N * r * ldx) * 2);
    L.A = take((size_t)(N * m * ldm) * 2);
    L.B = take((size_t)(N * m * ldm) * 2);
    L.total = o;
    return L;
}

template <typename T, bool VEC>
cudaError_t launch_prologue(const ProArgs& p, int N, cudaStream_t s) {
    const dim3 grid((unsigned)p.chunks, (unsigned)N);
    cudaError_t e = launch_pdl(muon_moment_kernel<T, VEC>, grid, dim3(NS_PRO_THREADS), 0, s, p);
    if (e != cudaSuccess) return e;
    return launch_pdl(muon_scale_kernel<T, VEC>, grid, dim3(NS_PRO_THREADS), 0, s, p);
}

}  // namespace

size_t ns_workspace_bytes(int64_t N, int64_t r, int64_t c) { return ns_layout(N, r, c).total; }

cudaError_t launch_newton_schulz(const NsCall& q, uint8_t* ws, int sms, uint64_t limit_ns, cudaStream_t s) {
    const NsLayout L = ns_layout(q.N, q.r, q.c);
    ProArgs pa = {};
    pa.U = q.U;
    pa.ld_u = q.ld_u;
    pa.st_u = q.st_u;
    pa.M = q.M;
    pa.mu = q.momentum;
    pa.nesterov = q.nesterov;
    pa.r = q.r;
    pa.c = q.c;
    pa.ld = (int)up8(q.c);
    pa.groups = L.groups;
    pa.chunks = L.chunks;
    pa.part = reinterpret_cast<float*>(ws + L.part);
    pa.xh = reinterpret_cast<__half*>(ws + L.xh0);
    pa.xl = reinterpret_cast<__half*>(ws + L.xl);
    const bool vec = q.ld_u % 8 == 0 && q.st_u % 8 == 0 && (reinterpret_cast<uintptr_t>(q.U) & 15u) == 0;
    cudaError_t e;
    if (q.u_bf16) e = vec ? launch_prologue<__nv_bfloat16, true>(pa, q.N, s) : launch_prologue<__nv_bfloat16, false>(pa, q.N, s);
    else e = vec ? launch_prologue<float, true>(pa, q.N, s) : launch_prologue<float, false>(pa, q.N, s);
    if (e != cudaSuccess) return e;
    count_launches(2);

    NsArgs a = {};
    a.N = q.N;
    a.r = q.r;
    a.c = q.c;
    a.tall = q.r > q.c;
    a.m = a.tall ? q.c : q.r;
    a.ldx = (int)up8(q.c);
    a.ldm = (int)up8(a.m);
    a.xh[0] = reinterpret_cast<__half*>(ws + L.xh0);
    a.xh[1] = reinterpret_cast<__half*>(ws + L.xh1);
    a.xl = reinterpret_cast<__half*>(ws + L.xl);
    a.A = reinterpret_cast<__half*>(ws + L.A);
    a.B = reinterpret_cast<__half*>(ws + L.B);
    for (int i = 0; i < 2; ++i)
        if (!make_weight_tmap_strided(&a.tmX[i], a.xh[i], a.c, a.r, a.N, a.ldx, (int64_t)a.r * a.ldx))
            return cudaErrorInvalidValue;
    if (!make_weight_tmap_strided(&a.tmA, a.A, a.m, a.m, a.N, a.ldm, (int64_t)a.m * a.ldm) ||
        !make_weight_tmap_strided(&a.tmB, a.B, a.m, a.m, a.N, a.ldm, (int64_t)a.m * a.ldm))
        return cudaErrorInvalidValue;
    ns_tiles(a.m, &a.bn_s, &a.nt_s);
    ns_tiles(a.c, &a.bn_x, &a.nt_x);
    a.mt_s = (a.m + NS_BM - 1) / NS_BM;
    a.mt_x = (a.r + NS_BM - 1) / NS_BM;
    a.sym_tiles = 0;
    for (int i = 0; i < a.mt_s; ++i) a.sym_tiles += a.nt_s - i * NS_BM / a.bn_s;
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
    if (a.m <= NS_THIN) {
        NsSteps st = {};
        st.steps = q.steps;
        for (int i = 0; i < 3 * q.steps; ++i) st.coef[i] = q.coef[i];
        e = launch_pdl(ns_thin_kernel, dim3((unsigned)a.N), dim3(NS_THIN_THREADS), 0, s, a, st);
        count_launches(1);
        return e != cudaSuccess ? e : cudaGetLastError();
    }
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_set[dev]) {
        e = cudaFuncSetAttribute(ns_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    for (int it = 0; it < q.steps; ++it) {
        a.ca = q.coef[3 * it];
        a.cb = q.coef[3 * it + 1];
        a.cc = q.coef[3 * it + 2];
        a.src = it & 1;
        a.last = it == q.steps - 1;
        for (int kind = NS_GRAM; kind <= NS_APPLY; ++kind) {
            if (kind == NS_POLY && a.cc == 0.f) continue;
            a.kind = kind;
            const int64_t work = (int64_t)a.N * (kind == NS_APPLY ? a.mt_x * a.nt_x : a.sym_tiles);
            e = launch_pdl(ns_gemm_kernel, dim3((unsigned)(work < sms ? work : sms)), dim3(NS_THREADS), NS_SMEM,
                           s, a);
            count_launches(1);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaGetLastError();
}

}  // namespace mv
