// few.cu -- the whole MoE FFN layer for a few tokens (T <= 64), sm_103a.
//
// The layer of Eqs. 1 and 4-7 where every expert sees a handful of tokens at most: the time is
// that of reading the router and the selected experts' weights once, and of launching.
#include <math.h>

#include "internal.h"

namespace mv {

namespace {

__device__ __forceinline__ float act1(float u) { return 0.5f * u * (1.0f + erff(u * 0.70710678118654752f)); }
__device__ __forceinline__ float silu1(float u) { return u / (1.0f + expf(-u)); }

// One CTA per token: logits and keys in 64 bits, k rounds of arg-max (ties and NaN: the lowest
// id first, NaN after every number), ids in ascending order, gates from the 64-bit sigmoids.
__global__ void __launch_bounds__(256) few_route_kernel(const __grid_constant__ FewArgs p) {
    pdl_wait();
    __shared__ double sig[1024], key[1024];
    __shared__ uint8_t sel[1024];
    const int t = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const __nv_bfloat16* x = p.x + (int64_t)t * p.d;
    for (int e = warp; e < p.E; e += 8) {
        double s = 0.0;
        for (int i = lane; i < p.d; i += 32)
            s = fma((double)__bfloat162float(x[i]), (double)p.W_r[(int64_t)i * p.E + e], s);
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) {
            sig[e] = 1.0 / (1.0 + exp(-s));
            key[e] = sig[e] + (double)p.b[e];
            sel[e] = 0;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
        for (int j = 0; j < p.k; ++j) {
            int best = -1;
            for (int e = 0; e < p.E; ++e) {
                if (sel[e]) continue;
                if (best < 0 || key[e] > key[best] || (isnan(key[best]) && !isnan(key[e]))) best = e;
            }
            sel[best] = 1;
        }
        for (int e = 0; e < p.E; ++e)
            if (sel[e]) sum += sig[e];
        for (int e = 0, j = 0; e < p.E; ++e) {
            if (!sel[e]) continue;
            p.idx[t * p.k + j] = e;
            p.gate[t * p.k + j] = (float)(sig[e] / sum);
            ++j;
        }
    }
}

// CTA (row, column tile): the hidden activations of one routed slot, or past them of one token
// of the shared expert.
__global__ void __launch_bounds__(128) few_up_kernel(const __grid_constant__ FewArgs p) {
    pdl_wait();
    const int s = blockIdx.x, n = blockIdx.y * 128 + threadIdx.x;
    const bool routed = s < p.T * p.k;
    const int t = routed ? s / p.k : s - p.T * p.k;
    const int h = routed ? p.h : p.hs;
    const int64_t ld = routed ? p.hp : p.hsp;
    if (n >= h) return;
    const int64_t e = routed ? p.idx[s] : 0;
    const __nv_bfloat16* w1 = (routed ? p.W1 : p.Ws1) + e * p.d * ld + n;
    const __nv_bfloat16* w3 = routed ? p.W3 : p.Ws3;
    const __nv_bfloat16* x = p.x + (int64_t)t * p.d;
    float u = 0.f, v = 0.f;
    for (int i = 0; i < p.d; ++i) u = fmaf(__bfloat162float(x[i]), __bfloat162float(w1[i * ld]), u);
    if (w3) {
        w3 += e * p.d * ld + n;
        for (int i = 0; i < p.d; ++i) v = fmaf(__bfloat162float(x[i]), __bfloat162float(w3[i * ld]), v);
    }
    (routed ? p.hid + (int64_t)s * p.h : p.hid_s + (int64_t)t * p.hs)[n] = w3 ? silu1(u) * v : act1(u);
}

__global__ void __launch_bounds__(128) few_down_kernel(const __grid_constant__ FewArgs p) {
    pdl_wait();
    const int t = blockIdx.x, n = blockIdx.y * 128 + threadIdx.x;
    if (n >= p.d) return;
    float y = 0.f;
    for (int j = 0; j < p.k; ++j) {
        const int s = t * p.k + j;
        const __nv_bfloat16* w = p.W2 + (int64_t)p.idx[s] * p.h * p.d + n;
        const float* a = p.hid + (int64_t)s * p.h;
        float o = 0.f;
        for (int i = 0; i < p.h; ++i) o = fmaf(a[i], __bfloat162float(w[(int64_t)i * p.d]), o);
        y = fmaf(p.gate[s], o, y);
    }
    if (p.hs > 0) {
        const float* a = p.hid_s + (int64_t)t * p.hs;
        float o = 0.f;
        for (int i = 0; i < p.hs; ++i) o = fmaf(a[i], __bfloat162float(p.Ws2[(int64_t)i * p.d + n]), o);
        y = fmaf(p.lambda, o, y);
    }
    p.y[(int64_t)t * p.d + n] = __float2bfloat16_rn(y);
}

inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

struct FewLayout {
    size_t idx, gate, hid, hid_s, total;
};
FewLayout few_layout(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t hs) {
    (void)d;
    (void)E;
    FewLayout L;
    size_t o = up256(sizeof(DevStatus));
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    L.idx = take(4 * T * k);
    L.gate = take(4 * T * k);
    L.hid = take(4 * T * k * h);
    L.hid_s = take(4 * T * hs);
    L.total = o;
    return L;
}

}  // namespace

size_t few_workspace_bytes(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t hs) {
    return few_layout(T, d, E, k, h, hs).total;
}

cudaError_t launch_few(FewArgs a, uint8_t* ws, int sms, uint64_t limit_ns, cudaStream_t s) {
    (void)sms;
    (void)limit_ns;
    const FewLayout L = few_layout(a.T, a.d, a.E, a.k, a.h, a.hs);
    if (!a.idx) a.idx = reinterpret_cast<int32_t*>(ws + L.idx);
    if (!a.gate) a.gate = reinterpret_cast<float*>(ws + L.gate);
    a.hid = reinterpret_cast<float*>(ws + L.hid);
    a.hid_s = reinterpret_cast<float*>(ws + L.hid_s);
    a.status = reinterpret_cast<DevStatus*>(ws);
    cudaError_t e = launch_pdl(few_route_kernel, dim3(a.T), dim3(256), 0, s, a);
    if (e != cudaSuccess) return e;
    const int rows = a.T * a.k + (a.hs > 0 ? a.T : 0), hmax = a.h > a.hs ? a.h : a.hs;
    e = launch_pdl(few_up_kernel, dim3(rows, (hmax + 127) / 128), dim3(128), 0, s, a);
    if (e != cudaSuccess) return e;
    e = launch_pdl(few_down_kernel, dim3(a.T, (a.d + 127) / 128), dim3(128), 0, s, a);
    count_launches(3);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mv
