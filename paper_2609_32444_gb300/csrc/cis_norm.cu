// cis_norm.cu -- the root-mean-square norm before the LM head: with the residual's addition and an
// output in 8 bits (cis_rmsnorm_fwd), and its gradients (cis_rmsnorm_bwd).
//
// Per row, with h = x + residual, in fp32 whatever the types:
//   y_j = w_j h_j r,   r = (mean_j h_j^2 + eps)^-1/2;
//   scale = max(max_j |y_j|, 2^-100) / 448,   q_j = e4m3(y_j / scale).
// max_j |y_j| = r max_j |w_j h_j|, so that one pass over the row's registers gives the sum of the
// squares and the scale.  The gradients, with g_j = dy_j w_j and c = r^2 mean_j g_j h_j:
//   dx_j = dh_j + r (g_j - h_j c),   dweight_j = sum_t dy_tj h_tj r_t.
//
// A row lies in the registers of one warp or CTA, 16 elements a thread, in 16-byte vectors where
// every row starts on 16 bytes and else an element at a time; each tensor is read once.  In the
// backward kernel a thread has the same columns in every row that it takes, so that dweight's sum
// stays in its registers (16 of them); the CTAs' sums meet in the workspace, in a fixed order.
//
// Bound: HBM for many rows; for few, the latency of a load, a reduction and a store.
#include <cuda_fp8.h>
#include <math.h>

#include "cis_kernels.h"
#include "cis_nvtx.h"

namespace cis {
namespace {

constexpr int64_t kMaxHidden = 16384;
constexpr float kLeastMax = 0x1p-100f;  // the least maximum that a row's scale is made for
constexpr float kE4m3Max = 448.0f;

struct NormArgs {
    const void *x, *residual;  // forward; backward: h, dh
    const void *dy;
    const void *w;
    int64_t T, ld_x, ld_r, ld_dy;
    int H;
    int w_f32;
    float eps;
    const uint8_t *mask;
    void *h_out, *y_out;  // forward; backward: y_out is dx
    uint8_t *q_out;
    float *scale_out;
    float *dw;      // backward: dweight, or the CTAs' sums [gridDim.x, H]
};

// E elements as they lie in memory.
template <typename T, int E> struct Pack;
template <> struct Pack<__nv_bfloat16, 8> {
    uint4 q;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        q = __ldg(reinterpret_cast<const uint4 *>(p));
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(w[i]);
            f[2 * i + 1] = bf16_hi(w[i]);
        }
    }
};
template <> struct Pack<float, 4> {
    float4 q;
    __device__ __forceinline__ void load(const float *p)
    {
        q = __ldg(reinterpret_cast<const float4 *>(p));
    }
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
        f[0] = q.x;
        f[1] = q.y;
        f[2] = q.z;
        f[3] = q.w;
    }
};
template <typename T> struct Pack<T, 1> {
    T q;
    __device__ __forceinline__ void load(const T *p) { q = __ldg(p); }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(q); }
};

// E elements rounded to T.  Written once and read by another kernel, if at all.
__device__ __forceinline__ void put(__nv_bfloat16 *p, const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&v);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put(float *p, const float (&f)[4])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void put(__nv_bfloat16 *p, const float (&f)[1])
{
    *p = __float2bfloat16_rn(f[0]);
}
__device__ __forceinline__ void put(float *p, const float (&f)[1]) { *p = f[0]; }

__device__ __forceinline__ uint32_t e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ void put_e4m3(uint8_t *p, const float (&f)[8])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(e4m3x2(f[0], f[1]) | e4m3x2(f[2], f[3]) << 16,
                                               e4m3x2(f[4], f[5]) | e4m3x2(f[6], f[7]) << 16);
}
__device__ __forceinline__ void put_e4m3(uint8_t *p, const float (&f)[4])
{
    *reinterpret_cast<uint32_t *>(p) = e4m3x2(f[0], f[1]) | e4m3x2(f[2], f[3]) << 16;
}
__device__ __forceinline__ void put_e4m3(uint8_t *p, const float (&f)[1])
{
    *p = __nv_cvt_float_to_fp8(f[0], __NV_SATFINITE, __NV_E4M3);
}

// The weights of E columns, in either type.
template <int E> __device__ __forceinline__ void weights_of(const NormArgs &a, int j, float (&w)[E])
{
    if constexpr (E == 1) {
        w[0] = a.w_f32 ? __ldg(static_cast<const float *>(a.w) + j)
                       : to_f32(__ldg(static_cast<const __nv_bfloat16 *>(a.w) + j));
    } else if (a.w_f32) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(
                static_cast<const float *>(a.w) + j + i));
            w[i] = v.x;
            w[i + 1] = v.y;
            w[i + 2] = v.z;
            w[i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(
                static_cast<const __nv_bfloat16 *>(a.w) + j + i));
            w[i] = bf16_lo(v.x);
            w[i + 1] = bf16_hi(v.x);
            w[i + 2] = bf16_lo(v.y);
            w[i + 3] = bf16_hi(v.y);
        }
    }
}

// A row's two numbers, over the TPR threads that have it: s is added up, and m added or (kMax)
// the larger, a NaN if there is one.  Every thread gets them.  `slots` alternate from row to row,
// so that one barrier does.
template <int TPR, bool kMax>
__device__ __forceinline__ void row_reduce(float &s, float &m, float2 (*slots)[32], int &turn)
{
    auto join = [](float a, float b) { return kMax ? max_nan(a, b) : a + b; };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        m = join(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    if constexpr (TPR > 32) {
        const int lane = threadIdx.x & 31;
        constexpr int W = TPR / 32;
        if (lane == 0)
            slots[turn][threadIdx.x >> 5] = make_float2(s, m);
        __syncthreads();
        const float2 v = slots[turn][lane < W ? lane : 0];
        s = lane < W ? v.x : 0.0f;
        m = lane < W ? v.y : 0.0f;
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            m = join(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
        s = __shfl_sync(0xffffffffu, s, 0);
        m = __shfl_sync(0xffffffffu, m, 0);
        turn ^= 1;
    }
}

template <int TPR> constexpr int kCta = TPR < 128 ? 128 : TPR;

// The forward kernel: TPR threads a row, V vectors of E elements each.
template <typename T, int E, int TPR, int V>
__global__ void __launch_bounds__(kCta<TPR>) cis_rmsnorm_fwd_kernel(const NormArgs a)
{
    constexpr int R = kCta<TPR> / TPR;  // rows of a CTA at a time
    __shared__ float2 slots[2][32];
    const int at = TPR > 32 ? threadIdx.x : threadIdx.x & 31;
    int turn = 0;
    for (int64_t t = (int64_t)blockIdx.x * R + (TPR > 32 ? 0 : threadIdx.x >> 5); t < a.T;
         t += (int64_t)gridDim.x * R) {
        T *h_out = a.h_out ? static_cast<T *>(a.h_out) + t * a.H : nullptr;
        T *y_out = a.y_out ? static_cast<T *>(a.y_out) + t * a.H : nullptr;
        uint8_t *q_out = a.q_out ? a.q_out + t * a.H : nullptr;
        if (a.mask && !a.mask[t]) {  // not read; zeros
            float z[E] = {};
            for (int k = 0; k < V; ++k) {
                const int j = (at + k * TPR) * E;
                if (j < a.H) {
                    if (h_out) put(h_out + j, z);
                    if (y_out) put(y_out + j, z);
                    if (q_out) put_e4m3(q_out + j, z);
                }
            }
            if (a.scale_out && at == 0)
                a.scale_out[t] = 0.0f;
            continue;
        }
        const T *x = static_cast<const T *>(a.x) + t * a.ld_x;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + t * a.ld_r : nullptr;
        Pack<T, E> px[V], pr[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = (at + k * TPR) * E;
            if (j < a.H) {
                px[k].load(x + j);
                if (r)
                    pr[k].load(r + j);
            }
        }
        float h[V][E], w[V][E], s = 0.0f, m = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = (at + k * TPR) * E;
            if (j < a.H) {
                weights_of(a, j, w[k]);
                px[k].get(h[k]);
                if (r) {
                    float f[E];
                    pr[k].get(f);
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        h[k][i] += f[i];
                }
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    s = fmaf(h[k][i], h[k][i], s);
                    w[k][i] *= h[k][i];
                    m = max_nan(m, fabsf(w[k][i]));
                }
                if (h_out)
                    put(h_out + j, h[k]);
            }
        }
        row_reduce<TPR, true>(s, m, slots, turn);
        const float rstd = 1.0f / sqrtf(s / (float)a.H + a.eps);
        if (y_out) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int j = (at + k * TPR) * E;
                if (j < a.H) {
                    float y[E];
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        y[i] = w[k][i] * rstd;
                    put(y_out + j, y);
                }
            }
        }
        if (q_out) {
            const float most = m * rstd, top = most < kLeastMax ? kLeastMax : most;
            const float up = kE4m3Max / top;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int j = (at + k * TPR) * E;
                if (j < a.H) {
                    float y[E];
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        y[i] = w[k][i] * rstd * up;
                    put_e4m3(q_out + j, y);
                }
            }
            if (at == 0)
                a.scale_out[t] = top / kE4m3Max;
        }
    }
}

// The backward kernel.
template <typename T, int E, int TPR, int V>
__global__ void __launch_bounds__(kCta<TPR>) cis_rmsnorm_bwd_kernel(const NormArgs a)
{
    constexpr int R = kCta<TPR> / TPR;
    __shared__ float2 slots[2][32];
    const int at = TPR > 32 ? threadIdx.x : threadIdx.x & 31;
    const int group = TPR > 32 ? 0 : threadIdx.x >> 5;
    int turn = 0;
    float acc[V][E] = {};
    for (int64_t t = (int64_t)blockIdx.x * R + group; t < a.T; t += (int64_t)gridDim.x * R) {
        T *dx = static_cast<T *>(a.y_out) + t * a.H;
        if (a.mask && !a.mask[t]) {
            float z[E] = {};
            for (int k = 0; k < V; ++k) {
                const int j = (at + k * TPR) * E;
                if (j < a.H)
                    put(dx + j, z);
            }
            continue;
        }
        const T *dy = static_cast<const T *>(a.dy) + t * a.ld_dy;
        const T *h = static_cast<const T *>(a.x) + t * a.ld_x;
        const T *dh = a.residual ? static_cast<const T *>(a.residual) + t * a.ld_r : nullptr;
        Pack<T, E> py[V], ph[V], pr[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = (at + k * TPR) * E;
            if (j < a.H) {
                py[k].load(dy + j);
                ph[k].load(h + j);
                if (dh)
                    pr[k].load(dh + j);
            }
        }
        float s = 0.0f, gh = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = (at + k * TPR) * E;
            if (j < a.H) {
                float w[E], y[E], x[E];
                weights_of(a, j, w);
                py[k].get(y);
                ph[k].get(x);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    s = fmaf(x[i], x[i], s);
                    gh = fmaf(y[i] * w[i], x[i], gh);
                }
            }
        }
        row_reduce<TPR, false>(s, gh, slots, turn);
        const float H = (float)a.H, rstd = 1.0f / sqrtf(s / H + a.eps);
        const float c = rstd * rstd * (gh / H);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = (at + k * TPR) * E;
            if (j < a.H) {
                float w[E], y[E], x[E], d[E] = {};
                weights_of(a, j, w);
                py[k].get(y);
                ph[k].get(x);
                if (dh)
                    pr[k].get(d);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    d[i] = fmaf(rstd, fmaf(-x[i], c, y[i] * w[i]), d[i]);
                    acc[k][i] = fmaf(y[i], x[i] * rstd, acc[k][i]);
                }
                put(dx + j, d);
            }
        }
    }
    float *out = a.dw + (int64_t)blockIdx.x * a.H;
    if constexpr (R > 1) {  // the CTA's warps together, in order
        __shared__ float part[R][32 * E * V];
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i)
                part[group][(at + k * 32) * E + i] = acc[k][i];
        __syncthreads();
        for (int j = threadIdx.x; j < a.H; j += kCta<TPR>) {
            float v = 0.0f;
#pragma unroll
            for (int g = 0; g < R; ++g)
                v += part[g][j];
            out[j] = v;
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int j = (at + k * TPR) * E + i;
                if (j < a.H)
                    out[j] = acc[k][i];
            }
    }
}

// dweight from the CTAs' sums: 32 columns a CTA, the n sums of each over 32 threads.
__global__ void __launch_bounds__(1024) cis_rmsnorm_dweight_kernel(const float *part, int n, int H,
                                                                   float *dw)
{
    __shared__ float sh[32][33];
    const int c = threadIdx.x & 31, w = threadIdx.x >> 5, j = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < H) {
#pragma unroll 8
        for (int i = w; i < n; i += 32)
            s += part[(int64_t)i * H + j];
    }
    sh[w][c] = s;
    __syncthreads();
    s = sh[c][w];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if (c == 0 && blockIdx.x * 32 + w < H)
        dw[blockIdx.x * 32 + w] = s;
}

cudaError_t sm_count(int *n)
{
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e != cudaSuccess ? e : cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
}

// Backward CTAs: as many as the registers of an SM hold, whose sums the workspace keeps.
constexpr int kBwdThreads = 512;  // a SM's, at most 128 registers each
constexpr int kMaxSms = 256;
int64_t bwd_ctas(int64_t T, int tpr, int sms)
{
    const int cta = tpr < 128 ? 128 : tpr, rows = cta / tpr;
    const int64_t most = (int64_t)sms * (kBwdThreads > cta ? kBwdThreads / cta : 1);
    const int64_t need = (T + rows - 1) / rows;
    return need < most ? need : most;
}
int64_t most_sums(int64_t T) { return T < kMaxSms * 4 ? T : kMaxSms * 4; }

template <typename T, int E, int TPR, int V>
cudaError_t launch(const NormArgs &a, bool bwd, void *workspace, cudaStream_t s)
{
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess)
        return e;
    if (!bwd) {
        constexpr int R = kCta<TPR> / TPR;
        const int64_t need = (a.T + R - 1) / R, most = (int64_t)sms * (2048 / kCta<TPR>);
        cis_rmsnorm_fwd_kernel<T, E, TPR, V>
            <<<(unsigned)(need < most ? need : most), kCta<TPR>, 0, s>>>(a);
        return cudaGetLastError();
    }
    NormArgs b = a;
    const int64_t n = bwd_ctas(a.T, TPR, sms < kMaxSms ? sms : kMaxSms);
    if (n > 1)
        b.dw = static_cast<float *>(workspace);
    cis_rmsnorm_bwd_kernel<T, E, TPR, V><<<(unsigned)n, kCta<TPR>, 0, s>>>(b);
    e = cudaGetLastError();
    if (e != cudaSuccess || n <= 1)
        return e;
    cis_rmsnorm_dweight_kernel<<<(unsigned)((a.H + 31) / 32), 1024, 0, s>>>(b.dw, (int)n, a.H,
                                                                            a.dw);
    return cudaGetLastError();
}

// By the row's length: 16 elements a thread (8 in the shortest rows, 32 in the longest).
template <typename T, int E>
cudaError_t launch_rows(const NormArgs &a, bool bwd, void *ws, cudaStream_t s)
{
    if (a.H <= 256)
        return launch<T, E, 32, 8 / E>(a, bwd, ws, s);
    if (a.H <= 512)
        return launch<T, E, 32, 16 / E>(a, bwd, ws, s);
    if (a.H <= 2048)
        return launch<T, E, 128, 16 / E>(a, bwd, ws, s);
    if (a.H <= 4096)
        return launch<T, E, 256, 16 / E>(a, bwd, ws, s);
    if (a.H <= 8192)
        return launch<T, E, 512, 16 / E>(a, bwd, ws, s);
    return launch<T, E, 512, 32 / E>(a, bwd, ws, s);
}

// Vectors where every row of every tensor starts on 16 bytes (q's on E, the weights' on theirs).
template <typename T> cudaError_t launch_type(const NormArgs &a, bool bwd, void *ws, cudaStream_t s)
{
    constexpr int E = 16 / sizeof(T);
    auto rows = [&](const void *p, int64_t ld) {
        return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (int64_t)sizeof(T))) & 15) == 0;
    };
    const bool vec = a.H % E == 0 && rows(a.x, a.ld_x) && rows(a.residual, a.ld_r) &&
                     rows(a.dy, a.ld_dy) && rows(a.h_out, a.H) && rows(a.y_out, a.H) &&
                     (reinterpret_cast<uintptr_t>(a.q_out) & (E - 1)) == 0 &&
                     (reinterpret_cast<uintptr_t>(a.w) & 15) == 0;
    return vec ? launch_rows<T, E>(a, bwd, ws, s) : launch_rows<T, 1>(a, bwd, ws, s);
}

bool norm_args_ok(const void *p, int32_t dtype, int64_t T, int64_t H, int64_t ld, const void *w,
                  int32_t w_dtype, double eps)
{
    return row_args_ok(p, dtype, T, H, ld) && (w_dtype == CIS_F32 || w_dtype == CIS_BF16) &&
           (reinterpret_cast<uintptr_t>(w) & (w_dtype == CIS_BF16 ? 1 : 3)) == 0 &&
           eps >= 1e-12 && eps <= 1.0;
}
bool typed(const void *p, int32_t dtype)
{
    return (reinterpret_cast<uintptr_t>(p) & (dtype == CIS_BF16 ? 1 : 3)) == 0;
}
cis_status_t status_of(cudaError_t e) { return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA; }

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" CIS_API cis_status_t cis_rmsnorm_fwd(const void *x, int32_t dtype, int64_t T, int64_t H,
                                                int64_t ld_x, const void *residual, int64_t ld_r,
                                                const void *weight, int32_t weight_dtype,
                                                double eps, const uint8_t *mask, void *h_out,
                                                void *y_out, void *q_out, float *scale_out,
                                                void *stream)
{
    NvtxRange nvtx_range("cis_rmsnorm_fwd");
    if (!norm_args_ok(x, dtype, T, H, ld_x, weight, weight_dtype, eps) ||
        !typed(residual, dtype) || !typed(h_out, dtype) || !typed(y_out, dtype) ||
        !aligned4(scale_out) || (residual != nullptr && ld_r < H))
        return CIS_ERR_INVALID_ARG;
    if (T == 0)
        return CIS_OK;
    if (x == nullptr || weight == nullptr || (q_out == nullptr) != (scale_out == nullptr) ||
        (y_out == nullptr && q_out == nullptr && h_out == nullptr))
        return CIS_ERR_INVALID_ARG;
    if (H > kMaxHidden)
        return CIS_ERR_UNSUPPORTED;
    NormArgs a = {};
    a.x = x;
    a.residual = residual;
    a.w = weight;
    a.T = T;
    a.ld_x = ld_x;
    a.ld_r = residual ? ld_r : 0;
    a.H = (int)H;
    a.w_f32 = weight_dtype == CIS_F32;
    a.eps = (float)eps;
    a.mask = mask;
    a.h_out = h_out;
    a.y_out = y_out;
    a.q_out = static_cast<uint8_t *>(q_out);
    a.scale_out = scale_out;
    return status_of(dtype == CIS_BF16
                         ? launch_type<__nv_bfloat16>(a, false, nullptr, (cudaStream_t)stream)
                         : launch_type<float>(a, false, nullptr, (cudaStream_t)stream));
}

extern "C" CIS_API cis_status_t cis_rmsnorm_bwd_workspace_size(int64_t T, int64_t H, size_t *bytes)
{
    if (bytes == nullptr || T < 0 || H <= 0)
        return CIS_ERR_INVALID_ARG;
    if (H > kMaxHidden)
        return CIS_ERR_UNSUPPORTED;
    *bytes = ws_round_up((size_t)(T > 0 ? most_sums(T) : 1) * (size_t)H * sizeof(float));
    return CIS_OK;
}

extern "C" CIS_API cis_status_t cis_rmsnorm_bwd(const void *dy, const void *h, int32_t dtype,
                                                int64_t T, int64_t H, int64_t ld_dy, int64_t ld_h,
                                                const void *weight, int32_t weight_dtype,
                                                const void *dh, int64_t ld_dh, double eps,
                                                const uint8_t *mask, void *dx, float *dweight,
                                                void *workspace, size_t workspace_bytes,
                                                void *stream)
{
    NvtxRange nvtx_range("cis_rmsnorm_bwd");
    size_t need = 0;
    if (!norm_args_ok(h, dtype, T, H, ld_h, weight, weight_dtype, eps) || !typed(dy, dtype) ||
        !typed(dh, dtype) || !typed(dx, dtype) || !aligned4(dweight) || ld_dy < H ||
        (dh != nullptr && ld_dh < H) || dweight == nullptr)
        return CIS_ERR_INVALID_ARG;
    const cis_status_t st = cis_rmsnorm_bwd_workspace_size(T, H, &need);
    if (st != CIS_OK)
        return st;
    if (T == 0)
        return status_of(cudaMemsetAsync(dweight, 0, (size_t)H * sizeof(float),
                                         (cudaStream_t)stream));
    if (dy == nullptr || h == nullptr || weight == nullptr || dx == nullptr ||
        workspace == nullptr || workspace_bytes < need ||
        (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
        return CIS_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = h;
    a.residual = dh;
    a.dy = dy;
    a.w = weight;
    a.T = T;
    a.ld_x = ld_h;
    a.ld_r = dh ? ld_dh : 0;
    a.ld_dy = ld_dy;
    a.H = (int)H;
    a.w_f32 = weight_dtype == CIS_F32;
    a.eps = (float)eps;
    a.mask = mask;
    a.y_out = dx;
    a.dw = dweight;
    return status_of(dtype == CIS_BF16
                         ? launch_type<__nv_bfloat16>(a, true, workspace, (cudaStream_t)stream)
                         : launch_type<float>(a, true, workspace, (cudaStream_t)stream));
}
