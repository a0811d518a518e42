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
// Its threads are few for their registers, so that rows are copied ahead to shared memory.
//
// Bound: HBM for many rows (forward, T=16384, H=2048 bf16, 40% masked: 33 us of kernel, 38 a call,
// for 32 of traffic); backward a row's own chain of copy, sums, reduction and store, some 2,500 cycles
// with 16 warps an SM and 16 valid rows a CTA (the same batch: 35 us and 3 for dweight's second step, for
// 28 of traffic; issue 56%, HBM 4.4 TB/s).  Rows go to CTAs by their number, whatever the mask: with
// such a batch's masks the fullest CTA has 20 to 22 valid rows (as many valid rows without a mask: 36 us
// a call for 42, 4 of them the zeros' traffic).  T=3001, H=2531 fp32: 24 for 14, an element at a time.
// One row: 3 us of kernel, 7 a call.
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
    __device__ __forceinline__ void shared(uint32_t a)
    {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                     : "r"(a)
                     : "memory");
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
    __device__ __forceinline__ void shared(uint32_t a)
    {
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w)
                     : "r"(a)
                     : "memory");
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
    __device__ __forceinline__ void shared(uint32_t a)
    {
        if constexpr (sizeof(T) == 4)
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(q) : "r"(a) : "memory");
    }
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

// The rows of a group of threads, t = first, first + step, ..., and which of the next ones count
// (bit i: row t + i step): the mask is read before the loads that it decides about, and what was
// read is looked at a row later.
struct RowWalk {
    static constexpr int kKnown = 8;
    const uint8_t *mask;
    int64_t T, step, t;
    unsigned bits, more;
    __device__ __forceinline__ RowWalk(const uint8_t *m, int64_t T_, int64_t first, int64_t step_)
        : mask(m), T(T_), step(step_), t(first), bits(0)
    {
        unsigned v[kKnown];
#pragma unroll
        for (int i = 0; i < kKnown; ++i)
            v[i] = valid(t + i * step);
#pragma unroll
        for (int i = 0; i < kKnown; ++i)
            bits |= (unsigned)(v[i] != 0) << i;
        more = valid(t + kKnown * step);
    }
    __device__ __forceinline__ unsigned valid(int64_t r) const
    {
        return r < T ? (mask ? (unsigned)__ldg(mask + r) : 1u) : 0u;
    }
    __device__ __forceinline__ bool on(int i) const { return bits >> i & 1; }
    __device__ __forceinline__ void advance()
    {
        bits = bits >> 1 | (unsigned)(more != 0) << (kKnown - 1);
        t += step;
        more = valid(t + kKnown * step);
    }
};

// Whether no thread has an element of its vector k, `step` elements behind the one before: the
// same for all, so that what is not there is not issued either.  Looked at for every second vector
// (T=3001, H=2531, rows not aligned: norm in fp32 36 to 33 us, bf16 to 8 bits 27 to 23, gradients in
// bf16 29 to 27; for every vector its branches cost more: 35, 25, 31).
template <int V> __device__ __forceinline__ bool past(int k, int step, int H)
{
    return k > 0 && k % 2 == 0 && k * step >= H;
}

// K tensors' rows on their way: a thread copies what it will use itself, V vectors of E elements of
// each, into places of its own in shared memory, S - 1 rows ahead, and waits for nobody else.
// Elements of 2 bytes by themselves cannot be copied so: they are loaded when they are used.  (Rows
// that start anywhere copied by 16 bytes and read by other threads, behind a barrier: 35 us for 27 at
// T=3001, H=2531 fp32.)
template <typename T, int E, int NT, int V, int K, int S> struct Rows {
    static constexpr bool kAsync = sizeof(Pack<T, E>) >= 4;
    static constexpr size_t kBytes = kAsync ? sizeof(Pack<T, E>) * NT * V * K * S : 0;
    const T *base[K];  // this thread's first element of row 0 (null: no such tensor)
    int64_t ld[K];
    int left, stride;  // elements from this thread's first on, and between its vectors
    int H;
    uint32_t place;
    int stage = 0;

    __device__ __forceinline__ void copy(int64_t t, int s)
    {
        if constexpr (kAsync) {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (base[i]) {
                    const T *row = base[i] + t * ld[i];
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        if (past<V>(k, stride, H))
                            break;
                        if (k * stride < left) {
                            const uint32_t to =
                                place + (uint32_t)(((s * K + i) * V + k) * NT *
                                                   sizeof(Pack<T, E>));
                            if constexpr (sizeof(Pack<T, E>) == 16)
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to),
                                             "l"(row + k * stride)
                                             : "memory");
                            else
                                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to),
                                             "l"(row + k * stride)
                                             : "memory");
                        }
                    }
                }
        }
    }
    // The first S - 1 rows.
    __device__ __forceinline__ void start(const RowWalk &w)
    {
#pragma unroll
        for (int i = 0; i < S - 1; ++i) {
            if (w.on(i))
                copy(w.t + i * w.step, i);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }
    // The current row, and one more on its way.
    __device__ __forceinline__ void take(const RowWalk &w, Pack<T, E> (&p)[K][V])
    {
        if constexpr (kAsync) {
            const int next = stage == 0 ? S - 1 : stage - 1;
            if (w.on(S - 1))
                copy(w.t + (S - 1) * w.step, next);
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
            if (w.on(0)) {
#pragma unroll
                for (int i = 0; i < K; ++i)
                    if (base[i])
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            if (past<V>(k, stride, H))
                                break;
                            if (k * stride < left)
                                p[i][k].shared(place + (uint32_t)(((stage * K + i) * V + k) * NT *
                                                                  sizeof(Pack<T, E>)));
                        }
            }
            stage = stage + 1 == S ? 0 : stage + 1;
        } else if (w.on(0)) {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (base[i])
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        if (past<V>(k, stride, H))
                            break;
                        if (k * stride < left)
                            p[i][k].load(base[i] + w.t * ld[i] + k * stride);
                    }
        }
    }
};

// The forward kernel: TPR threads a row, V vectors of E elements each.  Enough CTAs hide one
// another's latencies (rows copied ahead, as in the backward kernel, took 41 us for 38 at T=16384,
// H=2048, 40% padding; weights kept in registers, or packed instructions, 43).
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
                if (past<V>(k, TPR * E, a.H))
                    break;
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
            if (past<V>(k, TPR * E, a.H))
                break;
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
            if (past<V>(k, TPR * E, a.H))
                break;
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
                if (past<V>(k, TPR * E, a.H))
                    break;
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
                if (past<V>(k, TPR * E, a.H))
                    break;
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

// The backward kernel's threads an SM, whose rows on their way have kRowBytes of its shared memory
// (640 threads spill; 8 elements a thread and 768 took 49 us for 42 at T=16384, H=2048, 40% padding;
// rows read twice from shared memory allow 640 to 1024: 41.5 to 43, and 29 to 35 us for 27 at T=3001,
// H=2531 fp32: what the warps gave, the second reading took).
constexpr int kBwdThreads = 512, kRowBytes = 200 * 1024;
constexpr int kMaxSms = 256;
// CTAs of TPR threads (128 at least) an SM.
constexpr int ctas_of(int tpr, int threads)
{
    return threads > tpr && threads > 128 ? threads / (tpr < 128 ? 128 : tpr) : 1;
}
// The backward kernel.
template <typename T, int E, int TPR, int V, int S>
__global__ void __launch_bounds__(kCta<TPR>, ctas_of(TPR, kBwdThreads))
    cis_rmsnorm_bwd_kernel(const NormArgs a)
{
    constexpr int R = kCta<TPR> / TPR, kStep = TPR * E;
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    __shared__ float2 slots[2][32];
    if (threadIdx.x == 0)
        allow_next_grid();
    const int at = (TPR > 32 ? threadIdx.x : threadIdx.x & 31) * E;
    const int group = TPR > 32 ? 0 : threadIdx.x >> 5;
    int turn = 0;
    float acc[V][E] = {};
    RowWalk row(a.mask, a.T, (int64_t)blockIdx.x * R + group, (int64_t)gridDim.x * R);
    using In = Rows<T, E, kCta<TPR>, V, 3, S>;
    In in{{static_cast<const T *>(a.dy) + at, static_cast<const T *>(a.x) + at,
           a.residual ? static_cast<const T *>(a.residual) + at : nullptr},
          {a.ld_dy, a.ld_x, a.ld_r}, a.H - at, kStep, a.H,
          (uint32_t)__cvta_generic_to_shared(dyn_smem) +
              (uint32_t)(threadIdx.x * sizeof(Pack<T, E>))};
    in.start(row);
    float w[V][E];
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (at + k * kStep < a.H)
            weights_of(a, at + k * kStep, w[k]);
    for (; row.t < a.T; row.advance()) {
        T *dx = static_cast<T *>(a.y_out) + row.t * a.H;
        Pack<T, E> now[3][V];
        in.take(row, now);
        if (!row.on(0)) {
            float z[E] = {};
            for (int k = 0; k < V; ++k) {
                const int j = at + k * kStep;
                if (j < a.H)
                    put(dx + j, z);
            }
            continue;
        }
        float s = 0.0f, gh = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = at + k * kStep;
            if (past<V>(k, kStep, a.H))
                break;
            if (j < a.H) {
                float y[E], x[E];
                now[0][k].get(y);
                now[1][k].get(x);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    s = fmaf(x[i], x[i], s);
                    gh = fmaf(y[i] * w[k][i], x[i], gh);
                }
            }
        }
        row_reduce<TPR, false>(s, gh, slots, turn);
        const float H = (float)a.H, rstd = 1.0f / sqrtf(s / H + a.eps);
        const float c = rstd * rstd * (gh / H);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int j = at + k * kStep;
            if (past<V>(k, kStep, a.H))
                break;
            if (j < a.H) {
                float y[E], x[E], d[E] = {};
                now[0][k].get(y);
                now[1][k].get(x);
                if (a.residual)
                    now[2][k].get(d);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    d[i] = fmaf(rstd, fmaf(-x[i], c, y[i] * w[k][i]), d[i]);
                    acc[k][i] = fmaf(y[i], x[i] * rstd, acc[k][i]);
                }
                put(dx + j, d);
            }
        }
    }
    float *out = a.dw + (int64_t)blockIdx.x * a.H;
    if constexpr (R > 1) {  // the CTA's warps together, in order (where their rows were copied to)
        float(*part)[32 * E * V] = reinterpret_cast<float(*)[32 * E * V]>(dyn_smem);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i)
                part[group][at + k * kStep + i] = acc[k][i];
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
                const int j = at + k * kStep + i;
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
    grid_wait();
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

// Backward CTAs: as many as run at a time, whose sums the workspace keeps.
int64_t bwd_ctas(int64_t T, int tpr, int sms)
{
    const int cta = tpr < 128 ? 128 : tpr, rows = cta / tpr;
    const int64_t most = (int64_t)sms * ctas_of(tpr, kBwdThreads);
    const int64_t need = (T + rows - 1) / rows;
    return need < most ? need : most;
}
constexpr int64_t kMaxSums = kMaxSms * (kBwdThreads / 128);
int64_t most_sums(int64_t T) { return T < kMaxSums ? T : kMaxSums; }

// Rows on their way: four, or as many as fit.
template <typename T, int E, int NT, int V, int K> constexpr int stages_of(int ctas)
{
    return Rows<T, E, NT, V, K, 4>::kBytes * ctas <= kRowBytes   ? 4
           : Rows<T, E, NT, V, K, 2>::kBytes * ctas <= kRowBytes ? 2
                                                                 : 1;
}

template <typename T, int E, int TPR, int V>
cudaError_t launch(const NormArgs &a, bool bwd, void *workspace, cudaStream_t s)
{
    constexpr int NT = kCta<TPR>, R = NT / TPR;
    int sms = 0;
    cudaError_t e = sm_count(&sms);
    if (e != cudaSuccess)
        return e;
    if (!bwd) {
        const int64_t need = (a.T + R - 1) / R, most = (int64_t)sms * (2048 / NT);
        cis_rmsnorm_fwd_kernel<T, E, TPR, V>
            <<<(unsigned)(need < most ? need : most), NT, 0, s>>>(a);
        return cudaGetLastError();
    }
    constexpr int S = stages_of<T, E, NT, V, 3>(ctas_of(TPR, kBwdThreads));
    // (the sums have no place of their own: with 8 KB for them an SM held three CTAs, not four, for H
    // from 257 to 512; T=65536, H=500 fp32: 91.4 us for 92.9, H=512 85.0 either way)
    constexpr size_t rows = Rows<T, E, NT, V, 3, S>::kBytes;
    constexpr size_t sums = R > 1 ? sizeof(float) * R * 32 * E * V : 0;
    constexpr size_t smem = rows > sums ? rows : sums;
    auto kern = cis_rmsnorm_bwd_kernel<T, E, TPR, V, S>;
    if (smem > 32 * 1024 && (e = allow_smem(kern, smem)) != cudaSuccess)
        return e;
    NormArgs b = a;
    const int64_t n = bwd_ctas(a.T, TPR, sms < kMaxSms ? sms : kMaxSms);
    if (n > 1)
        b.dw = static_cast<float *>(workspace);
    kern<<<(unsigned)n, NT, smem, s>>>(b);
    e = cudaGetLastError();
    if (e != cudaSuccess || n <= 1)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.H + 31) / 32));
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, cis_rmsnorm_dweight_kernel, (const float *)b.dw, (int)n, a.H, a.dw);
    return e != cudaSuccess ? e : cudaGetLastError();
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
