// cis_topk.cu -- the K most likely tokens of each row with their log-probabilities
// (cis_topk_logprobs): a teacher's lists.
//
// A row's order is (z descending, index ascending); lp_k = z_k / tau - log sum e^{z / tau}.
//
// The row is read once, straight into registers (cis_expacc.cuh), as by the forward kernel;
// besides the sum of exponentials every thread keeps the maximum of each batch of vectors, in
// shared memory, and four maxima over a quarter of its batches each.  With C CTAs on the row
// and r = ceil(K / C), at least r entries of a CTA are not below the r-th largest of its
// maxima, and the least of those over the CTAs bounds the row's K largest from below.  For
// r <= 16 the CTA's is taken among its warps' four largest; above, it is the least of its 8
// warps' own ceil(r / 8)-th largest, which needs no exchange of more than one number.  The batches that reach that bound are read again (from L2), their entries
// that reach it are the candidates, and the first CTA sorts them.  A row with more candidates
// than fit (long runs of equal entries) is left to the exact kernel, which follows.
//
// Before (slices of the row in the shared memory of four CTAs, read three times): T=8192,
// V=151936, K=64 took 1336 us, at 16 warps an SM and 4900 issue slots a slice.
#include <math.h>

#include "cis_expacc.cuh"
#include "cis_nvtx.h"
#include "cis_select.cuh"

namespace cis {
namespace {

constexpr int kSelThreads = 512;
constexpr int kSelCluster = 8;

// Sort n <= 512 pairs in descending order (bitonic, padded with 0); all threads.
template <int NT> __device__ void sort_list(mass_t *list, int n)
{
    int size = 2;
    while (size < n)
        size *= 2;
    for (int i = threadIdx.x; i < size; i += NT)
        if (i >= n)
            list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int i = threadIdx.x; i < size / 2; i += NT) {
                const int lo = 2 * j * (i / j) + i % j, hi = lo + j;
                const mass_t x = list[lo], y = list[hi];
                if ((x < y) == ((lo & k) == 0)) {
                    list[lo] = y;
                    list[hi] = x;
                }
            }
            __syncthreads();
        }
}

__device__ __forceinline__ void fill_row(const TopkArgs &a, int64_t t, float lp, float lse)
{
    for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
        a.ids_out[t * a.K + k] = -1;
        a.lp_out[t * a.K + k] = lp;
    }
    if (threadIdx.x == 0 && a.lse_out)
        a.lse_out[t] = lse;
}

constexpr int32_t kTodo = -2;    // in a row's first id: left to the exact kernel

template <int NT> struct TopkShared {
    float part[kMaxCluster][3];  // each CTA's max, sum and bound
    MaxSumU red[NT / 32];
    float bound[NT / 32 * 4];
    int items, n;
    int count[kMaxCluster];
};

// A value that at least r (1 .. 128) of the warp's 128 maxima are not below: the r-th
// largest, rounded down to 16 bits.  Bit by bit from the first in which the warp's keys
// differ.
__device__ __forceinline__ float warp_bound(const float (&m)[4], int r)
{
    uint32_t k[4], lo = 0xffffu, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k[i] = order_key(m[i]) >> 16;
        lo = min(lo, k[i]);
        hi = max(hi, k[i]);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const int bits = 32 - __clz(lo ^ hi);
    uint32_t v = (hi >> bits) << bits;
    for (int b = bits - 1; b >= 0; --b) {
        const uint32_t mid = v | (1u << b);
        const uint32_t n = (k[0] >= mid) + (k[1] >= mid) + (k[2] >= mid) + (k[3] >= mid);
        if (__reduce_add_sync(0xffffffffu, n) >= (uint32_t)r)
            v = mid;
    }
    return v <= (order_key(-INFINITY) >> 16) ? -INFINITY : key_value(v << 16);
}

// The warp's kTop largest maxima, rounded down to 16 bits, into `out`.
constexpr int kTop = 4;
__device__ __forceinline__ void warp_top(const float (&m)[4], float *out)
{
    uint32_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // made different by the lane and place: one goes at a time
        k[i] = (order_key(m[i]) & 0xffff0000u) | ((threadIdx.x & 31) << 2) | i;
#pragma unroll
    for (int n = 0; n < kTop; ++n) {
        const uint32_t best = __reduce_max_sync(0xffffffffu, max(max(k[0], k[1]), max(k[2], k[3])));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            k[i] = k[i] == best ? 0u : k[i];
        const uint32_t v = best >> 16;
        if ((threadIdx.x & 31) == 0)
            out[n] = v <= (order_key(-INFINITY) >> 16) ? -INFINITY : key_value(v << 16);
    }
}
// The r-th largest (1 .. n) of n <= 32 values; every lane gets it.
__device__ __forceinline__ float nth_of(const float *v, int n, int r)
{
    const int lane = threadIdx.x & 31;
    const float x = lane < n ? v[lane] : -INFINITY;
    int before = 0;  // values ahead of this one
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const float y = __shfl_sync(0xffffffffu, x, i);
        before += y > x || (y == x && i < lane);
    }
    const unsigned who = __ballot_sync(0xffffffffu, before == r - 1);
    return __shfl_sync(0xffffffffu, x, who ? __ffs(who) - 1 : 0);
}

// The maxima of a vector's four quarters.
__device__ __forceinline__ void quarters(const Vec<__nv_bfloat16> &x, float (&m)[4])
{
    const uint32_t w[4] = {x.q.x, x.q.y, x.q.z, x.q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m[i] = max_nan(bf16_lo(w[i]), bf16_hi(w[i]));
}
__device__ __forceinline__ void quarters(const Vec<float> &x, float (&m)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m[i] = x.entry(i);
}

// kB vectors a batch (1: short rows, and the four maxima are over the vectors' quarters); r:
// see the top; cap: items and candidates that fit, a power of two.  Dynamic shared memory: cap candidates, cap items, the batches' maxima (and, in
// their place, the candidates of all CTAs).
template <typename InT, int NT, int kB>
__global__ void __launch_bounds__(NT)
    cis_topk_kernel(const __grid_constant__ TopkArgs a, unsigned cs, int r, int cap)
{
    constexpr int EV = Vec<InT>::kN;
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    __shared__ TopkShared<NT> sh;
    mass_t *list = reinterpret_cast<mass_t *>(dyn_smem);
    int *items = reinterpret_cast<int *>(list + cap);
    float *bmax = reinterpret_cast<float *>(items + cap);
    const int64_t t = blockIdx.x / cs;
    const unsigned rank = blockIdx.x - (unsigned)t * cs;
    const int tid = threadIdx.x;
    if (tid == 0)
        allow_next_grid();
    if (a.mask != nullptr && a.mask[t] == 0) {  // the same branch in every CTA of the row
        if (rank == 0)
            fill_row(a, t, -INFINITY, 0.0f);
        return;
    }
    if (tid == 0)
        sh.items = sh.n = 0;
    const InT *row = reinterpret_cast<const InT *>(a.logits) + t * a.ld;
    const int V = (int)a.V;
    const int head = row_head(row, V);
    const int nvec = (V - head) / EV;
    const int v0 = (int)((int64_t)nvec * rank / cs), v1 = (int)((int64_t)nvec * (rank + 1) / cs);
    const uint4 *rv = reinterpret_cast<const uint4 *>(row + head);

    ExpAcc<false, true> acc;
    acc.k = a.sc.kappa;
    acc.h = a.sc.huge;
    float q[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    float *mine = bmax + tid;
    int nb = 0;
    auto batch = [&](const Vec<InT> (&x)[kB]) {
        const float mx = vec_max<kB>(x);
        *mine = mx;
        mine += NT;
        ++nb;
        if constexpr (kB == 1) {
            float p[4];
            quarters(x[0], p);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[i] = max_nan(q[i], p[i]);
        } else {
            const float q0 = max_nan(q[0], mx);
            q[0] = q[1];
            q[1] = q[2];
            q[2] = q[3];
            q[3] = q0;
        }
        take<false, kB>(acc, x, mx);
    };
    int v = v0 + tid;
    for (; v + (kB - 1) * NT < v1; v += kB * NT) {
        Vec<InT> x[kB];
#pragma unroll
        for (int k = 0; k < kB; ++k)
            x[k].q = __ldg(rv + v + k * NT);
        batch(x);
    }
    if (kB > 1 && v < v1) {  // the last, partial batch: absent vectors count as -inf
        Vec<InT> x[kB];
#pragma unroll
        for (int k = 0; k < kB; ++k)
            x[k].q = v + k * NT < v1 ? __ldg(rv + v + k * NT)
                                     : make_uint4(Vec<InT>::kNone, Vec<InT>::kNone,
                                                  Vec<InT>::kNone, Vec<InT>::kNone);
        batch(x);
    }
    int end = -1;  // the ragged ends, fewer than 2 EV entries: one a thread of the first CTA
    float zend = -INFINITY;
    if (rank == 0) {
        const int tail0 = head + nvec * EV;
        if (tid < head)
            end = tid;
        else if (tid - head < V - tail0)
            end = tail0 + tid - head;
        if (end >= 0) {
            zend = to_f32(row[end]);
            acc.raise(zend);
            if (acc.m != -INFINITY)
                acc.add_entry(zend);
            q[0] = max_nan(q[0], zend);
        }
    }
    constexpr int W = NT / 32;
    const bool few = r <= 2 * W;
    if (few) {
        warp_top(q, sh.bound + kTop * (tid >> 5));
    } else {
        const float wb = warp_bound(q, (r + W - 1) / W);
        if ((tid & 31) == 0)
            sh.bound[tid >> 5] = wb;
    }
    MaxSumU o = block_exp<NT>(acc, sh.red);  // (its barriers)
    float bound = sh.bound[0];
    if (few) {
        bound = nth_of(sh.bound, kTop * W, r);
    } else {
#pragma unroll
        for (int w = 1; w < W; ++w)
            bound = fminf(bound, sh.bound[w]);
    }
    if (cs > 1) {
        cluster_sync_data();  // every CTA of the row has started
        if (tid < (int)cs) {
            float *to = cg::this_cluster().map_shared_rank(&sh.part[rank][0], tid);
            to[0] = o.m;
            to[1] = o.s;
            to[2] = bound;
        }
        cluster_sync_data();
        float M = sh.part[0][0], S = 0.0f;
        for (unsigned c = 0; c < cs; ++c) {
            M = fmaxf(M, sh.part[c][0]);
            bound = fminf(bound, sh.part[c][2]);
        }
        for (unsigned c = 0; c < cs; ++c)  // in rank order
            S += sh.part[c][1] * exp2f((sh.part[c][0] - M) * a.sc.kappa);
        o.m = M;
        o.s = S;
    }
    const bool bad = !(o.s > 0.0f && o.s < INFINITY) || !(fabsf(o.m) < INFINITY);

    // The batches that reach the bound, then their vectors, one a thread.
    for (int b = 0; b < nb; ++b) {
        const float x = bmax[b * NT + tid];
        if (x >= bound && x != -INFINITY) {
            const int at = atomicAdd(&sh.items, 1);
            if (at < cap)
                items[at] = v0 + b * kB * NT + tid;
        }
    }
    auto offer = [&](float z, int j) {
        if (z >= bound && z != -INFINITY) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < cap)
                list[at] = order_pair(order_key(z), (uint32_t)j);
        }
    };
    if (end >= 0)
        offer(zend, end);
    __syncthreads();
    const int m = min(sh.items, cap);
    for (int i = tid; i < m * kB; i += NT) {
        const int w = items[i / kB] + (i % kB) * NT;
        if (w >= v1)
            continue;
        Vec<InT> x;
        x.q = __ldg(rv + w);
#pragma unroll
        for (int k = 0; k < EV; ++k)
            offer(x.entry(k), head + w * EV + k);
    }
    __syncthreads();
    int n = sh.items > cap ? cap + 1 : sh.n;
    if (cs > 1) {  // the first CTA gathers the lists
        if (tid == 0)
            sh.n = n;
        cluster_sync_data();
        mass_t *all = reinterpret_cast<mass_t *>(bmax);
        if (rank == 0) {
            const cg::cluster_group cluster = cg::this_cluster();
            if (tid < (int)cs)
                sh.count[tid] = *cluster.map_shared_rank(&sh.n, tid);
            __syncthreads();
            n = 0;
            for (unsigned c = 0; c < cs; ++c) {
                const int k = sh.count[c];
                if (n + k <= cap && k <= cap) {
                    const mass_t *from = cluster.map_shared_rank(list, (int)c);
                    for (int i = tid; i < k; i += NT)
                        all[n + i] = from[i];
                    n += k;
                } else {
                    n = cap + 1;
                }
            }
        }
        cluster_sync_data();  // no CTA leaves while its list is read
        if (rank != 0)
            return;
        list = all;
    }
    if (bad) {
        fill_row(a, t, NAN, NAN);
        if (tid == 0)
            set_status(a.status, kStatusBadInput);
        return;
    }
    if (n > cap) {
        if (tid == 0)
            a.ids_out[t * a.K] = kTodo;
        return;
    }
    sort_list<NT>(list, n);
    const float ls = logf(o.s), lsl = log_residual(o.s, ls);
    for (int i = tid; i < a.K; i += NT) {
        if (i < n) {
            const mass_t p = list[i];
            float l, e;
            const float x = scaled_diff(key_value((uint32_t)(p >> 32)), o.m, a.sc, l);
            const float u = two_sum(x, -ls, e);
            a.ids_out[t * a.K + i] = (int32_t)(0xffffffffu - (uint32_t)p);
            a.lp_out[t * a.K + i] = u + (e + l - lsl);
        } else {
            a.ids_out[t * a.K + i] = -1;
            a.lp_out[t * a.K + i] = -INFINITY;
        }
    }
    if (tid == 0 && a.lse_out) {
        float e;
        const float p = o.m * a.sc.hi;
        const float pl = isfinite(p) ? fmaf(o.m, a.sc.hi, -p) + o.m * a.sc.lo : 0.0f;
        const float u = two_sum(p, ls, e);
        a.lse_out[t] = u + (e + pl + lsl);
    }
}

// Any row, exactly: a cluster per row reads it from memory once for each step.
template <typename InT>
__global__ void __launch_bounds__(kSelThreads)
    cis_topk_exact_kernel(const __grid_constant__ TopkArgs a, bool every)
{
    __shared__ SelectShared<kSelThreads> sh;
    int turn = 0;
    if (threadIdx.x == 0)
        allow_next_grid();
    grid_wait();
    RowsLeft<kSelThreads> rows(sh, a.T, gridDim.x / kSelCluster, blockIdx.x / kSelCluster);
    for (;;) {
        const int64_t t = rows.next([&](int64_t i) {
            return every || a.ids_out[i * a.K] == kTodo;
        });
        if (t < 0)
            break;
        RowSelect<InT, kSelThreads> rs(sh, reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V,
                                       turn);
        if (a.mask && a.mask[t] == 0) {
            if (rs.rank == 0)
                fill_row(a, t, -INFINITY, 0.0f);
            continue;
        }
        bool bad;
        const uint32_t mk = rs.max_key(bad);
        if (bad) {  // as every CTA of the cluster finds
            if (rs.rank == 0) {
                fill_row(a, t, NAN, NAN);
                if (threadIdx.x == 0)
                    set_status(a.status, kStatusBadInput);
            }
            continue;
        }
        const float M = key_value(mk);
        const int K = (int)(a.K < a.V ? a.K : a.V);
        mass_t above, equal;
        const uint32_t key =
            rs.select((mass_t)K, [](float, uint32_t) { return (mass_t)1; }, above, equal);
        const mass_t ties = (mass_t)K - above;
        if (rs.rank == 0 && threadIdx.x == 0)
            sh.n = 0;
        mass_t mass = 0, eq = 0, x, eq0;
        rs.each([&](int64_t, float z) {
            mass += fixed_mass(z, M, a.sc);
            eq += order_key(z) == key;
        });
        rs.cluster_sum(mass, eq, x, eq0);  // (its barrier: the list's count is 0)
        int *n = rs.cl.map_shared_rank(&sh.n, 0);
        mass_t *list = rs.cl.map_shared_rank(&sh.list[0], 0);
        mass_t seen = eq0;
        for (int64_t b = rs.j0; b < rs.j1; b += kSelThreads) {
            const int64_t j = b + threadIdx.x;
            const uint32_t k = j < rs.j1 ? order_key(to_f32(rs.row[j])) : 0;
            bool take = j < rs.j1 && k > key;
            if (seen < ties) {  // ties are taken by index
                const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
                const bool tie = j < rs.j1 && k == key;
                const unsigned w = __ballot_sync(0xffffffffu, tie);
                __syncthreads();
                if (lane == 0)
                    sh.red[0][wid] = __popc(w);
                __syncthreads();
                mass_t before = seen + __popc(w & ((1u << lane) - 1)), all = 0;
                for (int i = 0; i < kSelThreads / 32; ++i) {
                    before += i < wid ? sh.red[0][i] : 0;
                    all += sh.red[0][i];
                }
                take = take || (tie && before < ties);
                seen += all;
            }
            if (take)
                list[atomicAdd(n, 1)] = order_pair(k, (uint32_t)j);
        }
        rs.cl.sync();
        if (rs.rank == 0) {
            sort_list<kSelThreads>(sh.list, K);
            const double lm = log(mass_value(mass));
            const double inv = (double)a.sc.hi + (double)a.sc.lo;
            for (int i = threadIdx.x; i < a.K; i += kSelThreads) {
                const mass_t p = i < K ? sh.list[i] : 0;
                const float z = key_value((uint32_t)(p >> 32));
                const bool on = i < K && z != -INFINITY;
                a.ids_out[t * a.K + i] = on ? (int32_t)(0xffffffffu - (uint32_t)p) : -1;
                a.lp_out[t * a.K + i] =
                    on ? (float)(((double)z - (double)M) * inv - lm) : -INFINITY;
            }
            if (threadIdx.x == 0 && a.lse_out)
                a.lse_out[t] = (float)((double)M * inv + lm);
        }
        __syncthreads();
    }
    cg::this_cluster().sync();  // no CTA leaves while a peer reads its shared memory
}

template <typename InT, int NT, int kB>
cudaError_t launch_fast(const TopkArgs &a, int cs, cudaStream_t s)
{
    auto kern = cis_topk_kernel<InT, NT, kB>;
    const int64_t vecs = (a.V * (int64_t)sizeof(InT) / 16 + cs - 1) / cs;
    const int64_t nb = (vecs + kB * NT - 1) / (kB * NT);
    // short rows always fit, whatever their entries; a long one has some 2 K candidates
    const int cap = a.V <= 1024 ? 1024 : a.V <= 2048 ? 2048 : a.K <= 64 ? 512 : 1024;
    size_t maxima = (size_t)(nb * NT) * sizeof(float);
    if (cs > 1 && maxima < cap * sizeof(mass_t))
        maxima = cap * sizeof(mass_t);
    const size_t smem = cap * (sizeof(mass_t) + sizeof(int)) + maxima;
    if (smem > 200 * 1024)
        return cudaErrorNotSupported;
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * cs), 1, 1);
    cfg.blockDim = dim3(NT, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cs > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, a, (unsigned)cs, (a.K + cs - 1) / cs, cap);
}

// The exact kernel: every row, or those that the fast one before it left.
template <typename InT>
cudaError_t launch_exact(const TopkArgs &a, bool every, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    const int64_t groups = a.T < 38 ? a.T : 38;
    cfg.gridDim = dim3((unsigned)(groups * kSelCluster));
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kSelCluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = every ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, cis_topk_exact_kernel<InT>, a, every);
}

template <typename InT> cudaError_t launch_topk(const TopkArgs &a, cudaStream_t s)
{
    if (a.T * kMaxCluster > 0x7fffffffLL)
        return launch_exact<InT>(a, true, s);
    const int64_t nvec = a.V * (int64_t)sizeof(InT) / 16;
    int cs = 1;
    while (cs < kMaxCluster && a.T * cs * 2 <= 608 && nvec / (2 * cs) >= 512)
        cs *= 2;
    while (cs < kMaxCluster && nvec / cs > 65536)  // the maxima fit shared memory
        cs *= 2;
    const cudaError_t e = nvec <= 512         ? launch_fast<InT, 64, 1>(a, cs, s)
                          : nvec <= 4096 * cs ? launch_fast<InT, 256, 1>(a, cs, s)
                                              : launch_fast<InT, 256, 4>(a, cs, s);
    return e != cudaSuccess ? e : launch_exact<InT>(a, false, s);
}

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" CIS_API cis_status_t cis_topk_logprobs(const void *logits, int32_t dtype, int64_t T,
                                                  int64_t V, int64_t ld, int32_t K,
                                                  double temperature, const uint8_t *mask,
                                                  int32_t *ids_out, float *lp_out, float *lse_out,
                                                  int32_t *dev_status, void *stream)
{
    NvtxRange nvtx_range("cis_topk_logprobs");
    if (!row_args_ok(logits, dtype, T, V, ld) || K < 1 || K > CIS_MAX_TOPK ||
        !temperature_ok(temperature))
        return CIS_ERR_INVALID_ARG;
    if (T == 0)
        return CIS_OK;
    if (logits == nullptr || ids_out == nullptr || lp_out == nullptr)
        return CIS_ERR_INVALID_ARG;
    if (V > kMaxRowEntries)
        return CIS_ERR_UNSUPPORTED;
    TopkArgs a = {};
    a.logits = logits;
    a.T = T;
    a.V = V;
    a.ld = ld;
    a.K = K;
    a.sc = make_scale(temperature);
    a.mask = mask;
    a.ids_out = ids_out;
    a.lp_out = lp_out;
    a.lse_out = lse_out;
    a.status = dev_status;
    const cudaError_t e = dtype == CIS_BF16
                              ? launch_topk<__nv_bfloat16>(a, (cudaStream_t)stream)
                              : launch_topk<float>(a, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
