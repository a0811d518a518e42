// cis_topk.cu -- the K most likely tokens of each row with their log-probabilities
// (cis_topk_logprobs): a teacher's lists.
//
// A row's order is (z descending, index ascending); lp_k = z_k / tau - log sum e^{z / tau}.
//
// A cluster of CTAs holds the row in shared memory.  Its first pass keeps, besides the sum of
// exponentials, four maxima a thread, over disjoint quarters of the thread's entries.  With W
// warps in the cluster and r = ceil(K / W), at least K entries are not below the least of the
// warps' r-th largest maxima: that bound leaves some 2 K candidates of a row of any length
// (measured: 100 to 330 for K = 64, V = 151936), which the second pass finds and the first
// CTA puts in order by counting, for each, those before it.  A row with more candidates than
// fit (long runs of equal entries) is left to the exact kernel, which follows.
#include <math.h>

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

constexpr int kCand = 1024;     // candidates of a row
constexpr int kCandCta = 512;   // of one CTA
constexpr int32_t kTodo = -2;   // in a row's first id: left to the exact kernel

struct TopkShared {
    alignas(8) uint64_t bar[kChunks];
    alignas(8) uint64_t xbar;
    alignas(16) float4 part[kMaxCluster];  // max, sum, bound
    MaxSum red[16];
    float bound[16];
    int n;
    int count[kMaxCluster];
    alignas(16) mass_t list[kCandCta];
};

// The four maxima of a thread.
__device__ __forceinline__ void max_parts(const MaxAcc<__nv_bfloat16> &a, float (&m)[4])
{
    m[0] = __low2float(a.a0);
    m[1] = __high2float(a.a0);
    m[2] = __low2float(a.a1);
    m[3] = __high2float(a.a1);
}
__device__ __forceinline__ void max_parts(const MaxAcc<float> &a, float (&m)[4])
{
    for (int i = 0; i < 4; ++i)
        m[i] = a.m[i];
}

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

template <typename InT, int NT>
__global__ void __launch_bounds__(NT)
    cis_topk_kernel(const __grid_constant__ TopkArgs a, int64_t slice, int r)
{
    extern __shared__ __align__(128) uint8_t dyn_smem[];
    __shared__ TopkShared sh;
    uint8_t *slab = slab_start(dyn_smem);
    const ClusterPlace cl = cluster_place();
    const int64_t t = blockIdx.x / cl.size;
    const int tid = threadIdx.x;
    if (tid == 0)
        allow_next_grid();
    if (a.mask != nullptr && a.mask[t] == 0) {  // the same branch in the whole cluster
        if (cl.rank == 0)
            fill_row(a, t, -INFINITY, 0.0f);
        return;
    }
    const int64_t v0 = (int64_t)cl.rank * slice;
    const Slice<InT> sl(reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V, v0, slice);
    if (tid == 0) {
        for (int c = 0; c < kChunks; ++c)
            mbar_init_only(smem_u32(&sh.bar[c]), 1);
        mbar_init_only(smem_u32(&sh.xbar), 1);
        mbar_init_fence();
        mbar_expect_tx(smem_u32(&sh.xbar), (uint32_t)(cl.size * sizeof(float4)));
        sl.copy(slab, sh.bar);
        sh.n = 0;
    }
    if (tid >= 32 && tid < 64)
        sl.ends(slab, tid - 32);
    cluster_arrive_relaxed();
    __syncthreads();

    MaxAcc<InT> macc;
    for (int c = 0; c < kChunks && sl.chunk_begin(c) < sl.ng; ++c) {
        wait_or_flag(smem_u32(&sh.bar[c]), false, a.status);
        macc.consume(slab, sl.template first<NT>(c), sl.chunk_end(c), NT);
    }
    const float kappa = a.sc.kappa, m = macc.result();
    float s = 0.0f;
    if (m != -INFINITY) {
#pragma unroll 2
        for (int g = tid; g < sl.ng; g += NT) {
            float z[8];
            load8_any<InT>(slab, g, z);
            s += sum8_scaled(z, m, kappa);
        }
    }
    float parts[4];
    max_parts(macc, parts);
    const float wb = warp_bound(parts, r);
    if ((tid & 31) == 0)
        sh.bound[tid >> 5] = wb;
    const MaxSum mine = block_scaled<NT>(MaxSum{m, s}, sh.red, kappa);
    float bound = sh.bound[0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w)
        bound = fminf(bound, sh.bound[w]);
    cluster_wait();
    if (tid < (int)cl.size)
        st_async_quad(map_rank(smem_u32(&sh.part[cl.rank]), tid), mine.m, mine.s, bound,
                      map_rank(smem_u32(&sh.xbar), tid));
    wait_or_flag(smem_u32(&sh.xbar), true, a.status);
    float M = sh.part[0].x;
    for (unsigned q = 0; q < cl.size; ++q) {
        M = fmaxf(M, sh.part[q].x);
        bound = fminf(bound, sh.part[q].z);
    }

    // Pass 2: the candidates.
    auto keep = [&](float z, int e) {
        if (z >= bound && z != -INFINITY) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < kCandCta)
                sh.list[at] = order_pair(order_key(z), (uint32_t)(v0 + (e - sl.pad)));
        }
    };
    for (int g = tid; g < sl.ng; g += NT) {
        float z[8];
        load8<InT>(slab, g, z);
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 8; ++i)
            top = fmaxf(top, z[i]);
        if (top >= bound)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                keep(z[i], 8 * g + i);
    }
    cluster_sync_data();
    // The first CTA gathers the lists, in its slab.
    mass_t *all = reinterpret_cast<mass_t *>(slab);
    int n = 0;
    bool fits = true;
    if (cl.rank == 0) {
        const cg::cluster_group cluster = cg::this_cluster();
        if (tid < (int)cl.size)
            sh.count[tid] = *cluster.map_shared_rank(&sh.n, tid);
        __syncthreads();
        for (unsigned q = 0; q < cl.size; ++q) {
            const int c = sh.count[q];
            fits = fits && c <= kCandCta && n + c <= kCand;
            if (fits) {
                const mass_t *from = cluster.map_shared_rank(&sh.list[0], (int)q);
                for (int i = tid; i < c; i += NT)
                    all[n + i] = from[i];
                n += c;
            }
        }
    }
    cluster_sync_data();  // no CTA leaves while its list is read; the list is whole
    if (cl.rank != 0)
        return;
    float S = 0.0f;
    for (unsigned q = 0; q < cl.size; ++q)
        S += sh.part[q].y * ex2_ftz((sh.part[q].x - M) * kappa);
    if (tid == 0)
        grid_wait();
    __syncthreads();
    if (!(S > 0.0f && S < INFINITY) || M == INFINITY) {
        fill_row(a, t, NAN, NAN);
        if (tid == 0)
            set_status(a.status, kStatusBadInput);
        return;
    }
    if (!fits) {
        if (tid == 0)
            a.ids_out[t * a.K] = kTodo;
        return;
    }
    const float ls = logf(S), lsl = log_residual(S, ls);
    for (int i = tid; i < n; i += NT) {
        const mass_t p = all[i];
        int before = 0;
        for (int j = 0; j < n; ++j)
            before += all[j] > p;
        if (before < a.K) {
            float l, e;
            const float x = scaled_diff(key_value((uint32_t)(p >> 32)), M, a.sc, l);
            const float u = two_sum(x, -ls, e);
            a.ids_out[t * a.K + before] = (int32_t)(0xffffffffu - (uint32_t)p);
            a.lp_out[t * a.K + before] = u + (e + l - lsl);
        }
    }
    for (int i = n + tid; i < a.K; i += NT) {
        a.ids_out[t * a.K + i] = -1;
        a.lp_out[t * a.K + i] = -INFINITY;
    }
    if (tid == 0 && a.lse_out) {
        float e;
        const float p = M * a.sc.hi, pl = isfinite(p) ? fmaf(M, a.sc.hi, -p) + M * a.sc.lo : 0.0f;
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

template <typename InT, int NT>
cudaError_t launch_fast(const TopkArgs &a, const RowPlan &p, cudaStream_t s)
{
    auto kern = cis_topk_kernel<InT, NT>;
    size_t smem = slab_bytes(p.slice, sizeof(InT));
    if (smem < kCand * sizeof(mass_t) + 128)
        smem = kCand * sizeof(mass_t) + 128;
    const cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * p.cs), 1, 1);
    cfg.blockDim = dim3(NT, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int warps = p.cs * (NT / 32);
    return cudaLaunchKernelEx(&cfg, kern, a, p.slice, (a.K + warps - 1) / warps);
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
    const RowPlan p = row_plan(a.V, (int)sizeof(InT));
    if (p.cs == 0 || a.T * kMaxCluster > 0x7fffffffLL)
        return launch_exact<InT>(a, true, s);
    const cudaError_t e = p.nt == 128 ? launch_fast<InT, 128>(a, p, s)
                                      : launch_fast<InT, 256>(a, p, s);
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
