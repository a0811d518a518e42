// cis_topk.cu -- the K most likely tokens of each row with their log-probabilities
// (cis_topk_logprobs): a teacher's lists.
//
// A row's order is (z descending, index ascending); lp_k = z_k / tau - log sum e^{z / tau}.
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

// Any row, exactly: a cluster per row reads it from memory once for each step.
template <typename InT>
__global__ void __launch_bounds__(kSelThreads) cis_topk_exact_kernel(const TopkArgs a)
{
    __shared__ SelectShared<kSelThreads> sh;
    const unsigned group = blockIdx.x / kSelCluster, groups = gridDim.x / kSelCluster;
    int turn = 0;
    for (int64_t t = group; t < a.T; t += groups) {
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

template <typename InT> cudaError_t launch_exact(const TopkArgs &a, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    const int64_t groups = a.T < 76 ? a.T : 76;
    cfg.gridDim = dim3((unsigned)(groups * kSelCluster));
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kSelCluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cis_topk_exact_kernel<InT>, a);
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
                              ? launch_exact<__nv_bfloat16>(a, (cudaStream_t)stream)
                              : launch_exact<float>(a, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
