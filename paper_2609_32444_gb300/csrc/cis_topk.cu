// cis_topk.cu -- the K most likely tokens of each row with their log-probabilities
// (cis_topk_logprobs): a teacher's lists.
//
// A row's order is (z descending, index ascending); lp_k = z_k / tau - log sum e^{z / tau}.
//
// The row is read once (cis_rowpass.cuh); the first CTA sorts the row's candidates.  A row
// with more candidates than fit is left to the exact kernel, which follows: long runs of equal
// entries, a warp or a CTA whose stretch of ids is unlikely as a whole (the bound is the least of
// theirs), and, for K near 256, rows of a CTA of 64 threads (V=4000 in bf16: every row).
//
// Bound: HBM and instruction issue (64%) for many long rows, six CTAs an SM: T=8192, V=151936,
// K=64 takes 440 us, 5.7 TB/s.  Short rows and few rows wait for a row's last steps (the bound,
// the candidates, their order), in which a CTA loads next to nothing: T=2048, V=32003 fp32,
// K=128 65 us, 3.1 TB/s of the rows that are read; T=24, V=151936, K=20 16 us.  With the rows left
// it is the exact kernel, 3 us a row: the first of these takes 1.9 ms where the last eighth of the
// ids is half a deviation lower, and 25 ms where it is a whole one.  Slices of the row
// in the shared memory of four CTAs, read three times, took 1336 us at the first of these sizes.
#include <math.h>

#include "cis_nvtx.h"
#include "cis_rowpass.cuh"

namespace cis {
namespace {

__device__ __forceinline__ void fill_row(const TopkArgs &a, int64_t t, float lp, float lse)
{
    for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
        a.ids_out[t * a.K + k] = -1;
        a.lp_out[t * a.K + k] = lp;
    }
    if (threadIdx.x == 0 && a.lse_out)
        a.lse_out[t] = lse;
}

constexpr int32_t kTodo = -2;  // in a row's first id: left to the exact kernel

// r = ceil(K / CTAs of the row); cap: items and candidates that fit, a power of two.  Dynamic
// shared memory: cap candidates, cap items, the batches' maxima (and, in their place, the
// candidates of all CTAs).
//
// kMin: CTAs an SM that the registers are to leave room for.  1 (56 registers) where no SM has
// more than three (T=24, V=151936, K=20: 21.4 us with a cold L2 against 23.0; T=39: 25.5 against
// 27.1), 6 (40) for long fp32 rows (T=2048, V=32003, K=128: 74 against 78), else the compiler's
// choice, 40 to 48 (T=8192, V=151936 bf16, K=64: 453 against 464 with 6; T=2048, V=32000 bf16,
// K=20: 70 against 79 with 1; T=150, V=32000 bf16, K=64, 600 CTAs: 25 against 29).
template <typename InT, int NT, int kB, int kMin>
__global__ void __launch_bounds__(NT, kMin)
    cis_topk_kernel(const __grid_constant__ TopkArgs a, unsigned cs, int r, int cap)
{
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    __shared__ PassShared<NT> sh;
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
    if (cs > 1)
        cluster_arrive_relaxed();  // waited for before the exchange
    if (tid == 0)
        sh.items = sh.n = 0;
    RowPass<InT, NT, kB> pass(reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V, rank, cs,
                              bmax);
    ExpAcc<false, true> acc;
    acc.k = a.sc.kappa;
    acc.h = a.sc.huge;
    pass.stream(
        true, [&](const Vec<InT> (&x)[kB], float mx) { take<false, kB>(acc, x, mx); },
        [&](float z) {
            acc.raise(z);
            if (acc.m != -INFINITY)
                acc.add_entry(z);
        });
    pass.bound_put(sh, r);
    MaxSumU o = block_exp<NT>(acc, sh.red);  // (its barriers)
    float bound = pass.bound_get(sh, r);
    if (cs > 1) {
        exchange(sh, rank, cs, o.m, bound, o.s, 0.0f);
        float M = sh.part[0][0], S = 0.0f;
        for (unsigned c = 0; c < cs; ++c) {
            M = fmaxf(M, sh.part[c][0]);
            bound = fminf(bound, sh.part[c][1]);
        }
        for (unsigned c = 0; c < cs; ++c)  // in rank order
            S += sh.part[c][2] * ex2_ftz((sh.part[c][0] - M) * a.sc.kappa);
        o.m = M;
        o.s = S;
    }
    const bool bad = !(o.s > 0.0f && o.s < INFINITY) || !(fabsf(o.m) < INFINITY);
    int n = pass.collect(sh, bound, list, items, cap);
    if (cs > 1) {
        mass_t *all = reinterpret_cast<mass_t *>(bmax);
        n = gather_lists<NT>(sh, rank, cs, list, n, all, cap);
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

// The rows left, exactly: a cluster per row reads it from memory once for each step.
template <typename InT>
__global__ void __launch_bounds__(kSelThreads, 2)
    cis_topk_exact_kernel(const __grid_constant__ TopkArgs a)
{
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    SelectShared<kSelThreads> &sh = *reinterpret_cast<SelectShared<kSelThreads> *>(dyn_smem);
    int turn = 0;
    if (threadIdx.x == 0)
        allow_next_grid();
    grid_wait();
    RowsLeft<kSelThreads> rows(sh, a.T, gridDim.x / kSelCluster, blockIdx.x / kSelCluster);
    for (;;) {
        const int64_t t = rows.next([&](int64_t i) { return a.ids_out[i * a.K] == kTodo; });
        if (t < 0)
            break;
        RowSelect<InT, kSelThreads> rs(sh, reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V,
                                       turn);
        uint32_t least;
        const uint32_t mk = rs.max_key(least);
        const float M = key_value(mk), bottom = key_value(least);
        const int K = (int)(a.K < a.V ? a.K : a.V);
        mass_t above, equal;
        bool parts;
        mass_t want = (mass_t)K;
        const uint32_t key =
            rs.select(want, (float)K, 0.0f, M - bottom > 1024.0f ? M - 64.0f : bottom, M,
                      [](float) { return 1.0f; }, [](float) { return (mass_t)1; }, above, equal,
                      parts);
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

template <typename InT, int NT, int kB, int kMin>
cudaError_t launch_fast(const TopkArgs &a, const PassPlan &p, cudaStream_t s)
{
    auto kern = cis_topk_kernel<InT, NT, kB, kMin>;
    // Short rows always fit, whatever their entries.  Up to 64 of a list leave some 100 candidates
    // (at T=8192, V=151936, K=64 room for 512 takes 435 us a call, for 1024 442), longer ones some
    // 200 to 450, and on uneven rows more (K=128 at V=32003 takes 65 us with either).
    const int cap = a.V <= 1024 ? 1024 : a.V <= 2048 ? 2048 : a.K <= 64 ? 512 : 1024;
    const size_t all = p.cs > 1 ? cap * sizeof(mass_t) : 0;
    const size_t smem =
        cap * (sizeof(mass_t) + sizeof(int)) + (p.maxima < all ? all : p.maxima);
    const cudaError_t e =
        allow_smem(kern, 2048 * (sizeof(mass_t) + sizeof(int)) + kMostMaxima);
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
    cfg.numAttrs = p.cs > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, a, (unsigned)p.cs, (a.K + p.cs - 1) / p.cs, cap);
}

// The exact kernel.
template <typename InT>
cudaError_t launch_exact(const TopkArgs &a, cudaStream_t s)
{
    constexpr size_t smem = sizeof(SelectShared<kSelThreads>);
    const cudaError_t e = allow_smem(cis_topk_exact_kernel<InT>, smem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    const int64_t groups = a.T < 38 ? a.T : 38;  // two CTAs an SM
    cfg.gridDim = dim3((unsigned)(groups * kSelCluster));
    cfg.blockDim = dim3(kSelThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kSelCluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, cis_topk_exact_kernel<InT>, a);
}

template <typename InT> cudaError_t launch_topk(const TopkArgs &a, cudaStream_t s)
{
    const PassPlan p = pass_plan(a.T, a.V, (int)sizeof(InT));
    if (a.T * p.cs > 0x7fffffffLL)
        return cudaErrorNotSupported;
    const bool few = a.T * p.cs <= 3 * 152;
    const cudaError_t e = p.nt == 64   ? launch_fast<InT, 64, 1, 0>(a, p, s)
                          : p.kb == 4 ? launch_fast<InT, 256, 4, sizeof(InT) == 2 ? 0 : 6>(a, p, s)
                          : few       ? launch_fast<InT, 256, 1, 1>(a, p, s)
                                      : launch_fast<InT, 256, 1, 0>(a, p, s);
    return e != cudaSuccess ? e : launch_exact<InT>(a, s);
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
        !temperature_ok(temperature) || !aligned4(ids_out, lp_out, lse_out, dev_status))
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
    return e == cudaSuccess ? CIS_OK
                            : (e == cudaErrorNotSupported ? CIS_ERR_UNSUPPORTED : CIS_ERR_CUDA);
}
