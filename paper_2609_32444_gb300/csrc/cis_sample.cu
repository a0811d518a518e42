// cis_sample.cu -- sampling from rows of logits with given uniform numbers
// (cis_sample_tokens).
//
// Per row, with s = z / tau and the order of the entries (z descending, index ascending),
// the kept set is a prefix of that order:
//   top_k   the first top_k entries;
//   top_p   of those, the smallest prefix whose mass is at least top_p of theirs;
//   min_p   of those, the entries with s_j >= s_max + log(min_p).
// The sample is the first entry, by index, whose running kept mass is above u times the kept
// mass.  Every decision is taken on masses in whole numbers (cis_select.cuh).
#include <math.h>

#include "cis_nvtx.h"
#include "cis_select.cuh"

namespace cis {
namespace {

constexpr int kSelThreads = 512;
constexpr int kSelCluster = 8;

__device__ inline RowSettings row_settings(const SampleArgs &a, int64_t t)
{
    RowSettings r;
    const float tau = a.temperature ? a.temperature[t] : 1.0f;
    r.u = a.u[t];
    r.top_k = a.top_k ? a.top_k[t] : 0;
    r.top_p = a.top_p ? a.top_p[t] : 1.0f;
    r.min_p = a.min_p ? a.min_p[t] : 0.0f;
    r.greedy = tau == 0.0f;
    r.ok = (r.greedy || (tau >= 1e-3f && tau <= 1e3f)) && r.u >= 0.0f && r.u < 1.0f &&
           r.top_p > 0.0f && r.top_p <= 1.0f && r.min_p >= 0.0f && r.min_p <= 1.0f;
    r.sc = device_scale(r.greedy || !r.ok ? 1.0f : tau);
    r.tau = r.greedy || !r.ok ? 1.0f : tau;
    return r;
}

__device__ __forceinline__ void write_row(const SampleArgs &a, int64_t t, int32_t id, float lp,
                                          float lps)
{
    a.ids_out[t] = id;
    if (a.lp_out) a.lp_out[t] = lp;
    if (a.lps_out) a.lps_out[t] = lps;
}

// Any row, exactly: a cluster per row reads it from memory (L2 after the first time) once
// for each step.
template <typename InT>
__global__ void __launch_bounds__(kSelThreads) cis_sample_exact_kernel(const SampleArgs a)
{
    __shared__ SelectShared<kSelThreads> sh;
    const unsigned group = blockIdx.x / kSelCluster, groups = gridDim.x / kSelCluster;
    int turn = 0;
    for (int64_t t = group; t < a.T; t += groups) {
        RowSelect<InT, kSelThreads> rs(sh, reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V,
                                       turn);
        const bool first = rs.rank == 0 && threadIdx.x == 0;
        if (a.mask && a.mask[t] == 0) {
            if (first)
                write_row(a, t, -1, 0.0f, 0.0f);
            continue;
        }
        const RowSettings rset = row_settings(a, t);
        bool bad;
        const uint32_t mk = rs.max_key(bad);
        if (bad || !rset.ok) {  // as every CTA of the cluster finds
            if (first) {
                write_row(a, t, -1, NAN, NAN);
                set_status(a.status, kStatusBadInput);
            }
            continue;
        }
        const float M = key_value(mk);
        const Scale &sc = rset.sc;
        Kept kept{0, 0};
        mass_t above, equal;
        const int64_t k = rset.greedy ? 1 : rset.top_k;
        if (k > 0 && k < a.V) {
            kept.key = rs.select((mass_t)k, [](float, uint32_t) { return (mass_t)1; }, above, equal);
            kept.ties = (mass_t)k - above;
        }
        mass_t gt, eq, gt0, eq0;
        rs.kept_mass(kept.key, M, sc, gt, eq, gt0, eq0);
        mass_t wkey = kept.ties ? fixed_mass(key_value(kept.key), M, sc) : 0;
        bool moved = false;
        if (rset.top_p < 1.0f && !rset.greedy) {
            const mass_t target =
                (mass_t)ceil((double)rset.top_p * (double)(gt + kept.ties * wkey));
            if (target <= gt) {
                const uint32_t floor_key = kept.key;
                kept.key = rs.select(
                    target,
                    [&](float z, uint32_t key) {
                        return key > floor_key ? fixed_mass(z, M, sc) : (mass_t)0;
                    },
                    above, equal);
                wkey = fixed_mass(key_value(kept.key), M, sc);
                kept.ties = (target - above + wkey - 1) / wkey;
                moved = true;
            } else if (wkey) {
                kept.ties = min(kept.ties, (target - gt + wkey - 1) / wkey);
            }
        }
        if (rset.min_p > 0.0f) {
            const uint32_t low = min_p_key(M, rset.tau, rset.min_p);
            if (kept.key < low) {
                kept = Kept{low - 1, 0};
                wkey = 0;
                moved = true;
            }
        }
        if (moved)
            rs.kept_mass(kept.key, M, sc, gt, eq, gt0, eq0);
        const mass_t Z = gt + min(eq, kept.ties) * wkey;
        const mass_t target = (mass_t)((double)rset.u * (double)Z);
        int64_t j = 0;
        const bool have =
            rs.locate(kept, wkey, min(target, Z - 1), gt0, eq0, M, sc, j);
        // the row's own log-probability: its mass at temperature 1
        mass_t raw = 0, none = 0, x, y;
        const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};
        rs.each([&](int64_t, float z) { raw += fixed_mass(z, M, one); });
        rs.cluster_sum(raw, none, x, y);
        if (have && threadIdx.x == 0) {
            const float z = to_f32(rs.row[j]);
            const double d = (double)z - (double)M;
            write_row(a, t, (int32_t)j, (float)(d - log(mass_value(raw))),
                      rset.greedy ? 0.0f
                                  : (float)(d / (double)rset.tau - log(mass_value(Z))));
        }
        __syncthreads();
    }
    cg::this_cluster().sync();  // no CTA leaves while a peer reads its shared memory
}

template <typename InT> cudaError_t launch_exact(const SampleArgs &a, cudaStream_t s)
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
    return cudaLaunchKernelEx(&cfg, cis_sample_exact_kernel<InT>, a);
}

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" CIS_API cis_status_t cis_sample_tokens(
    const void *logits, int32_t dtype, int64_t T, int64_t V, int64_t ld, const float *u,
    const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
    const uint8_t *mask, int32_t *ids_out, float *lp_out, float *lp_sampled_out,
    int32_t *dev_status, void *stream)
{
    NvtxRange nvtx_range("cis_sample_tokens");
    if (!row_args_ok(logits, dtype, T, V, ld))
        return CIS_ERR_INVALID_ARG;
    if (T == 0)
        return CIS_OK;
    if (logits == nullptr || u == nullptr || ids_out == nullptr)
        return CIS_ERR_INVALID_ARG;
    if (V > kMaxRowEntries)
        return CIS_ERR_UNSUPPORTED;
    SampleArgs a = {};
    a.logits = logits;
    a.T = T;
    a.V = V;
    a.ld = ld;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.mask = mask;
    a.ids_out = ids_out;
    a.lp_out = lp_out;
    a.lps_out = lp_sampled_out;
    a.status = dev_status;
    const cudaError_t e = dtype == CIS_BF16
                              ? launch_exact<__nv_bfloat16>(a, (cudaStream_t)stream)
                              : launch_exact<float>(a, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
