// cis_logits.cu -- logits from 8-bit hidden states and weights (cis_lmhead_logits), sm_103a.
//
//   z_tv = (sum_h x_th w_vh) xs_t ws_v,   x, w e4m3, a scale a row of each; the sum in fp32.
//
// The weights are the tensor cores' M operand (128 vocabulary entries a tile, one a TMEM lane),
// the tokens the N operand (up to 256 a tile): a decoding step's few tokens make a narrow N, down
// to 16 columns, and no work is spent on rows that are not there.  Both operands lie K-major and
// arrive by TMA in blocks of 128 bytes along H (128-byte swizzle, zeros behind H, V and T).
// Persistent CTAs take tiles u, u + grid, ...: the token tiles of one vocabulary tile are
// neighbours, so that its weights come from HBM once.  Warp 0 loads, warp 1 issues tcgen05.mma
// (kind::f8f6f4, four K = 32 steps a block) into one of two TMEM accumulators, warps 2..9 take the
// other one to memory: a warp's 32 lanes are 32 neighbouring entries of one token's row.
//
// All waits are bounded: one that runs out sets CIS_ERR_DEVICE_TIMEOUT, and the CTA drains its own
// loads and MMAs and runs to its end.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <mutex>

#include "cis_kernels.h"
#include "cis_nvtx.h"
#include "cis_tc.cuh"

namespace cis {
namespace {

constexpr int kM = 128;           // vocabulary entries of a tile
constexpr int kMaxN = 256;        // tokens of a tile, at most
constexpr int kBlock = 128;       // bytes of a row that a stage holds
constexpr int kStageA = kM * kBlock;
constexpr int kMaxStages = 12;
constexpr int kRingBytes = 220 * 1024;
constexpr int kEpiWarps = 8;      // two per TMEM lane quadrant
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr size_t kSmem = kRingBytes + 1024;  // (the ring starts on 1024 bytes)

struct LogitsArgs {
    const float *xs, *ws;
    void *out;
    int64_t ld;
    int T, V;
    int nM, nN, nK;    // tiles and blocks
    int N;             // tokens of a tile
    int stages;
    uint32_t cols;     // TMEM columns
    int pairs;         // bf16: two entries a store
    int32_t *status;
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t accfull[2], accempty[2];
    uint64_t done;
    uint32_t tmem;
    int aborted;
};

// A wait that runs out marks the CTA and the call's status word: the roles then stop waiting.
struct Guard {
    volatile int *local;
    int32_t *status;
    __device__ __forceinline__ bool on() const { return *local != 0; }
    __device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity) const
    {
        if (tc::bar_try(bar, parity))
            return true;
        if (*local)
            return false;
        if (!tc::bar_wait(bar, parity)) {
            *local = 1;
            set_status(status, kStatusTimeout);
            return false;
        }
        return true;
    }
};

struct Stage {
    int i = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int n)
    {
        if (++i == n) {
            i = 0;
            phase ^= 1;
        }
    }
};

// D[tmem] (+)= A[smem] B[smem]^T: e4m3 operands, fp32 accumulator.
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                         bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate));
}
// Instruction descriptor: D fp32 (1 at bit 4), A and B e4m3 (0), both K-major, M x N.
__device__ __forceinline__ uint32_t idesc_e4m3(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// 16 consecutive columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
        "%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i)
        v[i] = __uint_as_float(r[i]);
}

// 16 tokens from t0 on of this lane's entry v.
template <typename OutT>
__device__ __forceinline__ void store_chunk(const LogitsArgs &g, const float (&acc)[16], int t0,
                                            int v, float ws, int lane)
{
    const int n = g.T - t0 < 16 ? g.T - t0 : 16;
    const float mine = lane < n ? __ldg(g.xs + t0 + lane) : 0.0f;
    float z[16];
#pragma unroll
    for (int c = 0; c < 16; ++c)
        z[c] = acc[c] * __shfl_sync(0xffffffffu, mine, c) * ws;
    if constexpr (sizeof(OutT) == 4) {
        float *p = static_cast<float *>(g.out) + (int64_t)t0 * g.ld + v;
        if (v < g.V)
#pragma unroll
            for (int c = 0; c < 16; ++c)
                if (c < n)
                    p[(int64_t)c * g.ld] = z[c];
    } else if (g.pairs) {
        // neighbouring lanes exchange one of two tokens: each stores two entries of one row
        const bool odd = lane & 1;
        __nv_bfloat16 *p = static_cast<__nv_bfloat16 *>(g.out) + (int64_t)(t0 + odd) * g.ld +
                           (v - odd);
#pragma unroll
        for (int c = 0; c < 16; c += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, odd ? z[c] : z[c + 1], 1);
            const __nv_bfloat162 w =
                odd ? __floats2bfloat162_rn(got, z[c + 1]) : __floats2bfloat162_rn(z[c], got);
            if (c + odd < n && v - odd < g.V)  // (V is even)
                *reinterpret_cast<__nv_bfloat162 *>(p + (int64_t)c * g.ld) = w;
        }
    } else {
        __nv_bfloat16 *p = static_cast<__nv_bfloat16 *>(g.out) + (int64_t)t0 * g.ld + v;
        if (v < g.V)
#pragma unroll
            for (int c = 0; c < 16; ++c)
                if (c < n)
                    p[(int64_t)c * g.ld] = __float2bfloat16_rn(z[c]);
    }
}

template <typename OutT>
__global__ void __launch_bounds__(kThreads, 1)
    cis_lmhead_logits_kernel(const __grid_constant__ CUtensorMap tmW,
                             const __grid_constant__ CUtensorMap tmX, const LogitsArgs g)
{
    extern __shared__ __align__(1024) uint8_t dsm[];
    uint8_t *ring = dsm + ((1024 - (tc::smem_addr(dsm) & 1023)) & 1023);
    __shared__ __align__(8) Shared sh;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int units = g.nM * g.nN, bytes = kStageA + g.N * kBlock;
    if (threadIdx.x == 0) {
        sh.aborted = 0;
        for (int s = 0; s < g.stages; ++s) {
            tc::bar_init(&sh.full[s], 1);
            tc::bar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc::bar_init(&sh.accfull[b], 1);
            tc::bar_init(&sh.accempty[b], kEpiWarps);
        }
        tc::bar_init(&sh.done, 1);
        tc::bar_init_fence();
    }
    if (warp == 1)
        tc::tmem_alloc(&sh.tmem, g.cols);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = sh.tmem, half = g.cols / 2;
    const Guard guard{&sh.aborted, g.status};

    if (warp == 0) {
        if (lane == 0) {
            Stage p;
            uint32_t used = 0, last = 0;
            for (int u = blockIdx.x; u < units && !guard.on(); u += gridDim.x) {
                const int v0 = u / g.nN * kM, t0 = u % g.nN * g.N;
                for (int k = 0; k < g.nK; ++k) {
                    if (!guard.wait(&sh.empty[p.i], p.phase ^ 1))
                        break;
                    tc::bar_expect_tx(&sh.full[p.i], (uint32_t)bytes);
                    used |= 1u << p.i;
                    last = (last & ~(1u << p.i)) | (p.phase << p.i);
                    uint8_t *st = ring + p.i * bytes;
                    tc::tma_load_2d(st, &tmW, k * kBlock, v0, &sh.full[p.i]);
                    tc::tma_load_2d(st + kStageA, &tmX, k * kBlock, t0, &sh.full[p.i]);
                    p.next(g.stages);
                }
            }
            // no load may still be landing when the CTA leaves
            for (int s = 0; s < g.stages; ++s)
                if (used & (1u << s))
                    tc::bar_wait(&sh.full[s], (last >> s) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            Stage p;
            const uint32_t id = idesc_e4m3(kM, g.N), s0 = tc::smem_addr(ring);
            int i = 0;
            for (int u = blockIdx.x; u < units && !guard.on(); u += gridDim.x, ++i) {
                const int acc = i & 1;
                guard.wait(&sh.accempty[acc], ((i >> 1) & 1) ^ 1);
                tc::fence_after_sync();
                const uint32_t d = tmem + acc * half;
                for (int k = 0; k < g.nK; ++k) {
                    if (!guard.wait(&sh.full[p.i], p.phase))
                        break;
                    tc::fence_after_sync();
                    const uint64_t a = tc::desc_sw128(s0 + p.i * bytes);
                    const uint64_t b = tc::desc_sw128(s0 + p.i * bytes + kStageA);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // 32 bytes a step
                        mma_e4m3(d, a + 2 * kk, b + 2 * kk, id, (k | kk) != 0);
                    tc::mma_commit(&sh.empty[p.i]);
                    p.next(g.stages);
                }
                tc::mma_commit(&sh.accfull[acc]);
            }
            // every MMA is done before TMEM is released
            tc::mma_commit(&sh.done);
            tc::bar_wait(&sh.done, 0);
        }
    } else {
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int i = 0;
        for (int u = blockIdx.x; u < units; u += gridDim.x, ++i) {
            const int acc = i & 1;
            const int v = u / g.nN * kM + quad * 32 + lane, t0 = u % g.nN * g.N;
            const float ws = v < g.V ? __ldg(g.ws + v) : 0.0f;
            bool ok = guard.wait(&sh.accfull[acc], (i >> 1) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok)
                break;
            tc::fence_after_sync();
            for (int c = 16 * part; c < g.N && t0 + c < g.T; c += 32) {
                float a[16];
                tmem_ld16(tmem + lanes + acc * half + c, a);
                store_chunk<OutT>(g, a, t0 + c, v, ws, lane);
            }
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0)
                tc::bar_arrive(&sh.accempty[acc]);
        }
    }
    __syncwarp();
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, g.cols);
    }
}

PFN_cuTensorMapEncodeTiled_v12000 tile_encoder()
{
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        cudaDriverEntryPointQueryResult q;
        void *f = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000,
                                             cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    });
    return fn;
}
// Rows of H bytes, boxes of 128 bytes x `box` rows.
bool byte_map(CUtensorMap *m, const void *ptr, int64_t H, int64_t rows, int box)
{
    auto enc = tile_encoder();
    if (!enc)
        return false;
    const cuuint64_t dims[2] = {(cuuint64_t)H, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)H};
    const cuuint32_t boxes[2] = {(cuuint32_t)kBlock, (cuuint32_t)box};
    const cuuint32_t es[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, boxes,
               es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename OutT>
cudaError_t launch(const CUtensorMap &w, const CUtensorMap &x, const LogitsArgs &g, cudaStream_t s)
{
    auto kern = cis_lmhead_logits_kernel<OutT>;
    int dev = 0, sms = 0;
    cudaError_t e = allow_smem(kern, kSmem);
    if (e == cudaSuccess)
        e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess)
        return e;
    const int64_t units = (int64_t)g.nM * g.nN;
    kern<<<(unsigned)(units < sms ? units : sms), kThreads, kSmem, s>>>(w, x, g);
    return cudaGetLastError();
}

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" CIS_API cis_status_t cis_lmhead_logits(const void *hidden, const float *hidden_scale,
                                                  const void *weight, const float *weight_scale,
                                                  int64_t T, int64_t H, int64_t V, void *logits,
                                                  int32_t logits_dtype, int64_t ld,
                                                  int32_t *dev_status, void *stream)
{
    NvtxRange nvtx_range("cis_lmhead_logits");
    if (!row_args_ok(logits, logits_dtype, T, V, ld) || H <= 0 || H > 0x7fffffffLL ||
        !aligned4(hidden_scale, weight_scale, dev_status))
        return CIS_ERR_INVALID_ARG;
    if (T == 0)
        return CIS_OK;
    if (hidden == nullptr || hidden_scale == nullptr || weight == nullptr ||
        weight_scale == nullptr || logits == nullptr)
        return CIS_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(hidden) | reinterpret_cast<uintptr_t>(weight)) & 15) != 0)
        return CIS_ERR_INVALID_ARG;
    if (H % 16 != 0)
        return CIS_ERR_UNSUPPORTED;
    LogitsArgs g = {};
    g.xs = hidden_scale;
    g.ws = weight_scale;
    g.out = logits;
    g.ld = ld;
    g.T = (int)T;
    g.V = (int)V;
    const int64_t nN = (T + kMaxN - 1) / kMaxN, nM = (V + kM - 1) / kM;
    g.N = (int)(((T + nN - 1) / nN + 15) / 16 * 16);
    if (nN * nM > 0x7fffffffLL)
        return CIS_ERR_UNSUPPORTED;
    g.nN = (int)nN;
    g.nM = (int)nM;
    g.nK = (int)((H + kBlock - 1) / kBlock);
    const int fit = kRingBytes / (kStageA + g.N * kBlock);
    g.stages = fit < kMaxStages ? fit : kMaxStages;
    g.cols = 32;
    while (g.cols < 2u * g.N)
        g.cols *= 2;
    g.pairs = logits_dtype == CIS_BF16 && V % 2 == 0 && ld % 2 == 0 &&
              (reinterpret_cast<uintptr_t>(logits) & 3) == 0;
    g.status = dev_status;
    CUtensorMap mw, mx;
    if (!byte_map(&mw, weight, H, V, kM) || !byte_map(&mx, hidden, H, T, g.N))
        return CIS_ERR_UNSUPPORTED;
    const cudaError_t e = logits_dtype == CIS_BF16
                              ? launch<__nv_bfloat16>(mw, mx, g, (cudaStream_t)stream)
                              : launch<float>(mw, mx, g, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
