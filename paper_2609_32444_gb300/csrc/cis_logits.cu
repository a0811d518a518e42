// cis_logits.cu -- logits from 8-bit hidden states and weights (cis_lmhead_logits), sm_103a.
//
//   z_tv = (sum_h x_th w_vh) xs_t ws_v,   x, w e4m3, a scale a row of each; the sum in fp32.
//
// The weights are the tensor cores' M operand (128 vocabulary entries a CTA, one a TMEM lane),
// the tokens the N operand: a decoding step's few tokens make a narrow N, down to 16 columns, and no
// work is spent on rows that are not there.  Both operands lie K-major and arrive by TMA in blocks
// of 128 bytes along H (128-byte swizzle, zeros behind H, V and T).  Persistent CTAs take tiles u,
// u + grid, ...: the token tiles of one vocabulary tile are neighbours, so that its weights come from
// HBM once.  Warp 0 loads, warp 1 issues tcgen05.mma (kind::f8f6f4, four K = 32 steps a block) into
// accumulators in TMEM, warps 2..17 take finished ones to memory: a warp's 32 lanes are 32 neighbouring
// entries of one token's row.
//
// Few tokens (at most 64): a CTA by itself, bound by the weights' way from HBM.  More: two CTAs, on
// two SMs, share a tile of 256 entries (cta_group::2); each loads its 128 entries and half of the
// tokens, so that the tokens' way from L2 is halved.  257 to 320 tokens are one tile of 192 and 128
// tokens, so that the weights are read once: TMEM holds two accumulators of the one and one of the
// other.  (Two of 160 took 70 us where no logits were stored, T=320, H=2048, V=151936: as long as
// 192 would.)
//
// Bound: HBM up to 256 tokens (H=2048, V=151936: T=1 51 us a call, 6.1 TB/s; T=256 67 us, 5.8; T=320
// 77 us); with more, no unit by itself.  T=2048, a call and its kernel, and how busy the tensor cores
// and L2 are: V=32000 84 and 79 us, 79% and 47% (bf16 logits), 94 and 93 us, 67% and 46% (fp32);
// V=32003 4 to 5 us more.  What stores add is known by these times only.  All at 2070 MHz: after some
// 50 ms of such calls the power cap takes the clock to 1440 to 1600 MHz, and T=320 takes 87 us, T=2048,
// V=32000 98 and 109.
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

constexpr int kM = 128;           // vocabulary entries of a CTA's tile
constexpr int kMaxN = 256;        // tokens of an accumulator, at most
constexpr int kBlock = 128;       // bytes of a row that a stage holds
constexpr int kStageA = kM * kBlock;
constexpr int kMaxStages = 12;
constexpr int kRingBytes = 220 * 1024;
constexpr int kSlots = 3;         // the first accumulator in turn with another one, the second one
constexpr int kEpiWarps = 16;     // four per TMEM lane quadrant
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr size_t kSmem = kRingBytes + 1024;  // (the ring starts on 1024 bytes)

struct LogitsArgs {
    const float *xs, *ws;
    void *out;
    int64_t ld;
    int T, V;
    int nM, nN, nK;    // tiles and blocks
    int N0, N1, subs;  // tokens of a tile's accumulators, and how many it has
    int tile;          // tokens of a tile
    int stages;
    uint32_t cols;     // TMEM columns
    int pairs;         // bf16: two entries a store
    int xs16;          // xs starts on 16 bytes
    int32_t *status;
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t accfull[kSlots], accempty[kSlots];
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

// A place in a ring, and the parity of its phase.
struct Ring {
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

// The loading and the MMA warp run as warps, so that the compiler keeps their addresses and
// descriptors in uniform registers; `one` is true in the lane that issues.  (One lane by itself, its
// operands moved to uniform registers each time, held the tensor cores up while the other warps were
// busy: T=1, H=2048, V=151936 took 56 us for 51.)
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(p));
    return p;
}
// (every warp leaves its loop together: lanes that read the mark at different times would else wait for
// one another in different places)
__device__ __forceinline__ bool all(bool x) { return __all_sync(0xffffffffu, x); }

// The leader's (rank 0) barrier at this offset, as a cluster address.
__device__ __forceinline__ uint32_t leader_bar(uint64_t *bar)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(tc::smem_addr(bar)));
    return a;
}
// An arrival there.  (Not a release at the cluster's scope: that waits for the stores of the warp's
// logits, 1 to 2 us, and only TMEM is handed over.)
__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes, uint32_t one)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t"
                 "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
                 "r"(bytes), "r"(one)
                 : "memory");
}
// A box into this CTA's shared memory; kPair: it completes on a barrier of the pair's leader.
template <bool kPair>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y,
                                         uint32_t bar, uint32_t one)
{
    if constexpr (kPair)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
            "@p cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global"
            ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar), "r"(one)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
            "@p cp.async.bulk.tensor.2d.shared::cluster.global"
            ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar), "r"(one)
            : "memory");
}

// D[tmem] (+)= A[smem] B[smem]^T: e4m3 operands, fp32 accumulator.  kPair: both CTAs' halves.
template <bool kPair>
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                         bool accumulate, uint32_t one)
{
    if constexpr (kPair)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(one));
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate), "r"(one));
}
// Arrives once every MMA issued so far is done, in both CTAs of a pair.
template <bool kPair> __device__ __forceinline__ void commit(uint32_t bar, uint32_t one)
{
    if constexpr (kPair)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t"
            "@p tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster"
            ".multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar),
            "h"((uint16_t)3), "r"(one)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t"
            "@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
            ::"r"(bar), "r"(one)
            : "memory");
}
template <bool kPair> __device__ __forceinline__ void alloc(uint32_t *dst, uint32_t cols)
{
    if constexpr (kPair) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         tc::smem_addr(dst)),
                     "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tc::tmem_alloc(dst, cols);
    }
}
template <bool kPair> __device__ __forceinline__ void dealloc(uint32_t taddr, uint32_t cols)
{
    if constexpr (kPair)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr),
                     "r"(cols)
                     : "memory");
    else
        tc::tmem_dealloc(taddr, cols);
}
// Instruction descriptor: D fp32 (1 at bit 4), A and B e4m3 (0), both K-major, M x N.
__device__ __forceinline__ uint32_t idesc_e4m3(int M, int N)
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// 8 consecutive columns of this thread's TMEM lane, on their way until tmem_wait.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                   "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
}
// (the registers pass through it, so that nothing that reads them comes before it)
template <int G> __device__ __forceinline__ void tmem_wait(uint32_t (&r)[G][8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < G; ++i)
        asm volatile("" : "+r"(r[i][0]), "+r"(r[i][1]), "+r"(r[i][2]), "+r"(r[i][3]), "+r"(r[i][4]),
                          "+r"(r[i][5]), "+r"(r[i][6]), "+r"(r[i][7]));
}

// 8 tokens from t0 on of this lane's entry, v0 + at (v0 the tile's first).  kFull: all 8 are there.
template <typename OutT, bool kFull>
__device__ __forceinline__ void store_group(const LogitsArgs &g, const uint32_t (&acc)[8], int t0,
                                            int v0, int at, float ws)
{
    const int n = kFull ? 8 : g.T - t0;
    float z[8];
#pragma unroll
    for (int c = 0; c < 8; c += 4) {
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (g.xs16 && c + 4 <= n) {
            x = __ldg(reinterpret_cast<const float4 *>(g.xs + t0 + c));
        } else {
            if (c < n) x.x = __ldg(g.xs + t0 + c);
            if (c + 1 < n) x.y = __ldg(g.xs + t0 + c + 1);
            if (c + 2 < n) x.z = __ldg(g.xs + t0 + c + 2);
            if (c + 3 < n) x.w = __ldg(g.xs + t0 + c + 3);
        }
        z[c] = __uint_as_float(acc[c]) * x.x * ws;
        z[c + 1] = __uint_as_float(acc[c + 1]) * x.y * ws;
        z[c + 2] = __uint_as_float(acc[c + 2]) * x.z * ws;
        z[c + 3] = __uint_as_float(acc[c + 3]) * x.w * ws;
    }
    // (a row's address is the warp's; a lane has its offset)
    OutT *row = static_cast<OutT *>(g.out) + (int64_t)t0 * g.ld + v0;
    if constexpr (sizeof(OutT) == 4) {
        if (v0 + at < g.V)
#pragma unroll
            for (int c = 0; c < 8; ++c, row += g.ld)
                if (kFull || c < n)
                    row[at] = z[c];
    } else if (g.pairs) {
        // neighbouring lanes exchange one of two tokens: each stores two entries of one row
        const bool odd = at & 1;
        const bool in = v0 + at - odd < g.V;  // (V is even)
        OutT *mine = row + (odd ? g.ld : 0) + (at - odd);
#pragma unroll
        for (int c = 0; c < 8; c += 2, mine += 2 * g.ld) {
            const float got = __shfl_xor_sync(0xffffffffu, odd ? z[c] : z[c + 1], 1);
            const __nv_bfloat162 w = __floats2bfloat162_rn(odd ? got : z[c], odd ? z[c + 1] : got);
            if (in && (kFull || c + odd < n))
                *reinterpret_cast<__nv_bfloat162 *>(mine) = w;
        }
    } else {
        if (v0 + at < g.V)
#pragma unroll
            for (int c = 0; c < 8; ++c, row += g.ld)
                if (kFull || c < n)
                    row[at] = __float2bfloat16_rn(z[c]);
    }
}

template <typename OutT, bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
    cis_lmhead_logits_kernel(const __grid_constant__ CUtensorMap tmW,
                             const __grid_constant__ CUtensorMap tmX,
                             const __grid_constant__ CUtensorMap tmX2, const LogitsArgs g)
{
    extern __shared__ __align__(1024) uint8_t dsm[];
    uint8_t *ring = dsm + ((1024 - (tc::smem_addr(dsm) & 1023)) & 1023);
    __shared__ __align__(8) Shared sh;
    constexpr int kCtas = kPair ? 2 : 1;

    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = kPair ? (int)tc::cluster_ctarank() : 0;
    const int units = g.nM * g.nN, first = blockIdx.x / kCtas, step = gridDim.x / kCtas;
    // a stage: this CTA's entries, and its part of each accumulator's tokens
    const int rows0 = g.N0 / kCtas, rows1 = g.N1 / kCtas;
    const int second = kStageA + rows0 * kBlock, bytes = second + rows1 * kBlock;
    if (threadIdx.x == 0) {
        sh.aborted = 0;
        for (int s = 0; s < g.stages; ++s) {
            tc::bar_init(&sh.full[s], 1);
            tc::bar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < kSlots; ++b) {
            tc::bar_init(&sh.accfull[b], 1);
            tc::bar_init(&sh.accempty[b], kCtas * kEpiWarps);
        }
        tc::bar_init(&sh.done, 1);
        tc::bar_init_fence();
    }
    if (warp == 1)
        alloc<kPair>(&sh.tmem, g.cols);
    tc::fence_before_sync();
    __syncthreads();
    if (kPair)
        tc::cluster_sync();  // the peer's barriers exist before anything signals them
    tc::fence_after_sync();
    const uint32_t tmem = sh.tmem;
    const Guard guard{&sh.aborted, g.status};

    const uint32_t s0 = tc::smem_addr(ring);
    if (warp == 0) {
        const uint32_t one = elect_one();
        Ring p;
        uint32_t used = 0, last = 0;
        for (int u = first; u < units && !all(guard.on()); u += step) {
            const int v0 = (u / g.nN * kCtas + rank) * kM, t0 = u % g.nN * g.tile;
            for (int k = 0; k < g.nK; ++k) {
                if (!all(guard.wait(&sh.empty[p.i], p.phase ^ 1)))
                    break;
                const uint32_t st = s0 + p.i * bytes, own = tc::smem_addr(&sh.full[p.i]);
                const uint32_t full = kPair ? leader_bar(&sh.full[p.i]) : own;
                if (rank == 0)
                    expect_tx(own, (uint32_t)(kCtas * bytes), one);
                used |= 1u << p.i;
                last = (last & ~(1u << p.i)) | (p.phase << p.i);
                load_box<kPair>(st, &tmW, k * kBlock, v0, full, one);
                load_box<kPair>(st + kStageA, &tmX, k * kBlock, t0 + rank * rows0, full, one);
                if (kPair && g.subs > 1)
                    load_box<kPair>(st + second, &tmX2, k * kBlock, t0 + g.N0 + rank * rows1, full,
                                    one);
                p.next(g.stages);
            }
        }
        // no load may still be landing when the CTA leaves (a pair's both CTAs' loads complete on
        // the leader's barriers, and the other CTA leaves after it)
        if (rank == 0)
            for (int s = 0; s < g.stages; ++s)
                if (used & (1u << s))
                    tc::bar_wait(&sh.full[s], (last >> s) & 1);
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t one = elect_one();
            const uint32_t id0 = idesc_e4m3(kM * kCtas, g.N0), id1 = idesc_e4m3(kM * kCtas, g.N1);
            const uint64_t a0 = tc::desc_sw128(s0), b0 = tc::desc_sw128(s0 + kStageA);
            const uint64_t c0 = tc::desc_sw128(s0 + second);
            Ring p, acc;
            uint32_t turn = 0;  // of the second accumulator
            for (int u = first; u < units && !all(guard.on()); u += step) {
                const uint32_t d0 = tmem + acc.i * g.N0, d1 = tmem + 2 * g.N0;
                guard.wait(&sh.accempty[acc.i], acc.phase ^ 1);
                if (kPair && g.subs > 1)
                    guard.wait(&sh.accempty[2], turn ^ 1);
                __syncwarp();
                tc::fence_after_sync();
                for (int k = 0; k < g.nK; ++k) {
                    if (!all(guard.wait(&sh.full[p.i], p.phase)))
                        break;
                    tc::fence_after_sync();
                    // (a start address is in the descriptor's low bits, in units of 16 bytes)
                    const uint64_t so = (uint64_t)(uint32_t)(p.i * bytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // 32 bytes a step
                        mma_e4m3<kPair>(d0, a0 + so + 2 * kk, b0 + so + 2 * kk, id0,
                                        (k | kk) != 0, one);
                    if (kPair && g.subs > 1) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_e4m3<kPair>(d1, a0 + so + 2 * kk, c0 + so + 2 * kk, id1,
                                            (k | kk) != 0, one);
                    }
                    commit<kPair>(tc::smem_addr(&sh.empty[p.i]), one);
                    p.next(g.stages);
                }
                commit<kPair>(tc::smem_addr(&sh.accfull[acc.i]), one);
                acc.next(2);
                if (kPair && g.subs > 1) {
                    commit<kPair>(tc::smem_addr(&sh.accfull[2]), one);
                    turn ^= 1;
                }
            }
            commit<kPair>(tc::smem_addr(&sh.done), one);
        }
        tc::bar_wait(&sh.done, 0);  // every MMA is done before TMEM is released
    } else {
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        Ring acc;
        uint32_t turn = 0;
        for (int u = first; u < units && !all(guard.on()); u += step) {
            const int v0 = (u / g.nN * kCtas + rank) * kM, at = quad * 32 + lane;
            const float ws = v0 + at < g.V ? __ldg(g.ws + v0 + at) : 0.0f;
            // the second accumulator first: the MMAs wait for it
            for (int i = g.subs - 1; i >= 0; --i) {
                const int t0 = u % g.nN * g.tile + (i ? g.N0 : 0), slot = i ? 2 : acc.i;
                const uint32_t phase = i ? turn : acc.phase;
                if (!__all_sync(0xffffffffu, guard.wait(&sh.accfull[slot], phase)))
                    break;
                tc::fence_after_sync();
                // all of the warp's columns, groups of 8, into registers; then the accumulator is
                // free, and the stores hold up nothing
                constexpr int kParts = kEpiWarps / 4, kGroups = kMaxN / 8 / kParts;
                uint32_t r[kGroups][8];
                const int groups = min((i ? g.N1 : g.N0), g.T - t0);
                const uint32_t from = tmem + lanes + slot * g.N0;
#pragma unroll
                for (int j = 0; j < kGroups; ++j)
                    if (8 * (part + kParts * j) < groups)
                        tmem_ld8(from + 8 * (part + kParts * j), r[j]);
                tmem_wait(r);
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (kPair)
                        arrive_cluster(leader_bar(&sh.accempty[slot]));
                    else
                        tc::bar_arrive(&sh.accempty[slot]);
                }
#pragma unroll
                for (int j = 0; j < kGroups; ++j) {
                    const int c = 8 * (part + kParts * j);
                    if (c + 8 <= groups)
                        store_group<OutT, true>(g, r[j], t0 + c, v0, at, ws);
                    else if (c < groups)
                        store_group<OutT, false>(g, r[j], t0 + c, v0, at, ws);
                }
                if (i)
                    turn ^= 1;
                else
                    acc.next(2);
            }
        }
    }
    __syncwarp();
    tc::fence_before_sync();
    __syncthreads();
    if (kPair) {
        tc::cluster_sync();
        // after a wait ran out the peer may have issued loads that the leader no longer waits for:
        // give them time to land
        if (sh.aborted && threadIdx.x == 0) {
            const long long t0 = clock64();
            while (clock64() - t0 < (1ll << 20)) {
            }
        }
        __syncthreads();
    }
    if (warp == 1) {
        tc::fence_after_sync();
        dealloc<kPair>(tmem, g.cols);
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

template <typename OutT, bool kPair>
cudaError_t launch(const CUtensorMap &w, const CUtensorMap &x, const CUtensorMap &x2,
                   const LogitsArgs &g, cudaStream_t s)
{
    auto kern = cis_lmhead_logits_kernel<OutT, kPair>;
    int dev = 0, sms = 0;
    cudaError_t e = allow_smem(kern, kSmem);
    if (e == cudaSuccess)
        e = cudaGetDevice(&dev);
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess)
        return e;
    constexpr int kCtas = kPair ? 2 : 1;
    const int64_t units = (int64_t)g.nM * g.nN;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(kCtas * (units < sms / kCtas ? units : sms / kCtas)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCtas;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kPair ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kern, w, x, x2, g);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// From how many tokens on two CTAs share a tile.
constexpr int64_t kPairTokens = 65;
// One tile of two accumulators, 192 tokens and the rest.
constexpr int64_t kFirst = 192, kTwoSubs = 320;

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
    const bool pair = T >= kPairTokens;
    const int ctas = pair ? 2 : 1, step = 16 * ctas;
    g.subs = pair && T > kMaxN && T <= kTwoSubs ? 2 : 1;
    const int64_t nN = g.subs == 2 ? 1 : (T + kMaxN - 1) / kMaxN;
    auto up = [&](int64_t n) { return (int)((n + step - 1) / step * step); };
    g.N0 = g.subs == 2 ? (int)kFirst : up((T + nN - 1) / nN);
    g.N1 = g.subs == 2 ? up(T - kFirst) : 0;
    g.tile = g.N0 + g.N1;
    const int64_t nM = (V + kM * ctas - 1) / (kM * ctas);
    if (nN * nM > 0x7fffffffLL)
        return CIS_ERR_UNSUPPORTED;
    g.nN = (int)nN;
    g.nM = (int)nM;
    g.nK = (int)((H + kBlock - 1) / kBlock);
    const int fit = kRingBytes / (kStageA + g.tile / ctas * kBlock);
    g.stages = fit < kMaxStages ? fit : kMaxStages;
    g.cols = 32;
    while (g.cols < (uint32_t)(2 * g.N0 + g.N1))
        g.cols *= 2;
    g.xs16 = (reinterpret_cast<uintptr_t>(hidden_scale) & 15) == 0;
    g.pairs = logits_dtype == CIS_BF16 && V % 2 == 0 && ld % 2 == 0 &&
              (reinterpret_cast<uintptr_t>(logits) & 3) == 0;
    g.status = dev_status;
    CUtensorMap mw, mx, mx2;
    if (!byte_map(&mw, weight, H, V, kM) || !byte_map(&mx, hidden, H, T, g.N0 / ctas) ||
        !byte_map(&mx2, hidden, H, T, (g.subs > 1 ? g.N1 : g.N0) / ctas))
        return CIS_ERR_UNSUPPORTED;
    auto run = logits_dtype == CIS_BF16
                   ? (pair ? launch<__nv_bfloat16, true> : launch<__nv_bfloat16, false>)
                   : (pair ? launch<float, true> : launch<float, false>);
    return run(mw, mx, mx2, g, (cudaStream_t)stream) == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
