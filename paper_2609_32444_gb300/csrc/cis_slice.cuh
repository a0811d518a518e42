// cis_slice.cuh -- one CTA's slice of a row in shared memory, for rows of any
// alignment and length: the distillation loss, which reads a row more than once, splits
// it over the CTAs of a cluster and holds every slice on chip.
//
// The slab starts at the 8-entry boundary of global memory at or before the slice:
// `pad` entries before the slice, and those after it up to a whole group of 8, are
// -inf.  Bulk copies bring the 16-byte blocks that lie inside the slice, plain loads
// the few entries at its two ends; nothing outside the slice is read.
//
// Exponents are formed as (z - m) kappa, kappa = log2e / temperature: one more packed
// subtraction for two entries than z kappa - m kappa, and in return no rounding of an
// offset to take out and no other form for maxima of any size (masked entries at
// -1e9 or the type's lowest value).
#pragma once

#include <cooperative_groups.h>

#include "cis_dsmem.cuh"
#include "cis_kernels.h"

namespace cis {
namespace {

struct ClusterPlace {
    unsigned rank, size;
};
__device__ __forceinline__ ClusterPlace cluster_place()
{
    const cooperative_groups::cluster_group c = cooperative_groups::this_cluster();
    return {c.block_rank(), c.num_blocks()};
}

template <typename InT> struct Slice {
    const InT *src;  // the slice's first entry
    int n;           // entries
    int pad;         // entries of the slab before it
    int ng;          // groups of 8 in the slab
    int qg;          // groups per copy chunk

    __device__ __forceinline__ Slice(const InT *row, int64_t V, int64_t v0, int64_t slice)
    {
        const int64_t left = V - v0;
        n = (int)(left <= 0 ? 0 : (left < slice ? left : slice));
        src = row + v0;
        pad = (int)(reinterpret_cast<uintptr_t>(src) / sizeof(InT) & 7);
        ng = n > 0 ? (pad + n + 7) / 8 : 0;
        qg = (ng + kChunks - 1) / kChunks;
    }
    __device__ __forceinline__ int chunk_begin(int c) const { return c * qg; }
    __device__ __forceinline__ int chunk_end(int c) const { return min(ng, (c + 1) * qg); }
    // The 16-byte blocks inside the slice, as addresses.
    __device__ __forceinline__ void blocks(uintptr_t &a0, uintptr_t &a1) const
    {
        const uintptr_t b0 = reinterpret_cast<uintptr_t>(src);
        const uintptr_t b1 = b0 + (uintptr_t)n * sizeof(InT);
        a1 = b1 & ~(uintptr_t)15;
        a0 = (b0 + 15) & ~(uintptr_t)15;
        a0 = a0 < a1 ? a0 : a1;
    }
    // One thread, the barriers initialised with one arrival each.
    __device__ __forceinline__ void copy(uint8_t *slab, uint64_t *bar) const
    {
        constexpr int kGroup = 8 * (int)sizeof(InT);
        uintptr_t a0, a1;
        blocks(a0, a1);
        const uintptr_t base = reinterpret_cast<uintptr_t>(src) - (uintptr_t)pad * sizeof(InT);
        for (int c = 0; c < kChunks && chunk_begin(c) < ng; ++c) {
            uintptr_t lo = base + (uintptr_t)chunk_begin(c) * kGroup;
            uintptr_t hi = base + (uintptr_t)chunk_end(c) * kGroup;
            lo = lo < a0 ? a0 : lo;
            hi = hi > a1 ? a1 : hi;
            const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) : 0u;
            const uint32_t b = smem_u32(&bar[c]);
            mbar_expect_tx(b, bytes);
            if (bytes)
                bulk_g2s(smem_u32(slab) + (uint32_t)(lo - base),
                         reinterpret_cast<const void *>(lo), bytes, b);
        }
    }
    // The ends, by the 32 lanes of one warp: the entries outside the blocks, at most 7
    // on each side, and the padding.
    __device__ __forceinline__ void ends(uint8_t *slab, int lane) const
    {
        if (n == 0)
            return;
        uintptr_t a0, a1;
        blocks(a0, a1);
        const uintptr_t b0 = reinterpret_cast<uintptr_t>(src);
        const int he = (int)((a0 > b0 ? a0 - b0 : 0) / sizeof(InT));
        const int te = (int)((a1 > b0 ? a1 - b0 : 0) / sizeof(InT));
        InT *sl = reinterpret_cast<InT *>(slab);
        // lanes 0..15 the head, 16..31 the tail (without a block: all of it is tail)
        const int e = lane < 16 ? lane : te + (lane - 16);
        if (lane < 16 ? e < he : e < n)
            sl[pad + e] = src[e];
        if (lane < pad)
            poke_neg_inf<InT>(slab, lane);
        if (lane < 8 * ng - pad - n)
            poke_neg_inf<InT>(slab, pad + n + lane);
    }
};

// CTAs per row, the entries of each (a multiple of 8) and the width of those that work on
// them: the smallest cluster whose slices are within 52 KB (bf16, four CTAs an SM) or 64 KB
// (fp32, three), up to 200 KB with 8 CTAs; cs = 0 where 8 cannot hold the row (over 819,200
// bf16 or 409,600 fp32 entries).  Measured with the distillation loss: T=8192, V=151936 bf16
// 830 us on 6 CTAs; in the form before pass 2 took two entries an instruction 856 on 6, 924 on 5,
// 1020 on 4, 858 to 882 on 7, 898 to 929 on 8; T=4096, V=32003 fp32 174 on 2 CTAs, 211 on 3, 180 on
// 4, 218 on 1.  128 threads for fp32 and for slices of at most 16384 entries, else 256: V=32000 bf16
// 100 against 110, V=32003 fp32 174 against 177, V=151936 866 against 856.
struct RowPlan {
    int cs;
    int64_t slice;
    int nt;
};
constexpr int64_t kMostSliceBytes = 200 * 1024;
inline RowPlan row_plan(int64_t V, int in_bytes)
{
    const int64_t target = (in_bytes == 2 ? 52 : 64) * 1024;
    for (int cs = 1; cs <= kMaxCluster; ++cs) {
        const int64_t slice = ((V + cs - 1) / cs + 7) / 8 * 8;
        if (slice * in_bytes <= target || cs == kMaxCluster) {
            if (slice * in_bytes > kMostSliceBytes)
                return {0, 0, 0};
            return {cs, slice, in_bytes == 4 || slice <= 16384 ? 128 : 256};
        }
    }
    return {0, 0, 0};
}

// Bytes of a slab of `slice` entries, whatever its alignment, and room to start it on
// a 128-byte boundary.
__host__ __device__ constexpr size_t slab_bytes(int64_t slice, int in_bytes)
{
    return (size_t)(slice + 16) * in_bytes + 128;
}
__device__ __forceinline__ uint8_t *slab_start(uint8_t *dyn)
{
    return dyn + ((128 - (smem_u32(dyn) & 127)) & 127);
}

// Sum of 2^{(z_i - m) kappa} over 8 values, added pairwise.
__device__ __forceinline__ float sum8_scaled(const float (&z)[8], float m, float kappa)
{
    const float2 nm = make_float2(-m, -m), k2 = make_float2(kappa, kappa);
    float2 e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x =
            __fmul2_rn(__fadd2_rn(make_float2(z[2 * i], z[2 * i + 1]), nm), k2);
        e[i] = make_float2(ex2_ftz(x.x), ex2_ftz(x.y));
    }
    const float2 s = __fadd2_rn(__fadd2_rn(e[0], e[1]), __fadd2_rn(e[2], e[3]));
    return s.x + s.y;
}

// The first NT threads' (max, sum), in all of them: the maximum first, then one rescaling a
// thread.  sh: NT / 32 slots, used once; barrier 1.
template <int NT>
__device__ __forceinline__ MaxSum block_scaled(MaxSum v, MaxSum *sh, float kappa)
{
    auto sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory"); };
    float M = v.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));  // (a NaN is kept by its sum)
    if ((threadIdx.x & 31) == 0)
        sh[threadIdx.x >> 5].m = M;
    sync();
    M = sh[0].m;
#pragma unroll
    for (int i = 1; i < NT / 32; ++i)
        M = fmaxf(M, sh[i].m);
    // an empty thread: s = 0, and e^{-inf} = 0
    float s = M == -INFINITY ? v.s : v.s * ex2_ftz((v.m - M) * kappa);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0)
        sh[threadIdx.x >> 5].s = s;
    sync();
    s = sh[0].s;
#pragma unroll
    for (int i = 1; i < NT / 32; ++i)
        s += sh[i].s;
    return {M, s};
}

// The pairs of a cluster's n <= 8 CTAs, by one warp: every lane gets their (max, sum), added
// in the same order everywhere.
__device__ __forceinline__ MaxSum warp_combine(const float2 *part, unsigned n, float kappa)
{
    const unsigned lane = threadIdx.x & 31;
    const float2 p = lane < n ? part[lane] : make_float2(-INFINITY, 0.0f);
    float M = p.x;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    M = __shfl_sync(0xffffffffu, M, 0);
    float S = M == -INFINITY ? p.y : p.y * ex2_ftz((p.x - M) * kappa);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
        S += __shfl_xor_sync(0xffffffffu, S, o);
    return {M, __shfl_sync(0xffffffffu, S, 0)};
}

// (z - m) / temperature as an unevaluated pair.
__device__ __forceinline__ float scaled_diff(float z, float m, const Scale &s, float &lo)
{
    float dl;
    const float d = two_sum(z, -m, dl), p = d * s.hi;
    lo = isfinite(p) ? fmaf(d, s.hi, -p) + fmaf(d, s.lo, dl * s.hi) : 0.0f;
    return p;
}

}  // namespace
}  // namespace cis
