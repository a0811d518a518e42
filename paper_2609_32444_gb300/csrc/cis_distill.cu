// cis_distill.cu -- the distillation loss against a teacher's lists and its gradient
// (cis_distill_fwd_bwd): one read of the logits, one write of dlogits.
//
// Per row, with p = softmax(z / tau), the listed tokens S = {j_k} and the teacher's
// log-probabilities a_k of them (kinds: cis_distill_kind_t):
//   topk     q = softmax(a):  L = sum_k q_k (log q_k - log p_k),  tau dL/dz_j = p_j - q_j
//   forward  q_k = e^{a_k}, the rest r = all j not in S with q_r = 1 - sum q:
//            L = sum_b q_b (log q_b - log p_b) over the listed tokens and r,
//            tau dL/dz_j = Q p_j - q_j,  for j in r  p_j (Q - q_r / p_r),  Q = sum_b q_b
//   reverse  L = sum_b p_b (log p_b - log q_b),
//            tau dL/dz_j = p_j (l_b(j) - L),  l_b = log p_b - log q_b.
// Outside the list every gradient is one multiple of e^{z_j / tau}: the second pass over
// the row is that product, and the listed entries (at most 256) are written after it.
//
// The listed entries are put at -inf in shared memory before the first pass, so that the
// sum over the rest is formed by itself: p_r = 1 - p_S would lose it where the list holds
// nearly all.
//
// A reverse gradient compares a token's l with L, both of which are formed from the outcomes that
// have a probability: a listed token at -1e9 has an l of that size and no p.
//
// Precision of L: it is a difference of terms far larger than itself.  With
// phi(d) = e^{-d} - 1 + d >= 0 and d_b = log q_b - log p_b,
//   sum_b q_b d_b = sum_b q_b phi(d_b) + sum_b q_b - sum_b p_b,
// whose last two sums are known (1, or p_S), so that every term is of L's own size, and a
// common error of the log p_b (that of the row's sum) falls out to first order.
#include <math.h>

#include "cis_exp.cuh"
#include "cis_nvtx.h"
#include "cis_slice.cuh"

namespace cis {
namespace {

constexpr unsigned kAll32 = 0xffffffffu;

// e^{-d} - 1 + d: its series where the terms cancel (the first left out is below 2^-26 of
// the sum), -d as it stands where e^{-d} is out of range.
__device__ __forceinline__ float phi_small(float d)
{
    float s = 1.0f / 362880.0f;
    s = fmaf(s, -d, 1.0f / 40320.0f);
    s = fmaf(s, -d, 1.0f / 5040.0f);
    s = fmaf(s, -d, 1.0f / 720.0f);
    s = fmaf(s, -d, 1.0f / 120.0f);
    s = fmaf(s, -d, 1.0f / 24.0f);
    s = fmaf(s, -d, 1.0f / 6.0f);
    s = fmaf(s, -d, 0.5f);
    return s * d * d;
}
// q phi(d) with d = log q - log p, for a term q d: q phi = p + q (d - 1).
__device__ __forceinline__ float bregman(float q, float p, float d)
{
    if (fabsf(d) <= 0.5f)
        return q * phi_small(d);
    return q == 0.0f ? p : p + q * (d - 1.0f);
}

struct ListShared {
    alignas(8) uint64_t bar[kChunks];
    alignas(8) uint64_t xbar;
    alignas(16) float2 part[kMaxCluster];
    MaxSum red[16];
    float2 row;  // the rest's max (or the row's, without a rest) and its entries' multiplier
};
// The list, after the slab and sized by its length.
struct ListView {
    int32_t *table;          // finds repeated ids
    int32_t *id;             // -1: empty
    float *z, *a, *value;
};
// Slots of that table, a power of two: at most half of them are taken.
__host__ __device__ constexpr int hash_slots(int K)
{
    int n = 64;
    while (n < 2 * K)
        n *= 2;
    return n;
}
constexpr size_t list_bytes(int K)
{
    return (size_t)((K + 3) / 4 * 4) * 16 + (size_t)hash_slots(K) * 4;
}

// A barrier of the first NT threads.
template <int NT> __device__ __forceinline__ void sync_warps()
{
    asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory");
}

// What the list warp knows before the row's sum: every lane has it.
struct ListSums {
    float ms, ss;      // (max, sum of e^{(z - ms) / tau}) over the listed
    float qh, ql;      // sum of q (forward, reverse) as a pair
    float am, lq;      // topk: max a and log of sum e^{a - am}
    bool any;
};

__device__ __forceinline__ float warp_sum_f(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v += __shfl_xor_sync(kAll32, v, o);
    return v;
}
__device__ __forceinline__ float warp_max_f(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v = max_nan(v, __shfl_xor_sync(kAll32, v, o));
    return v;
}

// log p_k = u + ul of a listed token, M the row's maximum, logS + logSl the log of its sum.
__device__ __forceinline__ float list_log(float z, float M, float logS, float logSl,
                                          const Scale &sc, float &ul)
{
    float l, e;
    const float x = scaled_diff(z, M, sc, l), u = two_sum(x, -logS, e);
    ul = e + l - logSl;
    return u;
}
// log p_k - a_k, rounded about once.
__device__ __forceinline__ float list_gap(float u, float ul, float a)
{
    float e;
    const float d = two_sum(u, -a, e);
    return d + (e + ul);
}

// e^a as a pair.  1 less their sum may be 10^-6, so that 2^-42 of each is asked for where they
// are not below 10^-13 themselves (with 2^-29 that rest was off by 2^-10 of itself).
__device__ __forceinline__ float list_share(float a, float &lo)
{
    if (!(a > -30.0f && a <= 0.5f))
        return exp_pair(a, 0.0f, lo);
    int n;
    const float s = exp_parts(a, 0.0f, lo, n), up = __int_as_float(((n >> 5) + 127) << 23);
    lo *= up;
    return s * up;
}

__device__ __forceinline__ ListSums list_sums(const ListView &li, int K, int kind, const Scale &sc)
{
    const int lane = threadIdx.x & 31;
    ListSums r{-INFINITY, 0.0f, 0.0f, 0.0f, -INFINITY, 0.0f, false};
    bool any = false;
    for (int k = lane; k < K; k += 32)
        if (li.id[k] >= 0) {
            any = true;
            r.ms = max_nan(r.ms, li.z[k]);
            r.am = max_nan(r.am, li.a[k]);
        }
    r.any = __any_sync(kAll32, any);
    r.ms = warp_max_f(r.ms);
    r.am = warp_max_f(r.am);
    float ss = 0.0f, sa = 0.0f, qh = 0.0f, ql = 0.0f;
#pragma unroll 2
    for (int k = lane; k < K; k += 32)
        if (li.id[k] >= 0) {
            float l;
            const float x = scaled_diff(li.z[k], r.ms, sc, l);
            if (r.ms != -INFINITY)
                ss += expf(x + l);
            if (kind == CIS_DISTILL_TOPK) {
                sa += expf(li.a[k] - r.am);
            } else {
                float e, lo;
                const float hi = list_share(li.a[k], lo);
                qh = two_sum(qh, hi, e);
                ql += e + lo;
            }
        }
    r.ss = warp_sum_f(ss);
    if (kind == CIS_DISTILL_TOPK) {
        r.lq = logf(warp_sum_f(sa));
        return r;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        float e;
        const float h = __shfl_xor_sync(kAll32, qh, o), l = __shfl_xor_sync(kAll32, ql, o);
        qh = two_sum(qh, h, e);
        ql += l + e;
    }
    r.qh = qh;
    r.ql = ql;
    return r;
}

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v)
{
    return __float2bfloat16_rn(v);
}

// W results to global memory with a streaming store.
template <typename OutT, int W>
__device__ __forceinline__ void store_w(OutT *dst, const float (&v)[W])
{
    if constexpr (sizeof(OutT) == 4) {
        static_assert(W == 4, "one 16-byte store");
        __stcs(reinterpret_cast<float4 *>(dst), make_float4(v[0], v[1], v[2], v[3]));
    } else {
        uint32_t w[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        if constexpr (W == 8)
            __stcs(reinterpret_cast<uint4 *>(dst), make_uint4(w[0], w[1], w[2], w[3]));
        else
            __stcs(reinterpret_cast<uint2 *>(dst), make_uint2(w[0], w[1]));
    }
}
// W entries of the slab.
template <typename InT, int W>
__device__ __forceinline__ void load_w(const uint8_t *slab, int g, float (&z)[W])
{
    if constexpr (W == 8) {
        load8<InT>(slab, g, z);
    } else if constexpr (sizeof(InT) == 4) {
        const float4 q = reinterpret_cast<const float4 *>(slab)[g];
        z[0] = q.x; z[1] = q.y; z[2] = q.z; z[3] = q.w;
    } else {
        const uint2 q = reinterpret_cast<const uint2 *>(slab)[g];
        z[0] = bf16_lo(q.x); z[1] = bf16_hi(q.x);
        z[2] = bf16_lo(q.y); z[3] = bf16_hi(q.y);
    }
}

// Zero n entries at dst (any alignment).
template <typename OutT, int NT> __device__ __forceinline__ void zero_entries(OutT *dst, int n)
{
    constexpr int EV = 16 / sizeof(OutT);
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / (int)sizeof(OutT);
    head = head < n ? head : n;
    const int nvec = (n - head) / EV, tail = head + nvec * EV;
    for (int v = threadIdx.x; v < nvec; v += NT)
        __stcs(reinterpret_cast<uint4 *>(dst + head) + v, make_uint4(0, 0, 0, 0));
    if ((int)threadIdx.x < head)
        dst[threadIdx.x] = from_float<OutT>(0.0f);
    else if ((int)threadIdx.x - head < n - tail)
        dst[tail + threadIdx.x - head] = from_float<OutT>(0.0f);
}

// NT threads have the row's slice; one warp more has the list.  That warp forms the list's sums
// while the others are in pass 1, the row's numbers once the cluster's pairs are there, and the
// listed entries' gradients and the loss while the others are in pass 2.  With the list's work
// done by the first warp in between, a slice of 76 KB spent 22,000 cycles on its SM, 5,900 of
// them in that work (T=8192, V=151936, K=64: 1240 us).
//
// Bound: HBM, as far as four CTAs an SM (three in fp32) keep it busy through their waits for the
// copy and for each other: T=8192, V=151936, K=64 830 us, 6.0 TB/s; T=4096, V=32000 reverse 96 us,
// 4.8 TB/s; T=4096, V=32003 fp32, K=128 170 us, 5.4 TB/s.  T=256, V=1024: 23 us a call, of which
// this kernel is 10.
//
// Three CTAs an SM asked for in fp32, which is what its slices leave room for: without it the
// compiler takes 40 registers, for more CTAs, and spills.
template <typename InT, typename OutT, int NT>
__global__ void __launch_bounds__(NT + 32, sizeof(InT) == 4 ? 3 : 0)
    cis_distill_kernel(const __grid_constant__ DistillArgs a, int64_t slice)
{
    constexpr int NA = NT + 32;  // all threads
    extern __shared__ __align__(128) uint8_t dyn_smem[];
    __shared__ ListShared sh;
    uint8_t *slab = slab_start(dyn_smem);
    const ClusterPlace cl = cluster_place();
    const int64_t t = blockIdx.x / cl.size;
    const int tid = threadIdx.x, K = a.K;
    const bool list_warp = tid >= NT;
    const int64_t v0 = (int64_t)cl.rank * slice;
    const Slice<InT> sl(reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V, v0, slice);
    OutT *orow = reinterpret_cast<OutT *>(a.dz) + t * a.ld_out + v0;
    const bool grad = a.dz != nullptr;

    if (tid == 0)
        allow_next_grid();
    // this thread's first slot of the list, asked for ahead of the mask's answer
    const int32_t *ids = a.ids + t * a.ld_list;
    const float *lps = a.lp + t * a.ld_list;
    const int id0 = tid < K ? ids[tid] : -1;
    const float lp0 = tid < K ? lps[tid] : 0.0f;
    auto leave = [&](float kl) {  // a row without a gradient
        if (grad)
            zero_entries<OutT, NA>(orow, sl.n);
        if (tid == 0) {
            grid_wait();  // in every CTA, so that this grid ends after the one before
            if (cl.rank == 0) {
                if (a.kl_out)
                    a.kl_out[t] = kl;
                a.ws_terms[t] = (double)kl;
            }
        }
    };
    if (a.mask != nullptr && a.mask[t] == 0) {  // the same branch in the whole cluster
        leave(0.0f);
        return;
    }
    const int slots = hash_slots(K), pad = (K + 3) / 4 * 4;
    ListView li;
    li.table = reinterpret_cast<int32_t *>(slab + slab_bytes(slice, sizeof(InT)) - 128);
    li.id = li.table + slots;
    li.z = reinterpret_cast<float *>(li.id + pad);
    li.a = li.z + pad;
    li.value = li.a + pad;
    for (int i = tid; i < slots; i += NA)
        li.table[i] = -1;
    if (tid == 0) {
        for (int c = 0; c < kChunks; ++c)
            mbar_init_only(smem_u32(&sh.bar[c]), 1);
        mbar_init_only(smem_u32(&sh.xbar), 1);
        mbar_init_fence();
        mbar_expect_tx(smem_u32(&sh.xbar), (uint32_t)(cl.size * sizeof(float2)));
        sl.copy(slab, sh.bar);
    }
    if (list_warp)
        sl.ends(slab, tid - NT);
    __syncthreads();
    // The list, while the copy is in flight; a repeated id is found in the table.
    bool bad = false;
    for (int k = tid; k < K; k += NA) {
        int id = k == tid ? id0 : ids[k];
        const float lp = k == tid ? lp0 : lps[k];
        float z = 0.0f;
        if (id == -1 || lp == -INFINITY) {
            id = -1;
        } else if (id < 0 || id >= a.V) {
            bad = true;
            id = -1;
        } else {
            z = to_f32(reinterpret_cast<const InT *>(a.logits)[t * a.ld + id]);
            unsigned h = ((unsigned)id * 2654435761u) >> 16 & (slots - 1);
            for (int i = 0; i < slots; ++i, h = (h + 1) & (slots - 1)) {
                const int32_t was = atomicCAS(&li.table[h], -1, id);
                if (was == -1)
                    break;
                if (was == id) {
                    bad = true;
                    break;
                }
            }
        }
        li.id[k] = id;
        li.z[k] = z;
        li.a[k] = lp;
    }
    bad = __syncthreads_or(bad) != 0;
    const float kappa = a.sc.kappa;
    auto landed = [&] {
        for (int c = 0; c < kChunks && sl.chunk_begin(c) < sl.ng; ++c)
            wait_or_flag(smem_u32(&sh.bar[c]), false, a.status);
    };
    if (bad) {  // as every CTA of the cluster finds
        landed();
        leave(NAN);
        if (tid == 0 && cl.rank == 0)
            set_status(a.status, kStatusBadId);
        return;
    }
    cluster_arrive_relaxed();

    // The list warp's own: what the loss needs of the row.
    ListSums ls;
    MaxSum rest{0.0f, 0.0f};
    float M = 0.0f, S = 0.0f, er = 0.0f, es = 0.0f, pr = 0.0f, qr = 0.0f, mean = 0.0f, Q = 1.0f;
    float sw = 0.0f, logS = 0.0f, logSl = 0.0f;
    if (!list_warp) {
        landed();
        for (int k = tid; k < K; k += NT) {
            const int64_t e = (int64_t)li.id[k] - v0;
            if (li.id[k] >= 0 && e >= 0 && e < sl.n)
                poke_neg_inf<InT>(slab, sl.pad + (int)e);
        }
        sync_warps<NT>();
        // Pass 1: this thread's maximum over the rest, then its sum.
        MaxAcc<InT> macc;
        macc.consume(slab, tid, sl.ng, NT);
        const float m = macc.result();
        float s = 0.0f;
        if (m != -INFINITY) {
#pragma unroll 2
            for (int g = tid; g < sl.ng; g += NT) {
                float z[8];
                load8_any<InT>(slab, g, z);
                s += sum8_scaled(z, m, kappa);
            }
        }
        const MaxSum mine = block_scaled<NT>(MaxSum{m, s}, sh.red, kappa);
        cluster_wait();  // every CTA has started
        if (tid < (int)cl.size)
            st_async_pair(map_rank(smem_u32(&sh.part[cl.rank]), tid), mine.m, mine.s,
                          map_rank(smem_u32(&sh.xbar), tid));
        cluster_arrive_relaxed();  // waited for at the end: no CTA leaves before its peers' stores
    } else {
        sw = 1.0f;
        if (tid == NT) {
            grid_wait();  // the workspace is the kernel before's until it has ended
            sw = a.scale[t] * a.coef;
            if (a.token_weight)
                sw *= a.token_weight[t];
        }
        __syncwarp();
        sw = __shfl_sync(kAll32, sw, 0);
        ls = list_sums(li, K, a.kind, a.sc);
        cluster_wait();
        if (!mbar_wait_cluster(smem_u32(&sh.xbar), 0)) {
            if (tid == NT)
                set_status(a.status, kStatusTimeout);
            mbar_wait_cluster(smem_u32(&sh.xbar), 0);  // one more bounded chance
        }
        cluster_arrive_relaxed();
        // The row's numbers, in every lane.
        rest = warp_combine(sh.part, cl.size, kappa);
        M = fmaxf(rest.m, ls.ms);
        float l, lr;
        const float xr = scaled_diff(rest.m, M, a.sc, lr), xs = scaled_diff(ls.ms, M, a.sc, l);
        er = rest.m == -INFINITY ? rest.s : rest.s * expf(xr + lr);
        es = ls.ms == -INFINITY ? ls.ss : ls.ss * expf(xs + l);
        S = er + es;
        if (M == -INFINITY || ls.ms != ls.ms)
            S = NAN;  // no finite entry, or NaN among the listed
        qr = (1.0f - ls.qh) - ls.ql;
        pr = er / S;
        logS = logf(S);
        logSl = log_residual(S, logS);
        // The sum of the rest's gradients; each entry has its share e^{(z - max) / tau} / sum of
        // it, which holds where p_r itself is below fp32's range.
        float mult = 0.0f;
        if (a.kind == CIS_DISTILL_TOPK) {
            mult = ls.any ? pr : 0.0f;
        } else if (a.kind == CIS_DISTILL_FORWARD) {
            if (qr < a.tail_min) {
                qr = 0.0f;
                Q = ls.qh + ls.ql;
            }
            mult = fmaf(Q, pr, -qr);  // (0 exactly where nothing is listed)
        } else {
            qr = fmaxf(qr, a.tail_min);
            if (ls.qh != ls.qh)
                qr = NAN;
            if (ls.ms != -INFINITY) {  // (else only the rest: its gradient is 0)
                // L from the outcomes that have a probability: a token that the student masks
                // (its log p at -1e9, or beyond fp32's range) counts nothing, and neither it nor
                // one that the teacher all but excludes is what the others are compared with
                float sum = 0.0f;
                for (int k = tid - NT; k < K; k += 32)
                    if (li.id[k] >= 0) {
                        float ul;
                        const float u = list_log(li.z[k], M, logS, logSl, a.sc, ul);
                        const float p = expf(u + ul);
                        sum = fmaf(p, p == 0.0f ? 0.0f : list_gap(u, ul, li.a[k]), sum);
                    }
                const float gr = pr == 0.0f ? 0.0f
                                            : (logf(rest.s) - logf(qr)) + ((xr + lr) - logS);
                mean = fmaf(pr, gr, warp_sum_f(sum));
                mult = pr * (gr - mean);
            }
        }
        if (tid == NT)
            sh.row = make_float2(
                rest.m == -INFINITY ? M : rest.m,
                S != S ? NAN : rest.s == 0.0f ? 0.0f : __fdividef(sw * a.sc.hi * mult, rest.s));
    }
    __syncthreads();

    if (list_warp) {
        // The listed entries: log p_k = (z_k - M) / tau - log S = u + ul.
        const bool first = cl.rank == 0;
        const float c = sw * a.sc.hi;
        float sum = 0.0f;
#pragma unroll 2
        for (int k = tid - NT; k < K; k += 32) {
            const int64_t e = (int64_t)li.id[k] - v0;
            const bool mine = grad && e >= 0 && e < sl.n;
            if (li.id[k] < 0 || !(first || mine))
                continue;
            float ul;
            const float z = li.z[k], lp = li.a[k], u = list_log(z, M, logS, logSl, a.sc, ul);
            const float p = expf(u + ul);
            float lq = lp, lql = 0.0f;
            if (a.kind == CIS_DISTILL_TOPK) {
                float e3;
                lq = two_sum(lp, -ls.am, e3);
                lq = two_sum(lq, -ls.lq, lql);
                lql += e3;
            }
            const float q = expf(lq + lql);
            if (mine) {
                float d;
                if (a.kind == CIS_DISTILL_REVERSE)
                    d = p == 0.0f ? 0.0f : p * (list_gap(u, ul, lp) - mean);
                else
                    d = fmaf(Q, p, -q);
                li.value[k] = c * d;
            }
            if (first) {
                float e2;
                const float d0 = two_sum(lq, -u, e2);
                const float d = z == -INFINITY ? INFINITY : d0 + (e2 + lql - ul);
                if (a.kind == CIS_DISTILL_REVERSE)
                    sum += p == 0.0f ? q : bregman(p, q, -d);
                else
                    sum += bregman(q, p, d);
            }
        }
        if (first) {  // the row's loss
            sum = warp_sum_f(sum);
            float kl;
            if (a.kind == CIS_DISTILL_TOPK) {
                kl = ls.any ? sum + pr : 0.0f;  // sum q - sum_S p = p_r
                if (S != S)
                    kl = NAN;
            } else {
                // d_r = log(q_r / p_r), from the logarithms where p_r leaves fp32's range
                const float ratio = qr * (S / er);
                float l, dr = fabsf(ratio - 1.0f) < 0.25f ? log1pf(fmaf(qr, S / er, -1.0f))
                                                          : logf(ratio);
                if (er < 1e-30f && rest.s > 0.0f)
                    dr = (logf(qr) - logf(rest.s) + logS) - (scaled_diff(rest.m, M, a.sc, l) + l);
                if (a.kind == CIS_DISTILL_FORWARD)
                    kl = qr > 0.0f ? sum + bregman(qr, pr, dr)
                                   : sum + (((ls.qh - 1.0f) + ls.ql) + pr);
                else
                    kl = sum + (pr == 0.0f ? qr : bregman(pr, qr, -dr)) +
                         (((1.0f - ls.qh) - ls.ql) - qr);
            }
            if (tid == NT) {
                if (a.kl_out)
                    a.kl_out[t] = kl;
                a.ws_terms[t] = (double)sw * (double)kl;
            }
        }
    } else if (grad) {
        // Pass 2: the rest's gradients; the listed entries are at -inf and get 0 here.
        const float2 row = sh.row;
        constexpr int W = sizeof(InT) == 4 || sizeof(OutT) == 4 ? 4 : 8;
        constexpr int EV = 16 / sizeof(OutT);
        const int phase = (int)(reinterpret_cast<uintptr_t>(orow) / sizeof(OutT)) - sl.pad;
        const bool whole = (phase & (EV - 1)) == 0;
        const int g0 = whole ? (sl.pad + W - 1) / W : 0;
        const int g1 = whole ? (sl.pad + sl.n) / W : 0;
        auto value = [&](float z) { return row.y * ex2_ftz((z - row.x) * kappa); };
#pragma unroll 2
        for (int g = g0 + tid; g < g1; g += NT) {
            float z[W], v[W];
            load_w<InT, W>(slab, g, z);
#pragma unroll
            for (int i = 0; i < W; i += 2) {  // value(), two entries an instruction
                const float2 x = __fmul2_rn(
                    __fadd2_rn(make_float2(z[i], z[i + 1]), make_float2(-row.x, -row.x)),
                    make_float2(kappa, kappa));
                const float2 y = __fmul2_rn(make_float2(ex2_ftz(x.x), ex2_ftz(x.y)),
                                            make_float2(row.y, row.y));
                v[i] = y.x;
                v[i + 1] = y.y;
            }
            store_w<OutT, W>(orow + (W * g - sl.pad), v);
        }
        const int e0 = whole ? min(sl.n, g0 ? W * g0 - sl.pad : 0) : 0;
        const int e1 = whole ? max(e0, W * g1 - sl.pad) : 0;
        const InT *se = reinterpret_cast<const InT *>(slab);
        for (int k = tid; k < e0 + (sl.n - e1); k += NT) {
            const int e = k < e0 ? k : e1 + (k - e0);
            orow[e] = from_float<OutT>(value(to_f32(se[sl.pad + e])));
        }
    }
    __syncthreads();  // the listed entries' values come after the zeros
    if (grad)
        for (int k = tid; k < K; k += NA) {
            const int64_t e = (int64_t)li.id[k] - v0;
            if (li.id[k] >= 0 && e >= 0 && e < sl.n)
                orow[e] = from_float<OutT>(li.value[k]);
        }
    cluster_wait();
}

template <typename InT, typename OutT, int NT>
cudaError_t launch_nt(const DistillArgs &a, const RowPlan &p, cudaStream_t s)
{
    auto kern = cis_distill_kernel<InT, OutT, NT>;
    const size_t smem = slab_bytes(p.slice, sizeof(InT)) + list_bytes(a.K);
    constexpr int64_t most = kMostSliceBytes / (int64_t)sizeof(InT);
    const cudaError_t e =
        allow_smem(kern, slab_bytes(most, sizeof(InT)) + list_bytes(CIS_MAX_TOPK));
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * p.cs), 1, 1);
    cfg.blockDim = dim3(NT + 32, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a, p.slice);
}

template <typename InT, typename OutT>
cudaError_t launch_distill_t(const DistillArgs &a, cudaStream_t s)
{
    const RowPlan p = row_plan(a.V, (int)sizeof(InT));
    return p.nt == 128 ? launch_nt<InT, OutT, 128>(a, p, s) : launch_nt<InT, OutT, 256>(a, p, s);
}

bool distill_params_ok(const cis_distill_params_t *p)
{
    return p != nullptr && p->kind >= CIS_DISTILL_FORWARD && p->kind <= CIS_DISTILL_TOPK &&
           (p->agg == CIS_AGG_TOKEN_MEAN || p->agg == CIS_AGG_SEQ_MEAN_TOKEN_MEAN) &&
           temperature_ok(p->temperature) && fabs(p->coef) <= 1e30 && p->tail_min >= 1e-30 &&
           p->tail_min <= 0.5;  // (the kernel has them in fp32)
}

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" {

CIS_API cis_status_t cis_distill_default_params(cis_distill_params_t *out)
{
    if (out == nullptr)
        return CIS_ERR_INVALID_ARG;
    out->kind = CIS_DISTILL_FORWARD;
    out->agg = CIS_AGG_TOKEN_MEAN;
    out->temperature = 1.0;
    out->coef = 1.0;
    out->tail_min = 1e-6;
    out->global_counts = nullptr;
    return CIS_OK;
}

CIS_API cis_status_t cis_distill_workspace_size(int64_t T, size_t *bytes)
{
    if (bytes == nullptr || T < 0)
        return CIS_ERR_INVALID_ARG;
    *bytes = ws_layout(T).total;
    return CIS_OK;
}

CIS_API cis_status_t cis_distill_fwd_bwd(const void *logits, int32_t dtype, int64_t T, int64_t V,
                                         int64_t ld, const int32_t *top_ids, const float *top_lp,
                                         int32_t K, int64_t ld_top, const float *token_weight,
                                         const uint8_t *mask, const int32_t *cu_seqlens, int64_t B,
                                         const cis_distill_params_t *params, void *dlogits,
                                         int32_t dlogits_dtype, int64_t ld_out, float *kl_out,
                                         double *loss_out, void *workspace,
                                         size_t workspace_bytes, void *stream)
{
    NvtxRange nvtx_range("cis_distill_fwd_bwd");
    if (!row_args_ok(logits, dtype, T, V, ld) || K < 1 || K > CIS_MAX_TOPK || ld_top < K ||
        !distill_params_ok(params) || !aligned4(top_ids, top_lp, token_weight, cu_seqlens, kl_out) ||
        (reinterpret_cast<uintptr_t>(loss_out) & 7))
        return CIS_ERR_INVALID_ARG;
    const bool grad = dlogits != nullptr;
    if (grad && !row_args_ok(dlogits, dlogits_dtype, T, V, ld_out))
        return CIS_ERR_INVALID_ARG;
    if (params->agg == CIS_AGG_SEQ_MEAN_TOKEN_MEAN && (cu_seqlens == nullptr || B < 0))
        return CIS_ERR_INVALID_ARG;
    const WsLayout L = ws_layout(T);
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
        workspace_bytes < L.total)
        return CIS_ERR_INVALID_ARG;
    if (T > 0 && (logits == nullptr || top_ids == nullptr || top_lp == nullptr))
        return CIS_ERR_INVALID_ARG;
    const int ib = dtype == CIS_BF16 ? 2 : 4;
    if (T > 0 && grad) {
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(logits);
        const uintptr_t a1 = a0 + (uintptr_t)((T - 1) * ld + V) * ib;
        const uintptr_t b0 = reinterpret_cast<uintptr_t>(dlogits);
        const uintptr_t b1 =
            b0 + (uintptr_t)((T - 1) * ld_out + V) * (dlogits_dtype == CIS_BF16 ? 2 : 4);
        if (a0 < b1 && b0 < a1)
            return CIS_ERR_INVALID_ARG;
    }
    if (row_plan(V, ib).cs == 0 || T * kMaxCluster > 0x7fffffffLL)
        return CIS_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)stream;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    DistillArgs a = {};
    a.logits = logits;
    a.T = T;
    a.V = V;
    a.ld = ld;
    a.ids = top_ids;
    a.lp = top_lp;
    a.K = K;
    a.ld_list = ld_top;
    a.token_weight = token_weight;
    a.mask = mask;
    a.scale = reinterpret_cast<float *>(ws + L.scale);
    a.dz = dlogits;
    a.ld_out = ld_out;
    a.kl_out = kl_out;
    a.ws_terms = reinterpret_cast<double *>(ws + L.terms);
    a.status = reinterpret_cast<int32_t *>(ws + L.status);
    a.kind = params->kind;
    a.sc = make_scale(params->temperature);
    a.tail_min = (float)params->tail_min;
    a.coef = (float)params->coef;
    PassArgs r = {};  // what the reduction needs
    r.T = T;
    r.mask = mask;
    r.ws_terms = a.ws_terms;
    r.status = a.status;
    r.red_parts = ws + L.parts;
    r.red_ticket = reinterpret_cast<uint32_t *>(ws + L.ticket);
    r.overlap = true;
    cudaError_t e = launch_scales(mask, T, cu_seqlens, B, params->agg,
                                  reinterpret_cast<float *>(ws + L.scale), a.status, r.red_ticket,
                                  s, params->global_counts);
    if (e == cudaSuccess && T > 0) {
        if (dtype == CIS_BF16)
            e = grad && dlogits_dtype == CIS_F32
                    ? launch_distill_t<__nv_bfloat16, float>(a, s)
                    : launch_distill_t<__nv_bfloat16, __nv_bfloat16>(a, s);
        else
            e = grad && dlogits_dtype == CIS_BF16 ? launch_distill_t<float, __nv_bfloat16>(a, s)
                                                  : launch_distill_t<float, float>(a, s);
    }
    if (e == cudaSuccess)
        e = launch_reduce(r, nullptr, loss_out, s);
    return e == cudaSuccess ? CIS_OK
                            : (e == cudaErrorNotSupported ? CIS_ERR_UNSUPPORTED : CIS_ERR_CUDA);
}

}  // extern "C"
