// cis_rowpass.cuh -- one read of a row straight into registers, and the row's largest entries
// (the teacher's lists, the sampler).
//
// The CTAs of a cluster, and the warps of a CTA, have consecutive stretches of the row; a
// warp reads kB 16-byte vectors a lane at a time (a batch).  Besides what the caller forms of
// them (sums of exponentials), every lane keeps the maximum of each of its batches, in shared
// memory, and four maxima over a quarter of its entries each.  A CTA's r-th largest of those
// maxima is a bound that at least r of its entries are not below, and the least of the CTAs'
// bounds, with r = ceil(K / CTAs), is one that the row's K largest are not below.  The batches
// that reach the bound are read again (from L2), and their entries that reach it are the
// candidates: a complete head of the row's order (186 of them for K = 128 in a row of 32,003,
// 50 for K = 20 in one of 151,936 on eight CTAs, where likely entries are spread evenly over the
// row; the least of the warps' and CTAs' bounds is as low as their least likely stretch).
#pragma once

#include "cis_select.cuh"

namespace cis {
namespace {

template <int NT> struct PassShared {
    float part[kMaxCluster][4];  // each CTA's max, bound and two sums
    MaxSumU red[NT / 32], red2[NT / 32];
    float bound[NT / 32 * kTop];
    int items, n;
    int count[kMaxCluster];
};

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

template <typename InT, int NT, int kB> struct RowPass {
    static constexpr int EV = Vec<InT>::kN, W = NT / 32;
    const InT *row;
    const uint4 *rv;
    int V, head, nvec;
    int v0, v1;    // this CTA's vectors
    int s0, s1;    // this warp's
    float *bmax;   // [batches][NT]
    int nb;
    int end;       // the entry outside the vectors that this thread has (-1: none)
    float zend;
    float q[4];

    __device__ __forceinline__ RowPass(const InT *r, int64_t V_, unsigned rank, unsigned cs,
                                       float *maxima)
        : row(r), V((int)V_), bmax(maxima), nb(0), end(-1), zend(-INFINITY)
    {
        head = row_head(row, V);
        nvec = (V - head) / EV;
        rv = reinterpret_cast<const uint4 *>(row + head);
        v0 = (int)((int64_t)nvec * rank / cs);
        v1 = (int)((int64_t)nvec * (rank + 1) / cs);
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        s0 = seg(w);
        s1 = seg(w + 1);
        // the ragged ends, fewer than EV entries each: the first ones to the first warp of
        // the row, the last ones to the last
        const int tail0 = head + nvec * EV;
        if (rank == 0 && w == 0 && lane < head)
            end = lane;
        if (rank == cs - 1 && w == W - 1 && lane >= 16 && lane - 16 < V - tail0)
            end = tail0 + lane - 16;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = -INFINITY;
    }
    __device__ __forceinline__ int seg(int w) const { return v0 + (v1 - v0) * w / W; }

    // take(vectors, their maximum) for every batch, one(entry) for the ragged ends.  Absent
    // vectors of the last batch count as -inf.
    template <typename Take, typename One>
    __device__ __forceinline__ void stream(bool maxima, Take take, One one)
    {
        float *mine = bmax + threadIdx.x;
        auto batch = [&](const Vec<InT> (&x)[kB]) {
            const float mx = vec_max<kB>(x);
            if (maxima) {
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
            }
            take(x, mx);
        };
        // One body for whole and partial batches: a row's code is fetched once for few vectors.
        const uint4 none = make_uint4(Vec<InT>::kNone, Vec<InT>::kNone, Vec<InT>::kNone,
                                      Vec<InT>::kNone);
        auto load = [&](int v) { return v < s1 ? __ldg(rv + v) : none; };
        int v = s0 + (threadIdx.x & 31);
        if constexpr (kB == 1) {  // a vector a batch, four of them on their way
            uint4 ahead[3] = {load(v), load(v + 32), load(v + 64)};
#pragma unroll 1
            for (; v < s1; v += 32) {
                Vec<InT> x[1];
                x[0].q = ahead[0];
                ahead[0] = ahead[1];
                ahead[1] = ahead[2];
                ahead[2] = load(v + 96);
                batch(x);
            }
        } else {
#pragma unroll 1
            for (; v < s1; v += kB * 32) {
                Vec<InT> x[kB];
#pragma unroll
                for (int k = 0; k < kB; ++k)
                    x[k].q = load(v + k * 32);
                batch(x);
            }
        }
        if (end >= 0) {
            zend = to_f32(row[end]);
            q[0] = max_nan(q[0], zend);
            one(zend);
        }
    }
    // The CTA's bound for r of its entries: put() before a barrier, get() after it.
    __device__ __forceinline__ static bool few(int r) { return r <= 2 * W; }
    __device__ __forceinline__ void bound_put(PassShared<NT> &sh, int r) const
    {
        // r <= 2 W: the CTA's is taken among its warps' four largest; above, it is the least
        // of the warps' own ceil(r / W)-th largest
        if (few(r)) {
            warp_top(q, sh.bound + kTop * (threadIdx.x >> 5));
        } else {
            const float b = warp_bound(q, (r + W - 1) / W);
            if ((threadIdx.x & 31) == 0)
                sh.bound[threadIdx.x >> 5] = b;
        }
    }
    __device__ __forceinline__ static float bound_get(const PassShared<NT> &sh, int r)
    {
        if (few(r))
            return nth_of(sh.bound, kTop * W, r);
        float b = sh.bound[0];
#pragma unroll
        for (int w = 1; w < W; ++w)
            b = fminf(b, sh.bound[w]);
        return b;
    }
    // This CTA's candidates, in no order: all its entries at `bound` or above, but -inf.
    // Returns their number, above cap if they do not fit (or the batches to read do not).
    __device__ int collect(PassShared<NT> &sh, float bound, mass_t *list, int *items, int cap)
    {
        const int tid = threadIdx.x;
        for (int b = 0; b < nb; ++b) {
            const float x = bmax[b * NT + tid];
            if (x >= bound && x != -INFINITY) {
                const int at = atomicAdd(&sh.items, 1);
                if (at < cap)
                    items[at] = (tid >> 5) << 24 | (s0 + b * kB * 32 + (tid & 31));
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
        // one vector of an item a thread, four of them asked for at a time (one by one this step
        // took 10,000 cycles of the 50,000 of a row of 32,003 fp32 entries, K = 128)
        const int m = min(sh.items, cap) * kB;
        for (int i = tid; i < m; i += 4 * NT) {
            Vec<InT> x[4];
            int v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = -1;
                if (i + k * NT < m) {
                    const int it = items[(i + k * NT) / kB];
                    const int at = (it & 0xffffff) + ((i + k * NT) % kB) * 32;
                    if (at < seg((it >> 24) + 1)) {
                        v[k] = at;
                        x[k].q = __ldg(rv + at);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (v[k] >= 0 && vec_max<1>({x[k]}) >= bound)
#pragma unroll
                    for (int e = 0; e < EV; ++e)
                        offer(x[k].entry(e), head + v[k] * EV + e);
        }
        __syncthreads();
        return sh.items > cap ? cap + 1 : sh.n;
    }
};

// The lists of a row's CTAs (the same `list` in each, n entries of it) together, into `all` of
// the first CTA, which gets their number (above cap: they do not fit).  With barriers of the
// cluster; no CTA goes on before its list is read.
template <int NT>
__device__ int gather_lists(PassShared<NT> &sh, unsigned rank, unsigned cs, mass_t *list, int n,
                            mass_t *all, int cap)
{
    if (threadIdx.x == 0)
        sh.n = n;
    cluster_sync_data();
    if (rank == 0) {
        const cg::cluster_group cluster = cg::this_cluster();
        if (threadIdx.x < cs)
            sh.count[threadIdx.x] = *cluster.map_shared_rank(&sh.n, (int)threadIdx.x);
        __syncthreads();
        n = 0;
        for (unsigned c = 0; c < cs; ++c) {
            const int k = sh.count[c];
            if (n + k <= cap && k <= cap) {
                const mass_t *from = cluster.map_shared_rank(list, (int)c);
                for (int i = threadIdx.x; i < k; i += NT)
                    all[n + i] = from[i];
                n += k;
            } else {
                n = cap + 1;
            }
        }
    }
    cluster_sync_data();
    return n;
}

// This CTA's numbers to every CTA of the row, which has arrived at the cluster's barrier once
// before.
template <int NT>
__device__ __forceinline__ void exchange(PassShared<NT> &sh, unsigned rank, unsigned cs, float m,
                                         float bound, float s, float raw)
{
    cluster_wait();  // every CTA of the row has started
    if (threadIdx.x < cs) {
        float *to = cg::this_cluster().map_shared_rank(&sh.part[rank][0], (int)threadIdx.x);
        to[0] = m;
        to[1] = bound;
        to[2] = s;
        to[3] = raw;
    }
    cluster_sync_data();
}

// CTAs a row and the vectors that the plan's CTAs have at most.  As for the forward kernel, a
// row is split only while the CTAs stay within 608 and keep 512 vectors each.  With 1216 instead,
// lists at T=512, V=32003 fp32, K=128 took 56 us a call for 37, and sampling at T=512, V=32003
// fp32 101 for 82; with 304, sampling at T=256, V=151936 73 for 66.
struct PassPlan {
    int cs, nt, kb;
    size_t maxima;  // bytes of the batches' maxima
};
// A CTA has at most 65537 vectors, a warp 8193 of them: 65 batches of four a lane.
constexpr size_t kMostMaxima = 65 * 256 * sizeof(float);
inline PassPlan pass_plan(int64_t T, int64_t V, int in_bytes)
{
    const int64_t nvec = V * in_bytes / 16;
    PassPlan p{1, nvec <= 512 ? 64 : 256, 4, 0};
    while (p.cs < kMaxCluster && T * p.cs * 2 <= 608 && nvec / (2 * p.cs) >= 512)
        p.cs *= 2;
    while (p.cs < kMaxCluster && nvec / p.cs > 65536)  // the maxima fit shared memory
        p.cs *= 2;
    if (nvec <= 4096 * p.cs)
        p.kb = 1;
    // a warp's share of a CTA's share, each rounded up
    const int64_t cta = (nvec + p.cs - 1) / p.cs, warp = (cta + p.nt / 32 - 1) / (p.nt / 32);
    p.maxima = (size_t)((warp + 32 * p.kb - 1) / (32 * p.kb)) * p.nt * sizeof(float);
    return p;
}

}  // namespace
}  // namespace cis
