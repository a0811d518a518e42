// cis_select.cuh -- exact selection in a row's order (value descending, index ascending)
// by a cluster of CTAs: the k largest, the smallest prefix of a given mass, the entry at
// which a running mass passes a number.
//
// Values are compared as 32-bit keys in the order of the numbers (-0 as +0).  Masses are
// whole numbers, e^{(z - M) / tau} in units of 2^-43 from an exponential that is right to
// 2^-42: their sums do not depend on the order they are formed in, so that every CTA, every
// split and every call come to the same entry, and 2^63 holds a row of 2^20 maxima.
#pragma once

#include <stddef.h>

#include "cis_exp.cuh"
#include "cis_expacc.cuh"
#include "cis_slice.cuh"

namespace cis {
namespace {

namespace cg = cooperative_groups;

constexpr int kMassBits = 43;
typedef unsigned long long mass_t;

__device__ __forceinline__ uint32_t order_key(float z)
{
    const uint32_t b = __float_as_uint(z + 0.0f);  // -0 + 0 = +0
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
// An entry in the order: larger is earlier.
__device__ __forceinline__ mass_t order_pair(uint32_t key, uint32_t index)
{
    return ((mass_t)key << 32) | (0xffffffffu - index);
}

// 1 / tau of a row's own temperature, as a pair (its residual from an FMA), and log2e / tau.
__device__ __forceinline__ Scale device_scale(float tau)
{
    Scale s;
    s.hi = 1.0f / tau;
    s.lo = s.hi * fmaf(-s.hi, tau, 1.0f);
    constexpr float log2e_lo = (float)(1.4426950408889634074 - (double)kLog2e);
    s.kappa = fmaf(kLog2e, s.hi, fmaf(kLog2e, s.lo, log2e_lo * s.hi));
    s.huge = kHugeLogit * tau;
    return s;
}

// e^{x + x_lo} in units of 2^-43, for -31 < x <= 0.
__device__ __forceinline__ unsigned long long fixed_exp(float x, float x_lo)
{
    float lo;
    int ni;
    const float s = exp_parts(x, x_lo, lo, ni);
    // in units of 2^-48 (lo is below 2^-23), then 2^{n >> 5}
    const long long v = ((long long)__float2uint_rn(s * 0x1p24f) << 24) +
                        (long long)__float2int_rn(lo * 0x1p48f);
    const int down = 48 - kMassBits - (ni >> 5);  // 5 .. 50
    return (unsigned long long)((v + (1ll << (down - 1))) >> down);
}
// e^{(z - M) / tau} in units of 2^-43, z <= M; 0 below e^-31, a quarter of a unit.
__device__ __forceinline__ mass_t fixed_mass(float z, float M, const Scale &sc)
{
    float dl;
    const float d = sum_pair(z, -M, dl), x = d * sc.hi;
    if (!(x > -31.0f))
        return 0;
    return fixed_exp(x, fmaf(d, sc.hi, -x) + fmaf(d, sc.lo, dl * sc.hi));
}
__device__ __forceinline__ double mass_value(mass_t m)
{
    return (double)m / (double)(1ull << kMassBits);
}

// A row's settings (cis_sample_tokens), checked.
struct RowSettings {
    Scale sc;
    float tau, u, top_p, min_p;
    int top_k;  // 0: off
    bool greedy, ok;
};

// The kept entries: those above `key`, and the first `ties` of those at it, by index.
struct Kept {
    uint32_t key;
    mass_t ties;
};

// The lowest key that min_p keeps: entries with (z - M) / tau >= log(min_p).
__device__ inline uint32_t min_p_key(float M, float tau, float min_p)
{
    const double lim = log((double)min_p), t = (double)tau;
    auto in = [&](float z) { return ((double)z - (double)M) / t >= lim; };
    float z = (float)((double)M + t * lim);
    z = z > M ? M : z;
    for (int i = 0; i < 4 && !in(z); ++i)
        z = nextafterf(z, INFINITY);
    for (int i = 0; i < 4 && in(nextafterf(z, -INFINITY)); ++i)
        z = nextafterf(z, -INFINITY);
    return order_key(z > M ? M : z);
}

// ------------------------------------------------------------------ candidates
// Sort n pairs in descending order (bitonic, padded with 0 up to a power of two); all threads.
// Up to 4 a thread they stay in registers, R neighbouring ones a thread: strides within a
// warp are shuffles, and shared memory and barriers are left for those across warps (512
// pairs on 256 threads: 6 stages of 45; every stage through shared memory took 660 cycles).
template <int NT, int R> __device__ void sort_regs(mass_t *list, int n, int size)
{
    const int first = (int)threadIdx.x * R;
    mass_t x[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        x[r] = first + r < n ? list[first + r] : 0;
    for (int k = 2; k <= size; k *= 2) {
        auto keep = [&](int r, int j, mass_t y) {  // the larger goes first in descending runs
            const int i = first + r;
            const bool more = ((i & j) == 0) == ((i & k) == 0);
            x[r] = (x[r] > y) == more ? x[r] : y;
        };
        int j = k / 2;
        for (; j >= 32 * R; j /= 2) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r)
                list[first + r] = x[r];
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r)
                keep(r, j, list[(first + r) ^ j]);
        }
        for (; j >= R; j /= 2)
#pragma unroll
            for (int r = 0; r < R; ++r)
                keep(r, j, __shfl_xor_sync(0xffffffffu, x[r], j / R));
#pragma unroll
        for (int h = R / 2; h > 0; h /= 2)
            if (h < k) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if ((r & h) == 0) {
                        const mass_t a = x[r], b = x[r | h];
                        keep(r, h, b);
                        x[r | h] = x[r] == a ? b : a;
                    }
            }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (first + r < size)
            list[first + r] = x[r];
    __syncthreads();
}
template <int NT> __device__ void sort_list(mass_t *list, int n)
{
    __syncthreads();
    if (n <= 96 && n <= NT) {
        // few: each pair counts those before it, without a barrier in between (different pairs
        // only; 64 of them: 900 cycles against 2,700)
        const mass_t p = (int)threadIdx.x < n ? list[threadIdx.x] : 0;
        int before = 0;
        if ((int)threadIdx.x < n)
#pragma unroll 4
            for (int i = 0; i < n; ++i)
                before += list[i] > p;
        __syncthreads();
        if ((int)threadIdx.x < n)
            list[before] = p;
        __syncthreads();
        return;
    }
    int size = 2;
    while (size < n)
        size *= 2;
    if (size <= NT)
        return sort_regs<NT, 1>(list, n, size);
    if (size <= 2 * NT)
        return sort_regs<NT, 2>(list, n, size);
    if (size <= 4 * NT)
        return sort_regs<NT, 4>(list, n, size);
    for (int i = threadIdx.x; i < size; i += NT)
        if (i >= n)
            list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int i = threadIdx.x; i < size / 2; i += NT) {
                const int lo = 2 * i - (i & (j - 1)), hi = lo + j;  // j a power of two
                const mass_t x = list[lo], y = list[hi];
                if ((x < y) == ((lo & k) == 0)) {
                    list[lo] = y;
                    list[hi] = x;
                }
            }
            __syncthreads();
        }
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

// The same for the whole of a row: the masses of e^{(z - M) / tau}, right to 2^-34 of each.
// With K = 512 log2e / tau as a pair, z K is n + f, |f| <= 1/2, by an FMA (rounded at 2^-26,
// whatever the size of z K); f and n are taken less those of M, and the mass is
// 2^{n >> 9} T[n & 511] e^{f ln2 / 512}, T[i] = 2^{i / 512} as a pair, the exponential by three
// terms.  34 instructions an entry and no branch, where fixed_mass takes some 60 and several:
// that bounds the kernels that add up whole rows.
constexpr int kRowTable = 512;
__device__ inline void fill_row_table(float2 *table)
{
    for (int i = threadIdx.x; i < kRowTable; i += blockDim.x) {
        const double x = (double)i * (0.693147180559945309417 / kRowTable);
        const float hi = (float)x;
        float lo;
        int n;
        const float s = exp_parts(hi, (float)(x - (double)hi), lo, n);
        const float up = n == 32 ? 2.0f : 1.0f;
        table[i] = make_float2(s * up, lo * up);  // (s * up in [1, 2))
    }
}
struct RowMass {
    const float2 *table;
    float low;         // entries below have no mass
    float base;        // 0, or M where z K would leave the range: z - M is exact then, as the
                       // entries that count are next to M
    float khi, klo, fM;
    int nM;

    __device__ __forceinline__ RowMass(const float2 *t, float M, float tau, const Scale &sc)
        : table(t)
    {
        low = M - 31.0f * tau;
        base = fabsf(M) < 5000.0f * tau ? 0.0f : M;
        // log2e = kLog2e + 1.9e-8, 1 / tau = hi + lo
        constexpr float log2e_lo = (float)(1.4426950408889634074 - (double)kLog2e);
        khi = 512.0f * kLog2e * sc.hi;
        klo = fmaf(512.0f * kLog2e, sc.hi, -khi) +
              512.0f * fmaf(kLog2e, sc.lo, log2e_lo * sc.hi);
        split(M - base, nM, fM);
    }
    __device__ __forceinline__ void split(float z, int &n, float &f) const
    {
        constexpr float magic = 12582912.0f;  // 1.5 * 2^23
        const float t = fmaf(z, khi, magic), w = t - magic;
        n = __float_as_int(t) - __float_as_int(magic);
        f = fmaf(z, klo, fmaf(z, khi, -w));
    }
    __device__ __forceinline__ mass_t operator()(float z) const
    {
        const bool in = z >= low;  // (M itself, however far apart its neighbours are)
        int n;
        float f;
        split(in ? z - base : 0.0f, n, f);
        n -= nM;
        f -= fM;
        const float2 T = table[n & (kRowTable - 1)];
        constexpr float c1 = (float)(0.693147180559945309417 / kRowTable);
        constexpr float c2 = (float)(0.5 * 0.693147180559945309417 / kRowTable *
                                     0.693147180559945309417 / kRowTable);
        constexpr float c3 = c1 * c2 / 3.0f;
        const float u = f * fmaf(f, fmaf(f, c3, c2), c1);  // below 2^-9
        const float lo = fmaf(T.x, u, T.y);
        // in units of 2^-39, then of 2^-43 and by 2^{n >> 9} (a shift of 0 .. 45)
        const long long v =
            ((long long)((__float_as_uint(T.x) & 0x7fffffu) | 0x800000u) << 20) +
            ((long long)__float2int_rn(lo * 0x1p39f) << 4);
        const int down = -(n >> 9) & 63;
        const unsigned long long m = (unsigned long long)((v + ((1ll << down) >> 1)) >> down);
        return in ? m : 0;
    }
};

// ------------------------------------------------------------------ clusters
constexpr int kSelThreads = 256;
constexpr int kSelCluster = 8;
constexpr int kBins = 32;
constexpr int kListMax = 1024;  // entries that a selection may come down to

template <int NT> struct SelectShared {
    alignas(16) mass_t list[kListMax];   // candidates
    alignas(16) float cols[kBins * NT];  // a selection's bins, a column a thread; then, as
                                         // kListMax mass_t, the cluster's list
    alignas(16) float2 table[kRowTable];
    mass_t part[2][2];      // this CTA's share of the running sums
    mass_t red[2][NT / 32];
    mass_t stretch[2][NT / 32];  // the warps' kept mass and ties
    mass_t hist[256];
    mass_t tot[256];
    mass_t above, equal;
    mass_t got;             // the entry that was found, plus 1
    float bins[2][kBins];
    float bin_over;
    uint32_t digit, low_key;
    int n;
    unsigned left[NT / 32]; // rows left to do, a bit each
    bool ready;             // the table is filled
};
static_assert(offsetof(SelectShared<kSelThreads>, cols) % alignof(mass_t) == 0 &&
                  sizeof(float) * kBins * kSelThreads >= sizeof(mass_t) * kListMax,
              "the columns hold the cluster's list");

// The rows that one cluster of the exact kernel takes, in order: rows group, group + groups,
// ... of which `left` says so, NT of them looked at together.  Every CTA of the cluster sees
// the same: the marks are read before any CTA goes on to write over one.
template <int NT> struct RowsLeft {
    SelectShared<NT> &sh;
    int64_t T, groups, base;
    int word = NT / 32;
    unsigned bits = 0;

    __device__ RowsLeft(SelectShared<NT> &s, int64_t T_, int64_t groups_, int64_t group)
        : sh(s), T(T_), groups(groups_), base(group - (int64_t)NT * groups_)
    {
    }
    template <typename F> __device__ int64_t next(F left)
    {
        for (;;) {
            while (bits == 0 && ++word < NT / 32)
                bits = sh.left[word];
            if (bits) {
                const int b = __ffs(bits) - 1;
                bits &= bits - 1;
                return base + (int64_t)(32 * word + b) * groups;
            }
            base += (int64_t)NT * groups;
            if (base >= T)
                return -1;
            const int64_t i = base + (int64_t)threadIdx.x * groups;
            const unsigned b = __ballot_sync(0xffffffffu, i < T && left(i));
            __syncthreads();
            if ((threadIdx.x & 31) == 0)
                sh.left[threadIdx.x >> 5] = b;
            cg::this_cluster().sync();
            word = -1;
        }
    }
};

// One cluster's work on one row.  CTA `rank` has the entries [j0, j1), and each of its warps a
// stretch of them; the row is read from memory (L2 after the first time) once for each step.
template <typename InT, int NT> struct RowSelect {
    static constexpr int EV = Vec<InT>::kN, W = NT / 32;
    static_assert(NT >= 256, "a histogram's bin a thread");
    SelectShared<NT> &sh;
    cg::cluster_group cl;
    unsigned rank, size;
    const InT *row;
    int64_t V, j0, j1;
    int head, v0, v1;
    int &buf;  // the exchanges' buffer in turn, across rows

    __device__ RowSelect(SelectShared<NT> &s, const InT *r, int64_t V_, int &turn)
        : sh(s), cl(cg::this_cluster()), row(r), V(V_), buf(turn)
    {
        rank = cl.block_rank();
        size = cl.num_blocks();
        head = row_head(row, (int)V);
        const int64_t nvec = (V - head) / EV;
        v0 = (int)(nvec * rank / size);
        v1 = (int)(nvec * (rank + 1) / size);
        j0 = rank == 0 ? 0 : head + (int64_t)v0 * EV;
        j1 = rank == size - 1 ? V : head + (int64_t)v1 * EV;
    }
    __device__ __forceinline__ int seg(int w) const
    {
        return v0 + (int)((int64_t)(v1 - v0) * w / W);
    }
    // The entries of warp w's stretch: [first(w), first(w + 1)).
    __device__ __forceinline__ int64_t first(int w) const
    {
        return w == 0 ? j0 : w == W ? j1 : head + (int64_t)seg(w) * EV;
    }
    // f(index of the first, entries, their number) for this CTA's entries, EV or fewer at a time
    // (those absent are -inf), each by a lane of its stretch's warp.
    template <typename F> __device__ __forceinline__ void vectors(F f) const
    {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const uint4 *rv = reinterpret_cast<const uint4 *>(row + head);
        const uint4 none = make_uint4(Vec<InT>::kNone, Vec<InT>::kNone, Vec<InT>::kNone,
                                      Vec<InT>::kNone);
        const int s1 = seg(w + 1);
        int v = seg(w) + lane;
        Vec<InT> x, y, t;  // two loads ahead
        x.q = v < s1 ? __ldg(rv + v) : none;
        y.q = v + 32 < s1 ? __ldg(rv + v + 32) : none;
        int64_t j = -1;  // the ragged ends come last, one entry as a vector
        const int64_t tail = head + (V - head) / EV * EV;
        if (rank == 0 && w == 0 && lane < head)
            j = lane;
        if (rank == size - 1 && w == W - 1 && lane >= 16 && tail + lane - 16 < V)
            j = tail + lane - 16;
#pragma unroll 1
        for (;;) {
            float z[EV];
            const bool body = v < s1;
            if (!body && j < 0)
                break;
            t.q = v + 64 < s1 ? __ldg(rv + v + 64) : none;
#pragma unroll
            for (int k = 0; k < EV; ++k)
                z[k] = x.entry(k);  // (-inf past the stretch)
            if (!body)
                z[0] = to_f32(row[j]);
            f(body ? head + (int64_t)v * EV : j, z, body ? EV : 1);
            if (!body)
                break;
            x = y;
            y = t;
            v += 32;
        }
    }
    // f(index, entry) for the same.
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        vectors([&](int64_t j, const float (&z)[EV], int n) {
#pragma unroll
            for (int k = 0; k < EV; ++k)
                if (k < n)
                    f(j + k, z[k]);
        });
    }
    template <typename T> __device__ __forceinline__ const T *peer(T *p, unsigned r)
    {
        return cl.map_shared_rank(p, (int)r);
    }
    __device__ __forceinline__ static void warp_sums(mass_t &a, mass_t &b)
    {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
    }
    // Two sums over the CTA; in every thread.
    __device__ void block_sum(mass_t &a, mass_t &b)
    {
        warp_sums(a, b);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) {
            sh.red[0][threadIdx.x >> 5] = a;
            sh.red[1][threadIdx.x >> 5] = b;
        }
        __syncthreads();
        a = b = 0;
        for (int w = 0; w < W; ++w) {
            a += sh.red[0][w];
            b += sh.red[1][w];
        }
    }
    // Two sums over the cluster, and their parts in the CTAs before this one.  The two
    // buffers take turns: a CTA writes one again only after the next exchange's barrier,
    // which its peers reach with their reads of this one done.
    __device__ void cluster_sum(mass_t &a, mass_t &b, mass_t &a_before, mass_t &b_before)
    {
        block_sum(a, b);
        if (threadIdx.x == 0) {
            sh.part[buf][0] = a;
            sh.part[buf][1] = b;
        }
        cl.sync();
        a = b = a_before = b_before = 0;
        for (unsigned r = 0; r < size; ++r) {
            const mass_t *p = peer(&sh.part[buf][0], r);
            const mass_t x = p[0], y = p[1];
            a_before += r < rank ? x : 0;
            b_before += r < rank ? y : 0;
            a += x;
            b += y;
        }
        buf ^= 1;
    }
    // The row's largest key, and its least but that of -inf.
    __device__ uint32_t max_key(uint32_t &least)
    {
        const uint32_t none = order_key(-INFINITY);
        uint32_t k = 0, l = 0xffffffffu;
        each([&](int64_t, float z) {
            const uint32_t q = order_key(z);
            k = max(k, q);
            l = q > none ? min(l, q) : l;
        });
        k = __reduce_max_sync(0xffffffffu, k);
        l = __reduce_min_sync(0xffffffffu, l);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) {
            sh.red[0][threadIdx.x >> 5] = k;
            sh.red[1][threadIdx.x >> 5] = l;
        }
        __syncthreads();
        mass_t a = 0, b = 0xffffffffu;
        for (int w = 0; w < W; ++w) {
            a = max(a, sh.red[0][w]);
            b = min(b, sh.red[1][w]);
        }
        if (threadIdx.x == 0) {
            sh.part[buf][0] = a;
            sh.part[buf][1] = b;
        }
        cl.sync();
        for (unsigned r = 0; r < size; ++r) {
            const mass_t *p = peer(&sh.part[buf][0], r);
            a = max(a, p[0]);
            b = min(b, p[1]);
        }
        buf ^= 1;
        least = (uint32_t)b;
        return (uint32_t)a;
    }
    // The key at which the weight of the entries from the largest on reaches `target`
    // (1 .. the total), the weight strictly above it and that at it.  weight(z): an entry's,
    // in whole numbers; approx(z): the same in fp32, `goal` the target likewise.  share > 0:
    // the target is ceil(share * the total), which the pass finds on its way.
    //
    // parts: the warps' weights above the key and their entries at it have been left in
    // sh.stretch, as kept_mass leaves them.
    //
    // Two levels of 32 bins, over [low, M] and then over the bin in which the fp32 weights
    // reach the goal, each thread with a column of its own (no atomics); then one pass adds
    // up the whole numbers above that bin and lists its entries, which the first CTA sorts.
    // Where they do not fit, or the bin was not the one, a radix selection does it.
    template <typename A, typename F>
    __device__ uint32_t select(mass_t &target, float goal, float share, float low, float M,
                               A approx, F weight, mass_t &above, mass_t &equal, bool &parts)
    {
        parts = false;
        uint32_t khi = order_key(M), klo = 0;  // the entries with klo < key <= khi
        float over = 0.0f;
        for (int level = 0; level < 4; ++level) {
            const float hi = key_value(khi), lo = klo ? key_value(klo) : low;
            const float inv = (float)kBins / (hi - lo);
            if (!(hi > lo) || !(inv < INFINITY) || !(inv > 0.0f))
                break;
            auto bin = [&](float z) {
                const float b = (hi - z) * inv;
                return b < (float)kBins ? (int)b : kBins - 1;
            };
            float *col = sh.cols + threadIdx.x;
            for (int b = 0; b < kBins; ++b)
                col[b * NT] = 0.0f;
            const float zhi0 = hi, zlo0 = klo ? lo : -INFINITY;
            const bool all_low = klo == 0;
            vectors([&](int64_t, const float (&z)[EV], int n) {
                float *c[EV], x[EV];
#pragma unroll
                for (int k = 0; k < EV; ++k) {
                    const bool in = k < n && z[k] <= zhi0 && (z[k] > zlo0 || all_low);
                    c[k] = col + (in ? bin(z[k]) : 0) * NT;
                    x[k] = in ? approx(z[k]) : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < EV; ++k)
                    *c[k] += x[k];
            });
            __syncthreads();
            const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
            for (int b = w; b < kBins; b += W) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < W; ++i)
                    s += sh.cols[b * NT + lane + 32 * i];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
                    s += __shfl_xor_sync(0xffffffffu, s, o);
                if (lane == 0)
                    sh.bins[buf][b] = s;
            }
            cl.sync();
            if (w == 0) {
                float s = 0.0f;
                for (unsigned r = 0; r < size; ++r)
                    s += peer(&sh.bins[buf][0], r)[lane];
                float incl = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const float y = __shfl_up_sync(0xffffffffu, incl, o);
                    incl += lane >= o ? y : 0.0f;
                }
                if (share > 0.0f && level == 0)
                    goal = share * __shfl_sync(0xffffffffu, incl, 31);
                const unsigned reach = __ballot_sync(0xffffffffu, over + incl >= goal);
                const int b = reach ? __ffs(reach) - 1 : kBins - 1;
                const float before = __shfl_sync(0xffffffffu, incl, b ? b - 1 : 0);
                // the largest key whose bin is b or beyond (lane 0), and the same for b + 1
                // (lane 1): bins do not fall as keys do
                if (lane < 2) {
                    uint32_t in = klo, out = khi;  // bin(in) >= at, or in = klo
                    if (bin(key_value(khi)) >= b + lane)
                        in = khi;
                    while (out - in > 1) {
                        const uint32_t mid = in + (out - in) / 2;
                        if (bin(key_value(mid)) >= b + lane)
                            in = mid;
                        else
                            out = mid;
                    }
                    if (lane == 0) {
                        sh.bin_over = over + (b ? before : 0.0f);
                        sh.digit = in;
                    } else {
                        sh.low_key = b < kBins - 1 ? in : klo;
                    }
                }
            }
            buf ^= 1;
            __syncthreads();
            khi = sh.digit;
            klo = sh.low_key;
            over = sh.bin_over;
            __syncthreads();
            if (level == 0)
                continue;
            // whole numbers above the bin, and its entries
            if (threadIdx.x == 0)
                sh.n = 0;
            __syncthreads();
            mass_t up = 0, n = 0, all_of = 0, x, y, at;
            const float zhi = key_value(khi), zlo = klo ? key_value(klo) : -INFINITY;
            vectors([&](int64_t j, const float (&z)[EV], int m) {
                mass_t w[EV];
                unsigned in = 0;  // (z = -inf has weight only where entries are counted: klo = 0
                                  // lists it)
#pragma unroll
                for (int k = 0; k < EV; ++k) {
                    w[k] = k < m ? weight(z[k]) : 0;
                    up += z[k] > zhi ? w[k] : 0;
                    all_of += w[k];
                    in |= (!(z[k] > zhi) && (z[k] > zlo || klo == 0) && w[k] != 0 ? 1u : 0u) << k;
                }
                if (in)
#pragma unroll
                    for (int k = 0; k < EV; ++k)
                        if (in >> k & 1) {
                            const int i = atomicAdd(&sh.n, 1);
                            if (i < kListMax)
                                sh.list[i] = order_pair(order_key(z[k]), (uint32_t)(j + k));
                        }
            });
            mass_t a = up, b = 0;
            warp_sums(a, b);
            __syncthreads();
            if ((threadIdx.x & 31) == 0) {
                sh.stretch[0][threadIdx.x >> 5] = a;
                sh.stretch[1][threadIdx.x >> 5] = 0;
            }
            n = threadIdx.x == 0 ? (mass_t)sh.n : 0;
            const int mine = sh.n;
            cluster_sum(up, n, x, at);
            if (n > kListMax)
                continue;  // another level
            if (share > 0.0f) {
                mass_t none = 0;
                cluster_sum(all_of, none, x, y);
                target = (mass_t)ceil((double)share * (double)all_of);
            }
            mass_t *all = cl.map_shared_rank(reinterpret_cast<mass_t *>(sh.cols), 0);
            for (int i = threadIdx.x; i < mine; i += NT)
                all[at + i] = sh.list[i];
            cl.sync();
            if (rank == 0)
                pick(reinterpret_cast<mass_t *>(sh.cols), (int)n, target, up, weight);
            cl.sync();
            const SelectShared<NT> *lead = peer(&sh, 0);
            const mass_t got = lead->got;
            above = lead->above;
            equal = lead->equal;
            cl.sync();
            if (!got)
                break;
            const uint32_t key = (uint32_t)(got - 1);
            for (int i = threadIdx.x; i < mine; i += NT) {
                const uint32_t k = (uint32_t)(sh.list[i] >> 32);
                const int64_t j = (int64_t)(0xffffffffu - (uint32_t)sh.list[i]);
                int of = 0;
                while (of < W - 1 && j >= first(of + 1))
                    ++of;
                if (k > key)
                    atomicAdd(&sh.stretch[0][of], weight(key_value(k)));
                else if (k == key)
                    atomicAdd(&sh.stretch[1][of], (mass_t)1);
            }
            __syncthreads();
            parts = true;
            return key;
        }
        if (share > 0.0f) {
            mass_t all_of = 0, none = 0, x, y;
            each([&](int64_t, float z) { all_of += weight(z); });
            cluster_sum(all_of, none, x, y);
            target = (mass_t)ceil((double)share * (double)all_of);
        }
        return radix(target, weight, above, equal);
    }
    // Among n entries, `up` weight before them: got = key + 1 where `target` is reached.
    template <typename F>
    __device__ void pick(mass_t *all, int n, mass_t target, mass_t up, F weight)
    {
        sort_list<NT>(all, n);
        const int per = (n + NT - 1) / NT, i0 = min(n, (int)threadIdx.x * per), i1 = min(n, i0 + per);
        auto own = [&](int i) {
            return weight(key_value((uint32_t)(all[i] >> 32)));
        };
        mass_t sum = 0;
        for (int i = i0; i < i1; ++i)
            sum += own(i);
        mass_t run = sum;
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const mass_t x = __shfl_up_sync(0xffffffffu, run, o);
            run += lane >= o ? x : 0;
        }
        if (threadIdx.x == 0)
            sh.got = 0;
        __syncthreads();
        if (lane == 31)
            sh.red[0][w] = run;
        __syncthreads();
        run += up - sum;
        for (int i = 0; i < w; ++i)
            run += sh.red[0][i];
        for (int i = i0; i < i1; ++i) {
            const mass_t next = run + own(i);
            if (run < target && next >= target)
                sh.got = (all[i] >> 32) + 1;
            run = next;
        }
        __syncthreads();
        const mass_t got = sh.got;
        mass_t a = 0, b = 0;
        for (int i = i0; i < i1; ++i) {
            const mass_t k = all[i] >> 32;
            a += k + 1 > got ? own(i) : 0;
            b += k + 1 == got ? own(i) : 0;
        }
        block_sum(a, b);
        if (threadIdx.x == 0) {
            sh.above = up + a;
            sh.equal = b;
        }
    }
    // The same by digits of 8 bits, whatever the entries.
    template <typename F>
    __device__ uint32_t radix(mass_t target, F weight, mass_t &above, mass_t &equal)
    {
        uint32_t prefix = 0;
        mass_t over = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            const int bin = threadIdx.x & 255;
            sh.hist[bin] = 0;
            __syncthreads();
            each([&](int64_t, float z) {
                const uint32_t k = order_key(z);
                if (shift == 24 || ((k ^ prefix) >> (shift + 8)) == 0) {
                    const mass_t w = weight(z);
                    if (w)
                        atomicAdd(&sh.hist[(k >> shift) & 255], w);
                }
            });
            cl.sync();
            mass_t s = 0;
            for (unsigned r = 0; r < size; ++r)
                s += *peer(&sh.hist[bin], r);
            sh.tot[bin] = s;
            __syncthreads();
            if (threadIdx.x < 32) {  // lane l: bins 255 - 8 l and the seven below it
                const int lane = threadIdx.x;
                s = 0;
                for (int i = 0; i < 8; ++i)
                    s += sh.tot[255 - 8 * lane - i];
                mass_t incl = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const mass_t v = __shfl_up_sync(0xffffffffu, incl, o);
                    incl += lane >= o ? v : 0;
                }
                mass_t run = over + incl - s;
                if (run < target && (run + s >= target || lane == 31)) {
                    int d = 255 - 8 * lane;
                    for (int i = 0; i < 7 && run + sh.tot[d] < target; ++i)
                        run += sh.tot[d--];
                    sh.digit = (uint32_t)d;
                    sh.above = run;
                    sh.equal = sh.tot[d];
                }
            }
            cl.sync();  // the peers' reads of the histogram are done as well
            prefix |= sh.digit << shift;
            over = sh.above;
        }
        above = over;
        equal = sh.equal;
        __syncthreads();
        return prefix;
    }
    // Mass above `key` and the number of entries at it, with the parts before this CTA; the
    // warps' parts stay in sh.stretch.
    __device__ void kept_mass(uint32_t key, const RowMass &mass, mass_t &gt, mass_t &eq,
                              mass_t &gt_before, mass_t &eq_before)
    {
        gt = eq = 0;
        const float zk = key ? key_value(key) : -INFINITY;
        vectors([&](int64_t, const float (&z)[EV], int n) {
#pragma unroll
            for (int k = 0; k < EV; ++k) {
                const mass_t x = mass(z[k]);  // (0 where absent)
                gt += z[k] > zk ? x : 0;
                eq += k < n && z[k] == zk;
            }
        });
        mass_t a = gt, b = eq;
        warp_sums(a, b);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) {
            sh.stretch[0][threadIdx.x >> 5] = a;
            sh.stretch[1][threadIdx.x >> 5] = b;
        }
        cluster_sum(gt, eq, gt_before, eq_before);
    }
    // The same from the parts that a selection by these masses has left.
    __device__ void kept_parts(mass_t &gt, mass_t &eq, mass_t &gt_before, mass_t &eq_before)
    {
        const bool one = threadIdx.x < W;
        gt = one ? sh.stretch[0][threadIdx.x] : 0;
        eq = one ? sh.stretch[1][threadIdx.x] : 0;
        cluster_sum(gt, eq, gt_before, eq_before);
    }
    // The first entry, by index, whose running kept mass is above t (below the total): the
    // CTA that has it returns true in all its threads, with the index.  After kept_mass for
    // this key.
    __device__ bool locate(const Kept &kept, mass_t wkey, mass_t t, mass_t gt_before,
                           mass_t eq_before, const RowMass &mass, int64_t &index)
    {
        auto upto = [&](mass_t gt, mass_t eq) { return gt + min(eq, kept.ties) * wkey; };
        mass_t gt = gt_before, eq = eq_before;
        if (upto(gt, eq) > t)
            return false;  // an earlier CTA's
        int w = 0;
        for (; w < W; ++w) {
            const mass_t g = gt + sh.stretch[0][w], e = eq + sh.stretch[1][w];
            if (upto(g, e) > t)
                break;
            gt = g;
            eq = e;
        }
        if (w == W)
            return false;  // a later one's
        __syncthreads();
        if (threadIdx.x == 0)
            sh.got = 0;
        for (int64_t b = first(w); b < first(w + 1); b += NT) {
            const int64_t j = b + threadIdx.x;
            const bool in = j < first(w + 1);
            const float z = in ? to_f32(row[j]) : -INFINITY;
            const uint32_t k = order_key(z);
            const mass_t own = in && k > kept.key ? mass(z) : 0;
            const bool tie = in && k == kept.key;
            // this thread's place in the block's order: sums over the entries up to it
            const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
            mass_t iw = own, it = tie;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const mass_t x = __shfl_up_sync(0xffffffffu, iw, o);
                const mass_t y = __shfl_up_sync(0xffffffffu, it, o);
                iw += lane >= o ? x : 0;
                it += lane >= o ? y : 0;
            }
            __syncthreads();
            if (lane == 31) {
                sh.red[0][wid] = iw;
                sh.red[1][wid] = it;
            }
            __syncthreads();
            mass_t tw = 0, tt = 0;
            for (int i = 0; i < W; ++i) {
                const mass_t x = sh.red[0][i], y = sh.red[1][i];
                iw += i < wid ? x : 0;
                it += i < wid ? y : 0;
                tw += x;
                tt += y;
            }
            if (in && upto(gt + iw, eq + it) > t && upto(gt + iw - own, eq + it - tie) <= t)
                sh.got = (mass_t)j + 1;
            __syncthreads();
            if (sh.got) {
                index = (int64_t)sh.got - 1;
                return true;
            }
            gt += tw;
            eq += tt;
        }
        return false;
    }
};

}  // namespace
}  // namespace cis
