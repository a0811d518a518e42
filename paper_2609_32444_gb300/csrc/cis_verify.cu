// cis_verify.cu -- verification of drafted tokens against the target's probabilities, from given
// uniform numbers (cis_verify_tokens).
//
// Per request, with p_i = softmax(z_i / tau) of the target's rows, q_i the distribution that draft
// x_i came from, in order:  x_i is kept where u_i q_i(x_i) < p_i(x_i).  After the first one that
// is not, at i, the request's last token is drawn from max(p_i - q_i, 0) (from p_i where that adds
// up to less than 2^-32: a draft from q_i is rejected that seldom); after the last draft,
// from the target's next row.  At temperature 0 p is all on the row's first largest entry.
//
// Two kernels.  The first reads every row once, a row's stretches on CTAs of their own: maximum
// and sums of exponentials at tau and at 1.  In the second, CTAs that each have a few segments of
// a request's row put the stretches together, go through the drafts, and add up the row's masses; the
// last of them to finish draws the token.  Sums of fp32 exponentials decide a draft only where
// their error cannot matter: with E = 2^-20 a sum is off by less than 6 E of itself (cis_sample.cu),
// so that p and u q farther apart than 16 E of the larger are in the order they seem.  Else the
// draft, and in any case the last token, is decided by whole numbers: masses e^{(z - M) / tau} / S
// in units of 2^-60, right to 2^-35 of each, S the first kernel's sum.  What S is off by is common
// to a row; the sums of both rows' masses, SP and SQ, take it out again: q's share in p's unit is
// Q (1 + delta), delta = SP / SQ - 1, below 2^-16.  So that one pass does, a segment keeps SP, SQ
// and, of the entries where P is above Q, the sums of P - Q and of Q, from which max(p - q, 0)
// follows once delta is known; entries whose sign delta could turn are put in a list instead (a
// few of a row; some hundreds where bf16 logits and drafts differ by the same step in many).  Where
// the roundings of these sums could matter, a segment's entries are looked at again.
// Sums of whole numbers depend on no order.
//
// Bound: the first kernel by HBM (B=64, 4 drafts, V=151936 bf16: 32 us, 5.4 TB/s).  The second, 43 to
// 50 us of the call's 75 to 80, by nothing that is full (46 to 62% of its issue slots): each CTA fills
// the table (2 us), puts the stretches together and decides all drafts (2.4), as all of its request's
// do, and adds up its masses (7: 58 instructions an entry of two rows), in two waves of CTAs, and a
// request's last CTA draws (5 to 8).  With few requests the steps that depend on one another are all
// there is: stretches, drafts, sums, ticket, prefix, entry (B=1: 5 and 15 us, 19 to 21 a call).
#include <math.h>

#include "cis_nvtx.h"
#include "cis_rowpass.cuh"

namespace cis {
namespace {

// A stretch of a target row, and of its draft's.
struct Part {
    float m, s, s1;  // maximum, sums of e^{(z - m) / tau} and of e^{z - m}
    int arg;         // temperature 0: the first entry that is the maximum
    float md, sd;
    int unused[2];
};
static_assert(sizeof(Part) == 32, "two 16-byte words");

struct VerifyArgs {
    const void *z, *zd;
    int64_t ld, ldd;
    int B, D, V;
    int64_t N;
    const int32_t *ids, *cu;
    const float *u, *u_last, *tau, *tau_d;
    const uint8_t *mask;
    int32_t *tokens, *kept;
    float *lp, *lps;
    int32_t *status;
    Part *parts;  // [N + B][stretches]
    int stretches;
    struct Segment *segs;  // [B][segments]
    ulonglong2 *undecided;  // [B][segments][kListed]
    uint32_t *tickets;     // [B]: the second kernel's CTAs that have finished
    int groups, segments;  // of a request
};

constexpr int kVerifyThreads = 256, kWarps = kVerifyThreads / 32;
constexpr int kMaxStretches = 64;  // two a lane

// A request, checked.
struct Request {
    int a, n;         // its first draft and their number
    float tau, tau_d;
    bool on, ok, greedy, model;  // model: q from the draft's logits (else all on the draft)
};
__device__ __forceinline__ Request request(const VerifyArgs &g, int b)
{
    Request r;
    r.on = g.mask == nullptr || g.mask[b] != 0;
    r.ok = true;
    r.a = r.n = 0;
    r.tau = r.tau_d = 1.0f;
    r.greedy = r.model = false;
    if (!r.on)
        return r;
    const int64_t a = g.cu[b], e = g.cu[b + 1];
    r.tau = g.tau ? g.tau[b] : 1.0f;
    r.tau_d = g.tau_d ? g.tau_d[b] : 1.0f;
    const float u = g.u_last[b];
    r.ok = a >= 0 && a <= e && e <= g.N && e - a <= g.D && u >= 0.0f && u < 1.0f &&
           (r.tau == 0.0f || (r.tau >= 1e-3f && r.tau <= 1e3f)) &&
           (g.zd == nullptr || r.tau_d == 0.0f || (r.tau_d >= 1e-3f && r.tau_d <= 1e3f));
    if (!r.ok)
        return r;
    r.a = (int)a;
    r.n = (int)(e - a);
    r.greedy = r.tau == 0.0f;
    r.model = g.zd != nullptr && !r.greedy && r.tau_d > 0.0f;
    return r;
}

// e^{(m - M) / tau}, to 2^-22; 0 from -inf.
__device__ __forceinline__ float share_of(float m, float M, const Scale &sc)
{
    float lo;
    const float e = expf(scaled_diff(m, M, sc, lo));
    return fmaf(e, lo, e);
}
// The lanes' sums together, as sums of e^{z - m}, in every lane: each at its own whole offset, so
// that they move to the largest's by powers of two (where the maximum is too large for that, by
// the exponential).
template <bool kScaled> __device__ __forceinline__ MaxSumU warp_exp(const ExpAcc<false, kScaled> &acc)
{
    float M = acc.m;  // (a NaN is kept by its lane's sum)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    ExpAcc<false, kScaled> all = acc;
    all.m = M;
    all.c = M == -INFINITY ? 0.0f : ceilf(M * acc.kappa());
    float s = acc.S, d;
    if constexpr (kScaled)
        s += acc.lost;
    if (all.fast()) {
        d = acc.fast() ? acc.c - all.c : fmaf(acc.m, acc.kappa(), -all.c);
    } else {
        s = acc.result().s;
        d = acc.m == -INFINITY ? -INFINITY : (acc.m - M) * acc.kappa();
    }
    s *= ex2_ftz(d);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if (M == -INFINITY)
        return {M, s, 0.0f};
    all.S = s;
    if constexpr (kScaled)
        all.lost = 0.0f;
    return all.result();
}
// The log of a row's mass, and what it is short of it.
struct LogMass {
    float log, rest;
};
__device__ __forceinline__ LogMass log_mass(float mass)
{
    const float ls = logf(mass);
    return {ls, log_residual(mass, ls)};
}
// The log-probability of z: (z - M) / tau - log of the row's mass; at most 0, whatever the mass's
// roundings.
__device__ __forceinline__ float log_prob(float z, float M, const Scale &sc, const LogMass &m)
{
    float l, e;
    const float x = scaled_diff(z, M, sc, l), u = two_sum(x, -m.log, e);
    return fminf(u + (e + l - m.rest), 0.0f);
}

// CTAs an SM: fp32 rows have more instructions a byte (B=128, up to 8 drafts, V=32003: 66 us a call
// for 71 with three, on the same inputs; bf16 rows, B=64, 4 drafts, V=151936: 82 for 80).
template <typename InT> constexpr int kRowCtas = sizeof(InT) == 4 ? 4 : 3;

// A stretch of one row, of the target's or (the items behind theirs) a draft's, by a warp of its
// own: no barrier holds a warp whose loads have come.  Four vectors a lane at a time, with the next
// four on their way.
template <typename InT>
__global__ void __launch_bounds__(kVerifyThreads, kRowCtas<InT>)
    cis_verify_rows_kernel(const __grid_constant__ VerifyArgs g)
{
    constexpr int EV = Vec<InT>::kN, kB = 4;
    if (threadIdx.x == 0)
        allow_next_grid();
    const int lane = threadIdx.x & 31, rows = g.B * (g.D + 1);
    const int id = (int)blockIdx.x * kWarps + (int)(threadIdx.x >> 5);
    int item = id / g.stretches;
    const int st = id - item * g.stretches;
    if (item < g.B && st == 0 && lane == 0)
        g.tickets[item] = 0;
    const bool draft = item >= rows;
    item -= draft ? rows : 0;
    const int i = item / g.B, b = item - i * g.B;
    if (i > g.D)
        return;
    const Request r = request(g, b);
    if (!r.on || !r.ok || i > r.n || (draft && (!r.model || i == r.n)))
        return;
    const InT *row = draft ? static_cast<const InT *>(g.zd) + ((int64_t)r.a + i) * g.ldd
                           : static_cast<const InT *>(g.z) + ((int64_t)r.a + b + i) * g.ld;
    const int head = row_head(row, g.V), nvec = (g.V - head) / EV;
    const int v0 = nvec * st / g.stretches, v1 = nvec * (st + 1) / g.stretches;
    const uint4 *rv = reinterpret_cast<const uint4 *>(row + head), *at = rv + v0 + lane;
    const int full = (v1 - v0) / (32 * kB);
    Vec<InT> x[kB];
    uint4 next[kB];
    if (full > 0) {
#pragma unroll
        for (int k = 0; k < kB; ++k)
            next[k] = __ldg(at + 32 * k);
    }
    const float tau = draft ? r.tau_d : r.greedy ? 1.0f : r.tau;
    const Scale sc = device_scale(tau);
    const bool two = !draft && g.lp && tau != 1.0f;
    ExpAcc<false, true> acc;
    acc.k = sc.kappa;
    acc.h = sc.huge;
    ExpAcc<false> raw;
    auto batch = [&] {
        const float mx = vec_max<kB>(x);
        take<false, kB>(acc, x, mx);
        if (two)
            take<false, kB>(raw, x, mx);
    };
#pragma unroll 1
    for (int k0 = 1; k0 <= full; ++k0) {
#pragma unroll
        for (int k = 0; k < kB; ++k)
            x[k].q = next[k];
        at += 32 * kB;
        if (k0 < full) {
#pragma unroll
            for (int k = 0; k < kB; ++k)
                next[k] = __ldg(at + 32 * k);
        }
        batch();
    }
    const int left = v1 - v0 - full * 32 * kB;
    if (left > 0) {
        const uint4 none = make_uint4(Vec<InT>::kNone, Vec<InT>::kNone, Vec<InT>::kNone,
                                      Vec<InT>::kNone);
#pragma unroll
        for (int k = 0; k < kB; ++k)
            x[k].q = lane + 32 * k < left ? __ldg(at + 32 * k) : none;
        batch();
    }
    // the ragged ends, fewer than EV entries each: to the first and the last stretch
    const int tail = head + nvec * EV;
    int end = -1;
    if (st == 0 && lane < head)
        end = lane;
    if (st == g.stretches - 1 && lane >= 16 && lane - 16 < g.V - tail)
        end = tail + lane - 16;
    float zend = -INFINITY;
    if (end >= 0) {
        zend = to_f32(row[end]);
        acc.raise(zend);
        if (acc.m != -INFINITY)
            acc.add_entry(zend);
        if (two) {
            raw.raise(zend);
            if (raw.m != -INFINITY)
                raw.add_entry(zend);
        }
    }
    const MaxSumU o = warp_exp(acc);
    Part &out = g.parts[((int64_t)r.a + b + i) * g.stretches + st];
    if (draft) {
        if (lane == 0) {
            out.md = o.m;
            out.sd = o.s;
        }
        return;
    }
    const float s1 = two ? warp_exp(raw).s : o.s;
    int first = 0x7fffffff;
    if (r.greedy) {  // (read again, from L2)
#pragma unroll 1
        for (int v = v0 + lane; v < v1 && first == 0x7fffffff; v += 32 * kB) {
#pragma unroll
            for (int k = 0; k < kB; ++k)
                x[k].q = __ldg(rv + min(v + 32 * k, v1 - 1));
#pragma unroll
            for (int k = kB - 1; k >= 0; --k) {
                const Vec<InT> y[1] = {x[k]};
                if (vec_max<1>(y) == o.m) {
#pragma unroll
                    for (int e = EV - 1; e >= 0; --e)
                        first = y[0].entry(e) == o.m ? head + min(v + 32 * k, v1 - 1) * EV + e
                                                     : first;
                }
            }
        }
        if (end >= 0 && zend == o.m)
            first = min(first, end);
        first = __reduce_min_sync(0xffffffffu, first);
    }
    if (lane == 0) {
        out.m = o.m;
        out.s = o.s;
        out.s1 = s1;
        out.arg = first;
    }
}

// ------------------------------------------------------------------ the request
enum : int { kAccept = 0, kReject = 1, kOpen = 2, kBadRow = 3, kBadDraft = 4 };

constexpr int kUnitBits = 60;
constexpr int kSteps = 2048;  // the table's, from 1 to 2

// A row's masses, e^{(z - M) / tau} / S in units of 2^-60.  With Y = 2048 log2 of it, n + f,
// |f| <= 1: 2^{n >> 11} T[n & 2047] e^{f ln2 / 2048}, T[i] = 2^{i / 2048} in 62 bits, the exponential
// by three terms.  z K and the row's own n are whole numbers taken off by one FMA, whose rest is
// exact for bf16 entries and else right to 2^-25; f and f ln2 / 2048 are rounded to 2^-24 of
// themselves, and their product with T to 2^-36: 2^-35 of the mass in all.  Entries below e^-42
// are 0.  (No fp64: two lanes a cycle.)
struct RowShare {
    float khi, klo;  // K = 2048 log2e / tau
    float magic;     // 1.5 2^23 less the row's n
    float f0;        // its fraction
    float base;      // 0, or M where z K would leave the range: the entries that count are next to
                     // M then, and z - M is exact
    float low;       // of z - base: a mass of 0
    float unit;      // 2048 log2 S as it was taken
    // depth: from where on entries are 0, in units of e.  A draft's row has 0.2 more than the
    // target's: entries that both forbid are then as far apart as any.
    static constexpr float kDepth = 41.75f;  // (a shift of 63 bits, below 42.28)
    __device__ void set(float M, float tau, const Scale &sc, float S, float depth)
    {
        constexpr float log2e_lo = (float)(1.4426950408889634074 - (double)kLog2e);
        khi = kSteps * kLog2e * sc.hi;
        klo = fmaf(kSteps * kLog2e, sc.hi, -khi) +
              kSteps * fmaf(kLog2e, sc.lo, log2e_lo * sc.hi);
        base = fabsf(M) < 1250.0f * tau ? 0.0f : M;
        unit = kSteps * log2f(S);
        const float x = M - base, h = x * khi, n = rintf(h), m = rintf(unit);
        const float f = ((h - n) + (unit - m)) + (fmaf(x, khi, -h) + x * klo), r = rintf(f);
        magic = 12582912.0f - (n + m + r);
        f0 = f - r;
        low = x - (depth - 0.6931472f / kSteps * unit) * tau;
    }
    // Y: its whole part (as its place in t's bits) and fraction
    __device__ __forceinline__ float split(float z, float &t) const
    {
        const float x = fmaxf(z - base, low);
        t = fmaf(x, khi, magic);
        return fmaf(x, khi, magic - t) + fmaf(x, klo, -f0);
    }
    __device__ __forceinline__ mass_t operator()(const mass_t *table, float z) const
    {
        float t;
        const float f = split(z, t);
        return mass(table, t, f * fmaf(f, fmaf(f, kC3, kC2), kC1));
    }
    // e^{f ln2 / 2048} - 1 in units of 2^-36
    static constexpr double kStep = 0.693147180559945309417 / kSteps;
    static constexpr float kC1 = (float)(kStep * 0x1p36), kC2 = (float)(kStep * kStep / 2 * 0x1p36),
                           kC3 = (float)(kStep * kStep * kStep / 6 * 0x1p36);
    __device__ __forceinline__ static mass_t mass(const mass_t *table, float t, float u)
    {
        const int n = __float_as_int(t);  // and 1.5 2^23, whose low 11 bits are 0
        const mass_t T = table[n & (kSteps - 1)];
        const mass_t m = T + (mass_t)((long long)(int)(T >> 36) * __float2int_rn(u));
        return m >> (62 - kUnitBits + (0x4b400000 >> 11) - (n >> 11));
    }
};

// Two entries' masses, of two rows or of one, with packed instructions: the same as RowShare's.
struct TwoShares {
    float2 khi, klo, magic, nf0, nbase, low;
    __device__ __forceinline__ TwoShares(const RowShare &a, const RowShare &b)
        : khi(make_float2(a.khi, b.khi)), klo(make_float2(a.klo, b.klo)),
          magic(make_float2(a.magic, b.magic)), nf0(make_float2(-a.f0, -b.f0)),
          nbase(make_float2(-a.base, -b.base)), low(make_float2(a.low, b.low))
    {
    }
    __device__ __forceinline__ float2 split(float2 z, float2 &t) const
    {
        float2 x = __fadd2_rn(z, nbase);
        x.x = fmaxf(x.x, low.x);
        x.y = fmaxf(x.y, low.y);
        t = __ffma2_rn(x, khi, magic);
        const float2 nw = __ffma2_rn(t, make_float2(-1.0f, -1.0f), magic);
        return __fadd2_rn(__ffma2_rn(x, khi, nw), __ffma2_rn(x, klo, nf0));
    }
    __device__ __forceinline__ static void masses(const mass_t *table, float2 t, float2 f,
                                                  mass_t &a, mass_t &b)
    {
        float2 u = __ffma2_rn(f, make_float2(RowShare::kC3, RowShare::kC3),
                              make_float2(RowShare::kC2, RowShare::kC2));
        u = __ffma2_rn(f, u, make_float2(RowShare::kC1, RowShare::kC1));
        u = __fmul2_rn(f, u);
        a = RowShare::mass(table, t.x, u.x);
        b = RowShare::mass(table, t.y, u.y);
    }
};

// T, to 2^-58 of itself: every step is the product of the roots 2^{1/2}, 2^{1/4}, ... of its bits,
// each the whole square root of the one before.
struct alignas(16) Steps {
    mass_t t[kSteps];
};
constexpr Steps exp2_steps()
{
    using wide = unsigned __int128;
    Steps s{};
    s.t[0] = 1ull << 62;
    mass_t root = 1ull << 63;
    for (int bit = kSteps / 2; bit > 0; bit >>= 1) {
        const wide square = (wide)root << 62;
        root = 0;
        for (int b = 62; b >= 0; --b) {
            const mass_t r = root | 1ull << b;
            root = (wide)r * r <= square ? r : root;
        }
        for (int i = bit; i < kSteps; i += 2 * bit) {
            // (the bits above are in s.t[i - bit] already)
            s.t[i] = (mass_t)((wide)s.t[i - bit] * root >> 62);
        }
    }
    return s;
}
__device__ const Steps kExp2Steps = exp2_steps();
__device__ inline void fill_table(mass_t *table)
{
    const ulonglong2 *from = reinterpret_cast<const ulonglong2 *>(kExp2Steps.t);
#pragma unroll
    for (int i = threadIdx.x; i < kSteps / 2; i += kVerifyThreads)
        reinterpret_cast<ulonglong2 *>(table)[i] = __ldg(from + i);
}

// What is left of p counts from 2^-32 on: below, it would be made of the masses' errors.
constexpr mass_t kLeastLeft = 1ull << (kUnitBits - 32);

// A segment's sums: of both rows' masses, of what is left of the first (P - Q, or P), and of Q
// where something is left; and the number of entries that are not in the last two, as their sign
// is not settled.  The masses of kListed of them are listed; with more, all entries are looked at
// again.
constexpr int kListed = 16;
struct Segment {
    mass_t p, q, left, q_left;
    mass_t undecided;
};

// A row of the request, its draft and what they come to.
struct Level {
    float m, s, md, sd;
    LogMass log, log1;  // of the target's mass at tau and at 1
    float u, zx, dx;    // the draft's number and logits
    int arg, id, state;
    RowShare p, q;
};

struct RequestShared {
    Level level[CIS_MAX_DRAFTS + 1];
    alignas(16) mass_t table[kSteps];
    mass_t warps[2][kWarps];
    mass_t rest;
    unsigned many[kWarps];        // segments whose entries are looked at again, and
    mass_t more[kVerifyThreads];  // what is left in them
    int undecided[kWarps];
    int seg, found, end, last;
};

// The rows that a token is drawn from.
template <typename InT> struct DrawRow {
    const InT *p, *q;  // q: null without a draft's row
    int V, id;         // the draft, or -1
    bool residual;     // something is taken off: q, or the draft itself
    int head, nvec;    // p's 16-byte vectors
    int segs;
    bool same;         // q's are the same

    __device__ __forceinline__ void enter(const InT *p_, const InT *q_, int V_, int id_, int segs_)
    {
        p = p_;
        q = q_;
        V = V_;
        id = id_;
        residual = id >= 0;
        segs = segs_;
        head = row_head(p, V);
        nvec = (V - head) / Vec<InT>::kN;
        same = q == nullptr ||
               ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) == 0;
    }
    // Segment s has the entries [start(s), start(s + 1)): a warp's whole turns, 32 vectors each, so
    // that all lanes have some (B=96, V=151936 without draft rows: 51 us for 54).
    __device__ __forceinline__ int start(int s) const
    {
        if (s == 0 || s >= segs)
            return s == 0 ? 0 : V;
        const int turn = (int)((int64_t)((nvec + 31) / 32) * s / segs);
        return head + min(nvec, 32 * turn) * Vec<InT>::kN;
    }
};

// One segment's sums, by one warp; every lane gets them.
template <typename InT, bool kPair>
__device__ __forceinline__ Segment add_segment(const DrawRow<InT> &row, const RowShare &mp,
                                               const RowShare &mq, const mass_t *table, int s,
                                               int *count, ulonglong2 *list)
{
    constexpr int EV = Vec<InT>::kN;
    const int lane = threadIdx.x & 31, j0 = row.start(s), j1 = row.start(s + 1);
    const TwoShares two(mp, mq);
    mass_t sp = 0, sq = 0, left = 0, q_left = 0;
    float least = INFINITY;  // the least distance of a sign from its border
    if (kPair) {
        if (lane == 0)
            *count = 0;
        __syncwarp();
    }
    // kPair: an entry of both rows; else two entries of one
    auto add = [&](float a, float b) {
        float2 t;
        const float2 f = two.split(make_float2(a, b), t);
        mass_t P, Q;
        TwoShares::masses(table, t, f, P, Q);
        if constexpr (kPair) {
            sp += P;
            sq += Q;
            // Y's difference: settled beyond 0.05 / 2048 of log2, 2^-15.8 (delta is below 12 E)
            const float gap = (t.x - t.y) + (f.x - f.y);
            if (gap > 0.05f) {
                left += P;
                q_left += Q;
            }
            least = fminf(least, fabsf(gap));
        } else {
            sp += P + Q;
        }
    };
    auto check = [&](int j) {  // lists entry j where its sign is not settled
        float2 t;
        const float2 f = two.split(make_float2(to_f32(row.p[j]), to_f32(row.q[j])), t);
        if (fabsf((t.x - t.y) + (f.x - f.y)) <= 0.05f) {
            mass_t P, Q;
            TwoShares::masses(table, t, f, P, Q);
            const int at = P != 0 ? atomicAdd(count, 1) : kListed;
            if (at < kListed)
                list[at] = make_ulonglong2(P, Q);
        }
    };
    int from = j0, to = j0;  // the vectors' entries
    if (row.same) {
        from = s == 0 ? row.head : j0;
        to = s == row.segs - 1 ? row.head + row.nvec * EV : j1;
        const uint4 *vp = reinterpret_cast<const uint4 *>(row.p + from);
        const uint4 *vq = reinterpret_cast<const uint4 *>(row.q + (kPair ? from : 0));
        const int n = (to - from) / EV;
        const uint4 none = make_uint4(0, 0, 0, 0);
        Vec<InT> x, y;
        uint4 nx = lane < n ? __ldg(vp + lane) : none, ny = none;
        if constexpr (kPair)
            ny = lane < n ? __ldg(vq + lane) : none;
#pragma unroll 1
        for (int v = lane; v < n; v += 32) {
            x.q = nx;
            y.q = ny;
            if (v + 32 < n) {
                nx = __ldg(vp + v + 32);
                if constexpr (kPair)
                    ny = __ldg(vq + v + 32);
            }
            if constexpr (kPair) {
#pragma unroll
                for (int e = 0; e < EV; ++e)
                    add(x.entry(e), y.entry(e));
                if (least <= 0.05f) {
                    least = INFINITY;
#pragma unroll 1
                    for (int e = 0; e < EV; ++e)
                        check(from + v * EV + e);
                }
            } else {
#pragma unroll
                for (int e = 0; e < EV; e += 2)
                    add(x.entry(e), x.entry(e + 1));
            }
        }
    }
    // the entries before and after them
    const int edge = (from - j0) + (j1 - to);
#pragma unroll 1
    for (int i = lane; i < edge; i += 32) {
        const int j = i < from - j0 ? j0 + i : to + (i - (from - j0));
        add(to_f32(row.p[j]), kPair ? to_f32(row.q[j]) : -INFINITY);
        if (kPair && least <= 0.05f) {
            least = INFINITY;
            check(j);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        sp += __shfl_xor_sync(0xffffffffu, sp, o);
        if constexpr (kPair) {
            sq += __shfl_xor_sync(0xffffffffu, sq, o);
            left += __shfl_xor_sync(0xffffffffu, left, o);
            q_left += __shfl_xor_sync(0xffffffffu, q_left, o);
        }
    }
    if constexpr (kPair) {
        __syncwarp();
        return {sp, sq, left - q_left, q_left, (mass_t)*count};
    } else {
        left = sp;
        if (row.residual && row.id >= j0 && row.id < j1)  // all but the draft
            left -= mp(table, to_f32(row.p[row.id]));
        return {sp, 0, left, 0, 0};
    }
}

// The sums of two numbers a thread over the CTA, in every thread.
__device__ __forceinline__ void cta_sums(mass_t &x, mass_t &y, mass_t (*warps)[kWarps])
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        x += __shfl_xor_sync(0xffffffffu, x, o);
        y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
        warps[0][threadIdx.x >> 5] = x;
        warps[1][threadIdx.x >> 5] = y;
    }
    __syncthreads();
    x = y = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        x += warps[0][i];
        y += warps[1][i];
    }
}
// The sum of the threads before this one, and of all.
__device__ __forceinline__ mass_t cta_before(mass_t x, mass_t *warps, mass_t &all)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    mass_t run = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const mass_t y = __shfl_up_sync(0xffffffffu, run, o);
        run += lane >= o ? y : 0;
    }
    __syncthreads();
    if (lane == 31)
        warps[w] = run;
    __syncthreads();
    run -= x;
    all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        run += i < w ? warps[i] : 0;
        all += warps[i];
    }
    return run;
}

template <typename InT>
__global__ void __launch_bounds__(kVerifyThreads, 4)
    cis_verify_requests_kernel(const __grid_constant__ VerifyArgs g)
{
    constexpr int NT = kVerifyThreads;
    __shared__ RequestShared sh;
    const int b = blockIdx.x / g.groups, rank = blockIdx.x - b * g.groups;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const Request r = request(g, b);
    const int64_t out = (int64_t)b * (g.D + 1);
    auto fill = [&](int from, int32_t id, float v) {  // slots from `from` on
        for (int i = from + tid; i <= g.D; i += NT) {
            g.tokens[out + i] = id;
            if (g.lp) g.lp[out + i] = v;
            if (g.lps) g.lps[out + i] = v;
        }
    };
    auto refuse = [&](int32_t bits) {
        fill(0, -1, NAN);
        if (tid == 0) {
            g.kept[b] = -1;
            set_status(g.status, bits);
        }
    };
    const InT *z0 = static_cast<const InT *>(g.z) + ((int64_t)r.a + b) * g.ld;
    const InT *d0 = g.zd ? static_cast<const InT *>(g.zd) + (int64_t)r.a * g.ldd : nullptr;
    // what the first kernel does not change (a draft's logits are on their way while the table is
    // filled)
    static_assert(CIS_MAX_DRAFTS < NT, "a thread a level");
    if (r.on && r.ok) {
        const int id = tid < r.n ? g.ids[r.a + tid] : -1;
        const float u = tid < r.n ? g.u[r.a + tid] : 0.0f;
        const bool in = id >= 0 && id < g.V;
        const float zx = in ? to_f32(z0[tid * g.ld + id]) : 0.0f;
        const float dx = in && r.model ? to_f32(d0[tid * g.ldd + id]) : 0.0f;
        if (!r.greedy)
            fill_table(sh.table);
        if (tid <= r.n) {
            Level &v = sh.level[tid];
            v.id = id;
            v.u = u;
            v.zx = zx;
            v.dx = dx;
        }
    }
    __syncthreads();
    grid_wait();
    if (!r.on || !r.ok) {  // as every CTA of the request finds
        if (rank == 0) {
            if (r.on) {
                refuse(kStatusBadInput);
            } else {
                fill(0, -1, 0.0f);
                if (tid == 0)
                    g.kept[b] = -1;
            }
        }
        return;
    }
    const Scale sc = device_scale(r.greedy ? 1.0f : r.tau);
    const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};

    // Every row's stretches together, a warp a row.
    for (int i = w; i <= r.n; i += kWarps) {
        const bool draft = r.model && i < r.n;
        const Scale sd = device_scale(draft ? r.tau_d : 1.0f);
        const Part *parts = g.parts + ((int64_t)r.a + b + i) * g.stretches;
        Part p[kMaxStretches / 32];
        float M = -INFINITY, Md = -INFINITY;
#pragma unroll
        for (int c = 0; c < kMaxStretches / 32; ++c) {
            p[c] = Part{-INFINITY, 0.0f, 0.0f, 0x7fffffff, -INFINITY, 0.0f, {0, 0}};
            if (lane + 32 * c < g.stretches)
                p[c] = parts[lane + 32 * c];
            M = fmaxf(M, p[c].m);
            Md = draft ? fmaxf(Md, p[c].md) : Md;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
            Md = fmaxf(Md, __shfl_xor_sync(0xffffffffu, Md, o));
        }
        float s = 0.0f, s1 = 0.0f, sq = 0.0f;
        int arg = 0x7fffffff;
#pragma unroll
        for (int c = 0; c < kMaxStretches / 32; ++c)
            if (lane + 32 * c < g.stretches) {
                s += p[c].s * share_of(p[c].m, M, sc);
                s1 += p[c].s1 * share_of(p[c].m, M, one);
                if (draft)
                    sq += p[c].sd * share_of(p[c].md, Md, sd);
                arg = p[c].m == M ? min(arg, p[c].arg) : arg;
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            s1 += __shfl_xor_sync(0xffffffffu, s1, o);
            sq += __shfl_xor_sync(0xffffffffu, sq, o);
            arg = min(arg, __shfl_xor_sync(0xffffffffu, arg, o));
        }
        // what follows of the sums, of the target's in lane 0 and of the draft's in lane 1
        Level &v = sh.level[i];
        const bool second = lane & 1;
        const float mass = second ? sq : s, top = second ? Md : M;
        RowShare share;
        share.set(top, second ? r.tau_d : r.greedy ? 1.0f : r.tau, second ? sd : sc, mass,
                  second ? RowShare::kDepth + 0.2f : RowShare::kDepth);
        // (2^-21 more than the sums)
        const float own = share_of(second ? v.dx : v.zx, top, second ? sd : sc) / mass;
        const float other = __shfl_sync(0xffffffffu, own, 1);
        const LogMass log = log_mass(second ? s1 : s);  // (lane 1: at temperature 1)
        if (lane == 1) {
            v.q = share;
            v.log1 = log;
        }
        if (lane == 0) {
            v.p = share;
            v.log = log;
            v.m = M;
            v.s = s;
            v.md = Md;
            v.sd = sq;
            v.arg = arg;
            v.state = kAccept;
            if (!(s > 0.0f && s < INFINITY) || !(fabsf(M) < INFINITY) ||
                !(v.u >= 0.0f && v.u < 1.0f) ||
                (draft && (!(sq > 0.0f && sq < INFINITY) || !(fabsf(Md) < INFINITY)))) {
                v.state = kBadRow;
            } else if (i < r.n && (v.id < 0 || v.id >= g.V)) {
                v.state = kBadDraft;
            } else if (i < r.n && r.greedy) {
                v.state = v.id == arg ? kAccept : kReject;
            } else if (i < r.n) {
                // (where fp32 has no such number the draft is left open too)
                const float px = own, uq = draft ? v.u * other : v.u, most = fmaxf(px, uq);
                v.state = fabsf(px - uq) > 0x1p-16f * most && most > 1e-30f
                              ? (uq < px ? kAccept : kReject)
                              : kOpen;
            }
        }
    }
    __syncthreads();

    int k = 0;
    auto advance = [&] {  // to the next row that decides something
        while (sh.level[k].state == kAccept && k < r.n)
            ++k;
        return sh.level[k].state;
    };
    int state = advance();
    auto finish = [&](int32_t token, float z) {  // every thread
        if (state == kBadRow || state == kBadDraft) {
            refuse(state == kBadRow ? kStatusBadInput : kStatusBadId);
            return;
        }
        static_assert(2 * CIS_MAX_DRAFTS < NT, "a thread a log-probability");
        const int i = tid & (NT / 2 - 1);
        if (i <= k) {
            const Level &v = sh.level[i];
            const float x = i < k ? v.zx : z;
            if (tid == i) {
                g.tokens[out + i] = i < k ? v.id : token;
                if (g.lp) g.lp[out + i] = log_prob(x, v.m, one, v.log1);
            } else if (g.lps) {
                g.lps[out + i] = r.greedy ? 0.0f : log_prob(x, v.m, sc, v.log);
            }
        }
        fill(k + 1, -1, 0.0f);
        if (tid == 0)
            g.kept[b] = k;
    };
    if (r.greedy || state == kBadRow || state == kBadDraft) {
        if (rank == 0)
            finish(sh.level[k].arg, sh.level[k].m);
        return;
    }

    // The row's masses, a warp a segment.
    const int segs = g.segments, own_segs = segs / g.groups;
    Segment *mine = g.segs + (int64_t)b * segs;
    ulonglong2 *undecided = g.undecided + (int64_t)b * segs * kListed;
    DrawRow<InT> row;
    auto enter = [&] {
        const Level &v = sh.level[k];
        row.enter(z0 + k * g.ld, v.id >= 0 && r.model ? d0 + k * g.ldd : nullptr, g.V, v.id, segs);
    };
    auto sums = [&](int from, int to) {
        const RowShare mp = sh.level[k].p, mq = sh.level[k].q;
        for (int s = from + w; s < to; s += kWarps) {
            ulonglong2 *list = undecided + (int64_t)s * kListed;
            int *count = &sh.undecided[w];
            const Segment a =
                row.q && row.residual
                    ? add_segment<InT, true>(row, mp, mq, sh.table, s, count, list)
                    : add_segment<InT, false>(row, mp, mp, sh.table, s, count, list);
            __syncwarp();
            if (lane == 0)
                mine[s] = a;
        }
    };
    enter();
    sums(rank * own_segs, (rank + 1) * own_segs);
    if (g.groups > 1) {  // the request's last CTA goes on
        __threadfence();
        __syncthreads();
        if (tid == 0)
            sh.last = atomicAdd(&g.tickets[b], 1u) == (unsigned)g.groups - 1;
        __syncthreads();
        if (!sh.last)
            return;
        __threadfence();
    } else {
        __syncthreads();
    }
    bool minus = false;
    mass_t delta = 0, left = 0;
    auto off = [&](mass_t Q) {  // Q (1 + delta)
        const mass_t x = __umul64hi(Q, delta);
        return minus ? Q - x : Q + x;
    };
    RowShare sp_of, sq_of;  // level k's
    auto mass_of = [&](int j, float z, float d) -> mass_t {
        const mass_t P = sp_of(sh.table, z);
        if (!row.residual)
            return P;
        if (!row.q)
            return j == row.id ? 0 : P;
        const mass_t Q = off(sq_of(sh.table, d));
        return P > Q ? P - Q : 0;
    };
    auto mass = [&](int j) {
        return mass_of(j, to_f32(row.p[j]), row.q ? to_f32(row.q[j]) : 0.0f);
    };
    const float u_last = g.u_last[b];
    auto four = [&](const int (&j)[4]) {  // the masses of four entries (-1: none)
        float z[4], d[4];
        mass_t sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = j[i] >= 0 ? to_f32(row.p[j[i]]) : -INFINITY;
            d[i] = j[i] >= 0 && row.q ? to_f32(row.q[j[i]]) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sum += mass_of(j[i], z[i], d[i]);
        return sum;
    };
    // (where decreasing offsets make two requests share a row their sums may not be its own: then
    // too every index stays in the row, and the loops end)
    for (;;) {
        Segment a = {};
        if (tid == 0) {
            sh.seg = 0;
            sh.rest = 0;
        }
        ulonglong2 listed = make_ulonglong2(0, 0);  // the first of its list, if there is one
        if (tid < segs) {
            a = Segment{__ldcg(&mine[tid].p), __ldcg(&mine[tid].q), __ldcg(&mine[tid].left),
                        __ldcg(&mine[tid].q_left), __ldcg(&mine[tid].undecided)};
            listed = __ldcg(undecided + (int64_t)tid * kListed);
        }
        mass_t sp = a.p, sq = a.q;
        cta_sums(sp, sq, sh.warps);
        if (!(row.q && row.residual))
            sq = 1ull << kUnitBits;
        if (state == kOpen) {  // (rare: what follows is left to this CTA)
            if (tid == 0) {
                // p(x) = e^{(z - M) / tau} 2^-{unit / 2048} 2^60 / SP, and q's likewise
                Level &v = sh.level[k];
                auto share = [](float z, float M, float tau, float unit, mass_t sum) {
                    return exp(((double)z - (double)M) / (double)tau -
                               (double)unit * (0.693147180559945309417 / kSteps)) *
                           ((double)(1ull << kUnitBits) / (double)sum);
                };
                const double P = share(v.zx, v.m, r.tau, v.p.unit, sp);
                const double Q = row.q ? share(v.dx, v.md, r.tau_d, v.q.unit, sq) : 1.0;
                v.state = (double)v.u * Q < P ? kAccept : kReject;
            }
            __syncthreads();  // (of sh.level)
            const int was = k;
            state = advance();
            if (state == kBadRow || state == kBadDraft) {
                finish(-1, 0.0f);
                return;
            }
            if (k != was) {
                enter();
                sums(0, segs);
                __syncthreads();
                continue;
            }
        }
        sp_of = sh.level[k].p;
        sq_of = sh.level[k].q;
        left = a.left;
        if (row.q && row.residual) {
            // SP / SQ - 1 in units of 2^-64: to fp32, and then what that leaves
            minus = sp < sq;
            const mass_t gap = minus ? sq - sp : sp - sq;
            const float inv = 0x1p64f / (float)sq;
            delta = __float2ull_rz((float)gap * inv);
            delta += (mass_t)__float2ll_rn((float)(long long)(gap - __umul64hi(delta, sq)) * inv);
            const mass_t x = __umul64hi(a.q_left, delta);
            left = minus ? left + x : left - x;
            // the entries that were undecided, a thread a segment; where there were too many, all
            // of them, a warp a segment.  All of them too where the sum is less than the roundings of
            // its entries, a unit each: x is rounded once and an entry's Q delta for itself, so that it
            // can be below 0, or above it where no entry has a mass (flat rows that are nearly equal,
            // some 10^4 units an entry).
            const int n = (int)a.undecided;
            const bool again =
                n > kListed || (x != 0 && (long long)left < g.V / segs + 66 * Vec<InT>::kN);
            const unsigned many = __ballot_sync(0xffffffffu, again);
            auto settled = [&](const ulonglong2 &e) {
                const mass_t Q = off(e.y);
                return e.x > Q ? e.x - Q : 0;
            };
            if (!again) {
                left += n > 0 ? settled(listed) : 0;
                for (int i = 1; i < n; i += 3) {  // (kListed is 1 more than a multiple of 3)
                    const ulonglong2 *at = undecided + (int64_t)tid * kListed + i;
                    const ulonglong2 e0 = __ldcg(at), e1 = __ldcg(at + 1), e2 = __ldcg(at + 2);
                    left += settled(e0);
                    left += i + 1 < n ? settled(e1) : 0;
                    left += i + 2 < n ? settled(e2) : 0;
                }
            }
            if (lane == 0)
                sh.many[w] = many;
            __syncthreads();
            for (int i = 0; i < kWarps; ++i)
                for (unsigned bits = sh.many[i]; bits; bits &= bits - 1) {
                    const int s = 32 * i + __ffs(bits) - 1;
                    if (s % kWarps != w)
                        continue;
                    mass_t own = 0;
                    const int e = row.start(s + 1);
                    for (int j0 = row.start(s) + lane; j0 < e; j0 += 128) {
                        const int j[4] = {j0, j0 + 32 < e ? j0 + 32 : -1, j0 + 64 < e ? j0 + 64 : -1,
                                          j0 + 96 < e ? j0 + 96 : -1};
                        own += four(j);
                    }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
                        own += __shfl_xor_sync(0xffffffffu, own, o);
                    if (lane == 0)
                        sh.more[s] = own;
                }
            __syncthreads();
            if (again)
                left = sh.more[tid];
        }
        mass_t R, none;
        const mass_t before = cta_before(left, sh.warps[0], R);
        if (R > (row.residual ? kLeastLeft : 0)) {
            // The segment, and in it a thread's part.
            const mass_t goal = __umul64hi(R, __float2ull_rz(u_last * 0x1p64f));  // (below R)
            if (before <= goal && goal < before + left) {
                sh.seg = tid;
                sh.rest = goal - before;
            }
            if (tid == 0)
                sh.end = sh.found = -1;
            __syncthreads();
            const mass_t rest = sh.rest;
            const int s0 = row.start(sh.seg), s1 = row.start(sh.seg + 1);
            const int per = (s1 - s0 + NT - 1) / NT;
            const int a0 = min(s1, s0 + tid * per), a1 = min(s1, a0 + per);
            mass_t own = 0;
            int end = -1;  // the last entry with a mass
            mass_t m[4];  // of the last four
            for (int j = a0; j < a1; j += 4) {
                float z[4], d[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = j + i < a1 ? to_f32(row.p[j + i]) : -INFINITY;
                    d[i] = j + i < a1 && row.q ? to_f32(row.q[j + i]) : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    m[i] = mass_of(j + i, z[i], d[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    own += m[i];
                    end = m[i] ? j + i : end;
                }
            }
            atomicMax(&sh.end, end);
            mass_t at = cta_before(own, sh.warps[1], none);
            const bool mine_it = at <= rest && rest < at + own;
            if (mine_it && per <= 4) {
                int i = 0;
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    at += m[e];
                    i += at <= rest;
                }
                sh.found = a0 + i;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, mine_it && per > 4);
            if (hit) {  // the thread's entries, over its warp
                const int src = __ffs(hit) - 1, e = __shfl_sync(0xffffffffu, a1, src);
                int j = __shfl_sync(0xffffffffu, a0, src);
                mass_t passed = __shfl_sync(0xffffffffu, at, src);
                for (; j < e; j += 32) {
                    mass_t run = j + lane < e ? mass(j + lane) : 0;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const mass_t y = __shfl_up_sync(0xffffffffu, run, o);
                        run += lane >= o ? y : 0;
                    }
                    const unsigned over = __ballot_sync(0xffffffffu, passed + run > rest);
                    if (over) {
                        if (lane == 0)
                            sh.found = j + __ffs(over) - 1;
                        break;
                    }
                    passed += __shfl_sync(0xffffffffu, run, 31);
                }
            }
            __syncthreads();
            // (a segment's sum and its entries' are off from each other by their roundings, a unit
            // each: beyond the last entry it is that one)
            const int j = sh.found >= 0 ? sh.found : sh.end;
            if (j >= 0) {
                finish(j, to_f32(row.p[j]));
                return;
            }
        }
        if (!row.residual) {
            state = kBadRow;
            finish(-1, 0.0f);
            return;
        }
        // p is q: the whole of p
        row.residual = false;
        __syncthreads();
        sums(0, segs);
        __syncthreads();
    }
}

// A row's stretches: as many warps in all as the SMs hold at a time, 256 vectors each at least.
constexpr int64_t kSms = 152, kMostRowWarps = kRowCtas<float> * kWarps * kSms;
template <typename InT> int stretches_of(int64_t rows, int64_t V)
{
    const int64_t nvec = V * (int64_t)sizeof(InT) / 16;
    int64_t c = kRowCtas<InT> * kWarps * kSms / rows;
    c = c < nvec / 256 ? c : nvec / 256;
    c = c < kMaxStretches ? c : kMaxStretches;
    return c < 1 ? 1 : (int)c;
}

// The second kernel's CTAs a request: four an SM in all, eight where entries are of two rows (the
// first requests' tokens are drawn while others are added up: B=64, 4 drafts, V=151936: 80 us for 81;
// B=128, V=32003 fp32: 70 for 73; without the draft's rows, B=96: 55 for 51), 256 entries a segment
// at least, and no more segments than a CTA has threads.
int groups_of(int64_t B, int64_t V, bool two)
{
    int64_t c = (two ? 1216 : 608) / B;
    c = c < V / (256 * kWarps) ? c : V / (256 * kWarps);
    c = c < kVerifyThreads / kWarps ? c : kVerifyThreads / kWarps;
    return c < 1 ? 1 : (int)c;
}

// Their segments: a multiple of the groups' warps, of 1024 entries at most where that many fit a
// CTA's threads.
int segments_of(int64_t V, int groups)
{
    const int step = groups * kWarps, most = kVerifyThreads / step * step;
    const int64_t want = (V + 1023) / 1024, up = (want + step - 1) / step * step;
    return (int)(up < most ? up : most);
}

struct VerifyLayout {
    size_t segs, undecided, tickets, total;
};
VerifyLayout verify_layout(int64_t B, int64_t V, int32_t D)
{
    VerifyLayout l;
    // (rows times their stretches: no more than the warps, or the rows)
    l.segs = ws_round_up((size_t)(B * (D + 1) + kMostRowWarps) * sizeof(Part));
    const int one = segments_of(V, groups_of(B, V, false));
    const int two = segments_of(V, groups_of(B, V, true));  // (may be fewer)
    const size_t n = (size_t)B * (one > two ? one : two);
    l.undecided = l.segs + ws_round_up(n * sizeof(Segment));
    l.tickets = l.undecided + ws_round_up(n * kListed * sizeof(ulonglong2));
    l.total = l.tickets + ws_round_up((size_t)B * sizeof(uint32_t));
    return l;
}

template <typename InT> cudaError_t launch_verify(const VerifyArgs &g, cudaStream_t s)
{
    const int64_t rows = (int64_t)g.B * (g.zd ? 2 * g.D + 1 : g.D + 1);
    // The second kernel's CTAs start beside the first one's: they need the shared memory that an SM
    // would else have given to its L1 (on the few SMs that were free they took 20,000 cycles for a
    // request of V=151936, for 7,500).
    cudaError_t e = cudaFuncSetAttribute(cis_verify_rows_kernel<InT>,
                                         cudaFuncAttributePreferredSharedMemoryCarveout, 60);
    if (e != cudaSuccess)
        return e;
    cis_verify_rows_kernel<InT>
        <<<(unsigned)((rows * g.stretches + kWarps - 1) / kWarps), kVerifyThreads, 0, s>>>(g);
    e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(g.B * g.groups));
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, cis_verify_requests_kernel<InT>, g);
    return e != cudaSuccess ? e : cudaGetLastError();
}

bool verify_sizes_ok(int64_t B, int64_t V, int32_t D)
{
    return B >= 0 && V > 0 && V <= 0x7fffffffLL && D >= 0 && D <= CIS_MAX_DRAFTS &&
           B <= (1 << 20);
}

}  // namespace
}  // namespace cis

using namespace cis;

extern "C" CIS_API cis_status_t cis_verify_workspace_size(int64_t B, int64_t V, int32_t max_drafts,
                                                          size_t *bytes)
{
    if (bytes == nullptr || !verify_sizes_ok(B, V, max_drafts))
        return CIS_ERR_INVALID_ARG;
    const int64_t n = B > 0 ? B : 1;
    *bytes = verify_layout(n, V, max_drafts).total;
    return CIS_OK;
}

extern "C" CIS_API cis_status_t cis_verify_tokens(
    const void *logits, int32_t dtype, int64_t B, int64_t N, int64_t V, int64_t ld,
    const int32_t *draft_ids, const int32_t *cu_drafts, int32_t max_drafts,
    const void *draft_logits, int64_t ld_draft, const float *u, const float *u_last,
    const float *temperature, const float *draft_temperature, const uint8_t *mask,
    int32_t *tokens_out, int32_t *kept_out, float *lp_out, float *lp_sampled_out,
    int32_t *dev_status, void *workspace, size_t workspace_bytes, void *stream)
{
    NvtxRange nvtx_range("cis_verify_tokens");
    size_t need = 0;
    if (cis_verify_workspace_size(B, V, max_drafts, &need) != CIS_OK || N < 0 ||
        N > B * (int64_t)max_drafts || !row_args_ok(logits, dtype, N + B, V, ld) ||
        (draft_logits != nullptr && !row_args_ok(draft_logits, dtype, N, V, ld_draft)) ||
        !aligned4(draft_ids, cu_drafts, u, u_last, temperature, draft_temperature, tokens_out,
                  kept_out, lp_out, lp_sampled_out, dev_status))
        return CIS_ERR_INVALID_ARG;
    if (B == 0)
        return CIS_OK;
    if (logits == nullptr || cu_drafts == nullptr || u_last == nullptr || tokens_out == nullptr ||
        kept_out == nullptr || (N > 0 && (draft_ids == nullptr || u == nullptr)) ||
        (lp_out != nullptr && lp_out == lp_sampled_out) || workspace == nullptr ||
        workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
        return CIS_ERR_INVALID_ARG;
    if (V > kMaxRowEntries)
        return CIS_ERR_UNSUPPORTED;
    VerifyArgs g = {};
    g.z = logits;
    g.zd = draft_logits;
    g.ld = ld;
    g.ldd = ld_draft;
    g.B = (int)B;
    g.D = max_drafts;
    g.V = (int)V;
    g.N = N;
    g.ids = draft_ids;
    g.cu = cu_drafts;
    g.u = u;
    g.u_last = u_last;
    g.tau = temperature;
    g.tau_d = draft_temperature;
    g.mask = mask;
    g.tokens = tokens_out;
    g.kept = kept_out;
    g.lp = lp_out;
    g.lps = lp_sampled_out;
    g.status = dev_status;
    const int64_t rows = N * (draft_logits ? 2 : 1) + B;
    g.stretches = dtype == CIS_BF16 ? stretches_of<__nv_bfloat16>(rows, V)
                                    : stretches_of<float>(rows, V);
    g.groups = groups_of(B, V, draft_logits != nullptr);
    g.segments = segments_of(V, g.groups);
    const VerifyLayout l = verify_layout(B, V, max_drafts);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    g.parts = reinterpret_cast<Part *>(ws);
    g.segs = reinterpret_cast<Segment *>(ws + l.segs);
    g.undecided = reinterpret_cast<ulonglong2 *>(ws + l.undecided);
    g.tickets = reinterpret_cast<uint32_t *>(ws + l.tickets);
    const cudaError_t e = dtype == CIS_BF16 ? launch_verify<__nv_bfloat16>(g, (cudaStream_t)stream)
                                            : launch_verify<float>(g, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
