// cis_verify.cu -- verification of drafted tokens against the target's probabilities, from given
// uniform numbers (cis_verify_tokens).
//
// Per request, with p_i = softmax(z_i / tau) of the target's rows, q_i the distribution that draft
// x_i came from, in order:  x_i is kept where u_i q_i(x_i) < p_i(x_i).  After the first one that
// is not, at i, the request's last token is drawn from max(p_i - q_i, 0); after the last draft,
// from the target's next row.  At temperature 0 p is all on the row's first largest entry.
//
// Two kernels.  The first reads every row once, a row's stretches on CTAs of their own: maximum
// and sums of exponentials at tau and at 1.  In the second a cluster has a request: it puts the
// stretches together, goes through the drafts, and draws the last token.  Sums of fp32
// exponentials decide a draft only where their error cannot matter: with E = 2^-20 a sum is off by
// less than 6 E of itself (cis_sample.cu), so that p and u q farther apart than 16 E of the larger
// are in the order they seem.  Else the draft, and in any case the last token, is decided by whole
// numbers, masses e^{(z - M) / tau} / S in units of 2^-60 right to 2^-42 of each, S the sum that
// the first kernel found: what S is off by is common to a row, and the exact sums of both rows'
// masses take it out again.  Sums of whole numbers depend on no order.
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
    Part *parts;  // [D + 1][B][chunks]
    int chunks;
};

constexpr int kVerifyThreads = 256;
constexpr int kMaxChunks = 32;  // a lane each

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
// The log-probability of z: (z - M) / tau - log of the row's mass; at most 0, whatever the mass's
// roundings.
__device__ __forceinline__ float log_prob(float z, float M, const Scale &sc, float mass)
{
    float l, e;
    const float x = scaled_diff(z, M, sc, l), ls = logf(mass);
    const float u = two_sum(x, -ls, e);
    return fminf(u + (e + l - log_residual(mass, ls)), 0.0f);
}

template <typename InT, int kB> using Pass = RowPass<InT, kVerifyThreads, kB>;

// One row's stretch: its maximum and sum at sc, and with `two` that at 1.
template <typename InT, int kB>
__device__ __forceinline__ MaxSumU stretch(PassShared<kVerifyThreads> &sh, Pass<InT, kB> &ps,
                                           const Scale &sc, bool two, float &s1)
{
    ExpAcc<false, true> acc;
    acc.k = sc.kappa;
    acc.h = sc.huge;
    ExpAcc<false> raw;
    auto entry = [&](auto &e, float z) {
        e.raise(z);
        if (e.m != -INFINITY)
            e.add_entry(z);
    };
    ps.stream(
        false,
        [&](const Vec<InT> (&x)[kB], float mx) {
            take<false, kB>(acc, x, mx);
            if (two)
                take<false, kB>(raw, x, mx);
        },
        [&](float z) {
            entry(acc, z);
            if (two)
                entry(raw, z);
        });
    const MaxSumU o = block_exp<kVerifyThreads>(acc, sh.red);
    s1 = two ? block_exp<kVerifyThreads>(raw, sh.red2).s : o.s;
    return o;
}

template <typename InT, int kB>
__global__ void __launch_bounds__(kVerifyThreads)
    cis_verify_rows_kernel(const __grid_constant__ VerifyArgs g)
{
    constexpr int NT = kVerifyThreads, EV = Vec<InT>::kN;
    __shared__ PassShared<NT> sh;
    __shared__ int first;
    if (threadIdx.x == 0)
        allow_next_grid();
    const int c = blockIdx.x % g.chunks, item = blockIdx.x / g.chunks;
    const int i = item / g.B, b = item % g.B;
    const Request r = request(g, b);
    if (!r.on || !r.ok || i > r.n)
        return;
    const InT *row = static_cast<const InT *>(g.z) + ((int64_t)r.a + b + i) * g.ld;
    const Scale sc = device_scale(r.greedy ? 1.0f : r.tau);
    Part out = {};
    Pass<InT, kB> ps(row, g.V, c, g.chunks, nullptr);
    const MaxSumU o = stretch<InT, kB>(sh, ps, sc, g.lp && sc.hi != 1.0f, out.s1);
    out.m = o.m;
    out.s = o.s;
    if (r.greedy) {  // (read again, from L2)
        if (threadIdx.x == 0)
            first = 0x7fffffff;
        __syncthreads();
        int at = 0x7fffffff;
        for (int v = ps.v0 + threadIdx.x; v < ps.v1; v += NT) {
            Vec<InT> x[1];
            x[0].q = __ldg(ps.rv + v);
            if (vec_max<1>(x) == o.m) {
#pragma unroll
                for (int e = EV - 1; e >= 0; --e)
                    at = x[0].entry(e) == o.m ? ps.head + v * EV + e : at;
                break;
            }
        }
        if (ps.end >= 0 && ps.zend == o.m)
            at = min(at, ps.end);
        if (at != 0x7fffffff)
            atomicMin(&first, at);
        __syncthreads();
        out.arg = first;
    }
    if (r.model && i < r.n) {
        __syncthreads();
        Pass<InT, kB> pd(static_cast<const InT *>(g.zd) + ((int64_t)r.a + i) * g.ldd, g.V, c,
                         g.chunks, nullptr);
        float unused;
        const MaxSumU d = stretch<InT, kB>(sh, pd, device_scale(r.tau_d), false, unused);
        out.md = d.m;
        out.sd = d.s;
    }
    if (threadIdx.x == 0)
        g.parts[((int64_t)i * g.B + b) * g.chunks + c] = out;
}

// ------------------------------------------------------------------ the request
enum : int { kAccept = 0, kReject = 1, kOpen = 2, kBadRow = 3, kBadDraft = 4 };
struct Level {
    double px, qx;  // p and q at the draft, by the first kernel's sums
    float m, s, s1, md, sd, zx;
    int arg, id, state;
};

// e^{(z - M) / tau - L} in units of 2^-60: right to 2^-42 of itself, 0 below e^-41.
constexpr int kUnitBits = 60;
struct ShareMass {
    Scale sc;
    float M, hi, lo;  // L = hi + lo
    __device__ __forceinline__ mass_t operator()(float z) const
    {
        float dl, e, r;
        const float d = sum_pair(z, -M, dl), x = d * sc.hi;
        const float y = sum_pair(x, -hi, e);
        if (!(y > -41.0f))
            return 0;
        const float yl = fmaf(d, sc.hi, -x) + fmaf(d, sc.lo, dl * sc.hi) + (e - lo);
        int n;
        const float s = exp_parts(y, yl, r, n);
        const long long v = ((long long)__float2uint_rn(s * 0x1p24f) << 24) +
                            (long long)__float2int_rn(r * 0x1p48f);
        const int up = kUnitBits - 48 + (n >> 5);  // 13 .. -48
        return up >= 0 ? (mass_t)v << up : (mass_t)((v + (1ll << (-up - 1))) >> -up);
    }
};

struct RequestShared {
    Level level[CIS_MAX_DRAFTS + 1];
    ShareMass p, q;
    mass_t sums[2][kMaxCluster][2];        // the CTAs' sums, in turn
    mass_t warps[2][kVerifyThreads / 32];  // this CTA's warps'
    mass_t scan_w[kVerifyThreads / 32];
    mass_t goal, delta;
    int minus, state;
};

template <typename InT> struct RequestRow {
    const InT *p, *q;  // q: null where the draft's distribution is all on it
    int id;            // -1: no draft (nothing is taken off)
};

// Entries [j0, j1), every `step`-th from j0 on: f(entry, target's value, draft's value).
template <typename InT, typename F>
__device__ __forceinline__ void entries(const RequestRow<InT> &r, int j0, int j1, int step, F f)
{
    constexpr int kAhead = 4;
#pragma unroll 1
    for (int j = j0; j < j1; j += kAhead * step) {
        float z[kAhead], d[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool in = j + k * step < j1;
            z[k] = in ? to_f32(r.p[j + k * step]) : -INFINITY;
            d[k] = in && r.q ? to_f32(r.q[j + k * step]) : -INFINITY;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (j + k * step < j1)
                f(j + k * step, z[k], d[k]);
    }
}

// The sums of two numbers a thread over the cluster, in every thread; sh.sums[turn] has the CTAs',
// sh.warps this CTA's warps'.  The two buffers in turn: whoever writes one for the next time but
// one has passed the barrier before which the others read it.
__device__ inline void cluster_sums(RequestShared &sh, unsigned rank, unsigned cs, int &turn,
                                    mass_t a, mass_t b, mass_t &A, mass_t &Bs)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    turn ^= 1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    __syncthreads();
    if (lane == 0) {
        sh.warps[0][w] = a;
        sh.warps[1][w] = b;
    }
    __syncthreads();
    if (threadIdx.x < cs) {
        mass_t s0 = 0, s1 = 0;
        for (int i = 0; i < kVerifyThreads / 32; ++i) {
            s0 += sh.warps[0][i];
            s1 += sh.warps[1][i];
        }
        mass_t *to = cg::this_cluster().map_shared_rank(&sh.sums[turn][rank][0], (int)threadIdx.x);
        to[0] = s0;
        to[1] = s1;
    }
    cluster_sync_data();
    A = Bs = 0;
    for (unsigned c = 0; c < cs; ++c) {
        A += sh.sums[turn][c][0];
        Bs += sh.sums[turn][c][1];
    }
}

template <typename InT>
__global__ void __launch_bounds__(kVerifyThreads)
    cis_verify_requests_kernel(const __grid_constant__ VerifyArgs g, unsigned cs)
{
    constexpr int NT = kVerifyThreads, W = NT / 32;
    __shared__ RequestShared sh;
    const int b = blockIdx.x / cs, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const unsigned rank = blockIdx.x - b * cs;
    const Request r = request(g, b);
    const int64_t out = (int64_t)b * (g.D + 1);
    auto fill = [&](int from, int32_t id, float v) {  // slots from `from` on
        if (rank == 0)
            for (int i = from + tid; i <= g.D; i += NT) {
                g.tokens[out + i] = id;
                if (g.lp) g.lp[out + i] = v;
                if (g.lps) g.lps[out + i] = v;
            }
    };
    auto refuse = [&](int32_t bits) {
        fill(0, -1, NAN);
        if (rank == 0 && tid == 0) {
            g.kept[b] = -1;
            set_status(g.status, bits);
        }
    };
    grid_wait();
    if (!r.on || !r.ok) {  // as every CTA of the cluster finds
        if (r.on) {
            refuse(kStatusBadInput);
        } else {
            fill(0, -1, 0.0f);
            if (rank == 0 && tid == 0)
                g.kept[b] = -1;
        }
        return;
    }
    cluster_sync_data();  // every CTA of the cluster has started
    const Scale sc = device_scale(r.greedy ? 1.0f : r.tau);
    const Scale sd = device_scale(r.model ? r.tau_d : 1.0f);
    const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};
    const InT *z0 = static_cast<const InT *>(g.z) + ((int64_t)r.a + b) * g.ld;
    const InT *d0 = g.zd ? static_cast<const InT *>(g.zd) + (int64_t)r.a * g.ldd : nullptr;

    // Every row's stretches together, a warp a row.
    for (int i = w; i <= r.n; i += W) {
        const bool in = lane < g.chunks, draft = r.model && i < r.n;
        Part p = {};
        p.m = p.md = -INFINITY;
        if (in)
            p = g.parts[((int64_t)i * g.B + b) * g.chunks + lane];
        float M = p.m, Md = p.md;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
            Md = fmaxf(Md, __shfl_xor_sync(0xffffffffu, Md, o));
        }
        float s = in ? p.s * share_of(p.m, M, sc) : 0.0f;
        float s1 = in ? p.s1 * share_of(p.m, M, one) : 0.0f;
        float sq = in && draft ? p.sd * share_of(p.md, Md, sd) : 0.0f;
        int arg = in && p.m == M ? p.arg : 0x7fffffff;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            s1 += __shfl_xor_sync(0xffffffffu, s1, o);
            sq += __shfl_xor_sync(0xffffffffu, sq, o);
            arg = min(arg, __shfl_xor_sync(0xffffffffu, arg, o));
        }
        if (lane == 0) {
            Level v = {0.0, 1.0, M, s, s1, Md, sq, 0.0f, arg, -1, kAccept};
            const float u = i < r.n ? g.u[r.a + i] : 0.0f;
            if (!(s > 0.0f && s < INFINITY) || !(fabsf(M) < INFINITY) ||
                !(u >= 0.0f && u < 1.0f) ||
                (draft && (!(sq > 0.0f && sq < INFINITY) || !(fabsf(Md) < INFINITY)))) {
                v.state = kBadRow;
            } else if (i < r.n) {
                v.id = g.ids[r.a + i];
                if (v.id < 0 || v.id >= g.V) {
                    v.state = kBadDraft;
                } else {
                    v.zx = to_f32(z0[i * g.ld + v.id]);
                    if (r.greedy) {
                        v.state = v.id == arg ? kAccept : kReject;
                    } else {
                        v.px = exp(((double)v.zx - (double)M) / (double)r.tau) / (double)s;
                        if (draft)
                            v.qx = exp(((double)to_f32(d0[i * g.ldd + v.id]) - (double)Md) /
                                       (double)r.tau_d) / (double)sq;
                        const double uq = (double)u * v.qx;
                        v.state = fabs(v.px - uq) > 0x1p-16 * fmax(v.px, uq)
                                      ? (uq < v.px ? kAccept : kReject)
                                      : (v.px > 0.0 ? kOpen : kReject);
                    }
                }
            }
            sh.level[i] = v;
        }
    }
    __syncthreads();

    RequestRow<InT> row = {z0, nullptr, -1};
    const int j0 = (int)((int64_t)g.V * (rank * W + w) / (cs * W));
    const int j1 = (int)((int64_t)g.V * (rank * W + w + 1) / (cs * W));
    int turn = 0;
    // Level i's rows, and their masses.
    auto enter = [&](int i) {
        const Level &v = sh.level[i];
        row.p = z0 + i * g.ld;
        row.id = v.id;
        row.q = v.id >= 0 && r.model ? d0 + i * g.ldd : nullptr;
        __syncthreads();
        if (tid == 0 || tid == 32) {
            const double L = log((double)(tid == 0 ? v.s : row.q ? v.sd : 1.0f));
            const float hi = (float)L;
            ShareMass m = {sc, v.m, hi, (float)(L - (double)hi)};
            if (tid == 0) {
                sh.p = m;
            } else {
                m.sc = sd;
                m.M = v.md;
                sh.q = m;
            }
        }
        __syncthreads();
    };
    // The sums of both rows' masses, in every thread (without a draft's row the second is 2^60).
    auto both_sums = [&](mass_t &sp, mass_t &sq) {
        mass_t a = 0, c = 0;
        const ShareMass mp = sh.p, mq = sh.q;
        entries(row, j0 + lane, j1, 32, [&](int, float z, float d) {
            a += mp(z);
            if (row.q)
                c += mq(d);
        });
        cluster_sums(sh, rank, cs, turn, a, c, sp, sq);
        if (!row.q)
            sq = 1ull << kUnitBits;
    };

    int k = 0, state = kAccept, summed = -1;
    mass_t sp = 0, sq = 0;
    for (;; ++k) {
        state = sh.level[k].state;
        if (state == kOpen) {
            enter(k);
            both_sums(sp, sq);
            summed = k;
            if (tid == 0) {
                const Level &v = sh.level[k];
                sh.state = (double)g.u[r.a + k] * v.qx * (double)sp < v.px * (double)sq ? kAccept
                                                                                       : kReject;
            }
            __syncthreads();
            state = sh.state;
        }
        if (state != kAccept || k == r.n)
            break;
    }
    if (state == kBadRow || state == kBadDraft) {
        refuse(state == kBadRow ? kStatusBadInput : kStatusBadId);
        cluster_sync_data();  // no CTA leaves while a peer writes its shared memory
        return;
    }
    if (rank == 0) {
        for (int i = tid; i < k; i += NT) {
            const Level &v = sh.level[i];
            g.tokens[out + i] = v.id;
            if (g.lp) g.lp[out + i] = log_prob(v.zx, v.m, one, v.s1);
            if (g.lps) g.lps[out + i] = r.greedy ? 0.0f : log_prob(v.zx, v.m, sc, v.s);
        }
        if (tid == 0)
            g.kept[b] = k;
    }
    fill(k + 1, -1, 0.0f);
    auto last = [&](int j, float z) {
        const Level &v = sh.level[k];
        g.tokens[out + k] = j;
        if (g.lp) g.lp[out + k] = log_prob(z, v.m, one, v.s1);
        if (g.lps) g.lps[out + k] = r.greedy ? 0.0f : log_prob(z, v.m, sc, v.s);
    };
    if (r.greedy) {
        if (rank == 0 && tid == 0)
            last(sh.level[k].arg, sh.level[k].m);
        cluster_sync_data();
        return;
    }

    // The last token: what is left of p.
    enter(k);
    if (row.q && summed != k)
        both_sums(sp, sq);
    if (tid == 0 && row.q) {  // sp / sq - 1 in units of 2^-64
        const double x = ((double)(long long)(sp - sq)) / (double)sq;
        sh.minus = x < 0.0;
        sh.delta = (mass_t)(fabs(x) * 0x1p64);
    }
    __syncthreads();
    const ShareMass mp = sh.p, mq = sh.q;
    const mass_t delta = sh.delta;
    const bool minus = sh.minus;
    bool residual = row.id >= 0;
    auto mass = [&](int j, float z, float d) -> mass_t {
        const mass_t P = mp(z);
        if (!residual)
            return P;
        if (!row.q)
            return j == row.id ? 0 : P;
        mass_t Q = mq(d);
        const mass_t off = __umul64hi(Q, delta);
        Q = minus ? Q - off : Q + off;
        return P > Q ? P - Q : 0;
    };
    mass_t R = 0, none;
    for (;;) {
        mass_t own = 0;
        entries(row, j0 + lane, j1, 32,
                [&](int j, float z, float d) { own += mass(j, z, d); });
        cluster_sums(sh, rank, cs, turn, own, 0, R, none);
        if (R > 0 || !residual)
            break;
        residual = false;  // p is q as far as can be told: the whole of p
    }
    if (tid == 0)
        sh.goal = min((mass_t)((double)g.u_last[b] * (double)R), R - 1);
    __syncthreads();
    // the CTA, the warp's stretch, and in it a thread's part
    const mass_t goal = sh.goal;
    mass_t base = 0;
    unsigned has = 0;
    while (has + 1 < cs && base + sh.sums[turn][has][0] <= goal)
        base += sh.sums[turn][has++][0];
    if (has == rank) {
        int ws = 0;
        while (ws + 1 < W && base + sh.warps[0][ws] <= goal)
            base += sh.warps[0][ws++];
        const int s0 = (int)((int64_t)g.V * (rank * W + ws) / (cs * W));
        const int s1 = (int)((int64_t)g.V * (rank * W + ws + 1) / (cs * W));
        const int per = (s1 - s0 + NT - 1) / NT;
        const int a0 = min(s1, s0 + tid * per), a1 = min(s1, a0 + per);
        mass_t own = 0;
        entries(row, a0, a1, 1, [&](int j, float z, float d) { own += mass(j, z, d); });
        mass_t run = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const mass_t x = __shfl_up_sync(0xffffffffu, run, o);
            run += lane >= o ? x : 0;
        }
        if (lane == 31)
            sh.scan_w[w] = run;
        __syncthreads();
        mass_t at = base + run - own;
        for (int i = 0; i < w; ++i)
            at += sh.scan_w[i];
        if (at <= goal && goal < at + own) {
            for (int j = a0; j < a1; ++j) {
                const float z = to_f32(row.p[j]);
                at += mass(j, z, row.q ? to_f32(row.q[j]) : 0.0f);
                if (at > goal) {
                    last(j, z);
                    break;
                }
            }
        }
    }
    cluster_sync_data();
}

// A row's stretches: as many CTAs as fill the SMs four times, 512 vectors at least each.
int chunks_of(int64_t B, int64_t D, int64_t V, int in_bytes)
{
    const int64_t nvec = V * in_bytes / 16, items = B * (D + 1);
    int64_t c = (608 + items - 1) / items;
    c = c < nvec / 512 ? c : nvec / 512;
    c = c < kMaxChunks ? c : kMaxChunks;
    return c < 1 ? 1 : (int)c;
}

template <typename InT> cudaError_t launch_verify(const VerifyArgs &g, cudaStream_t s)
{
    const unsigned grid = (unsigned)((int64_t)g.B * (g.D + 1) * g.chunks);
    if ((int64_t)g.V * (int)sizeof(InT) / 16 <= 4096 * (int64_t)g.chunks)
        cis_verify_rows_kernel<InT, 1><<<grid, kVerifyThreads, 0, s>>>(g);
    else
        cis_verify_rows_kernel<InT, 4><<<grid, kVerifyThreads, 0, s>>>(g);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    unsigned cs = 1;
    while (cs < kMaxCluster && (int64_t)g.B * cs * 2 <= 608 && g.V / (2 * cs) >= 2048)
        cs *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)g.B * cs);
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cs;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, cis_verify_requests_kernel<InT>, g, cs);
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
    const int c = chunks_of(n, max_drafts, V, 4);  // (bf16 rows have no more)
    *bytes = ws_round_up((size_t)n * (size_t)(max_drafts + 1) * (size_t)c * sizeof(Part));
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
    g.parts = static_cast<Part *>(workspace);
    g.chunks = chunks_of(B, max_drafts, V, dtype == CIS_BF16 ? 2 : 4);
    const cudaError_t e = dtype == CIS_BF16 ? launch_verify<__nv_bfloat16>(g, (cudaStream_t)stream)
                                            : launch_verify<float>(g, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK : CIS_ERR_CUDA;
}
