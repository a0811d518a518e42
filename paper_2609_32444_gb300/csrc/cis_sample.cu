// cis_sample.cu -- sampling from rows of logits with given uniform numbers
// (cis_sample_tokens).
//
// Per row, with s = z / tau and the order of the entries (z descending, index ascending),
// the kept set is a prefix of that order:
//   top_k   the first top_k entries;
//   top_p   of those, the smallest prefix whose mass is at least top_p of theirs;
//   min_p   of those, the entries with s_j >= s_max + log(min_p).
// The sample is the first entry, by index, whose running kept mass is above u times the kept
// mass.
//
// The row is read once (cis_rowpass.cuh), for its maximum and the sums of its exponentials at
// tau and at 1.  What follows depends on the row:
//   nothing cut off   the CTA, the warp and then, with that warp's stretch read again by the
//                     whole CTA, the thread in whose part the running mass passes u Z;
//   else              the row's candidates, sorted by the first CTA, with masses in whole
//                     numbers (cis_select.cuh).
// Masses of fp32 exponentials decide only where their error cannot matter.  With E = 2^-20: of an
// entry within 32 bits of the maximum an exponential is off by 2.4 E of itself at most (its
// exponent, in bits, is rounded by 2^-20, kappa by 2^-24 of it, and the instruction by 2^-22), the
// share of a CTA's sum in the row's by 0.3 E, and a sum of fp32 numbers by 2^-24 for each of the
// 22 roundings on an entry's way to the row's sum, 1.4 E.  A running mass C from the row's nearer
// end, with v = u or 1 - u its goal in units of Z, is therefore off from v Z by less than twice
// 4.1 E v Z: within 8.5 E v Z of its goal it is left open (from the first entry on, the sums'
// roundings would not shrink with 1 - u).  Entries farther below the maximum (to 44 bits, from
// where on a mass may as well be 0) are off by up to 3.6 E, of a mass of 2^-32 each at most.  Z
// itself, which top_p's goal is taken from where the list does not hold the row, is off by less
// than 4.3 E.  Rows left open, those with more candidates than fit or a kept set that reaches
// beyond them, and rows with |M| / tau above 5e5, whose exponents have another form, are left to a
// second kernel, which takes every decision on whole numbers: bf16 rows by counting their values,
// fp32 rows by cis_select.cuh's selection.
//
// Bound: instruction issue in the first kernel (two exponentials an entry where the temperature is
// not 1; four CTAs of 60 registers an SM, and forcing five into 48 took 126 us a call for 110 at
// T=1024, V=151936, top-k), and the rows left.  T=1024, V=151936, top-p at temperature 0.7: 118 us
// and, for the 36% of the rows that are left, 180; T=256, nothing cut off: 27 us and 50 for the one
// row in eight that is left, its steps one after another on eight CTAs; T=1, top-k and top-p: 24 us
// a call.
#include <math.h>

#include "cis_nvtx.h"
#include "cis_rowpass.cuh"

namespace cis {
namespace {

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

// A row that cannot be sampled, by one thread.
__device__ __forceinline__ void refuse_row(const SampleArgs &a, int64_t t)
{
    write_row(a, t, -1, NAN, NAN);
    set_status(a.status, kStatusBadInput);
}

constexpr int32_t kTodo = -2;   // as a row's id: left to the second kernel
constexpr int32_t kTaken = -3;  // which has begun with it
constexpr float kOpen = 8.5f * 0x1p-20f;   // of the goal: a running mass from the nearer end
constexpr float kSlack = 4.5f * 0x1p-20f;   // of the row's mass: top_p's goal
constexpr int kCap = 1024;     // batches to read again, and candidates, of a row
constexpr int kAim = 256;      // candidates aimed at where top_k does not say

// The row is left to the exact kernel, with its mass at temperature 1 and its maximum.
__device__ __forceinline__ void leave_row(const SampleArgs &a, int64_t t, float S1, float M)
{
    a.ids_out[t] = kTodo;
    if (a.lp_out)
        a.lp_out[t] = S1;
    if (a.lps_out)
        a.lps_out[t] = M;
}

// Inclusive sums over the CTA's threads, in `scan`; with barriers.
template <int NT, typename T> __device__ void block_scan(T v, T *scan, T *warps)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T x = __shfl_up_sync(0xffffffffu, v, o);
        v += lane >= o ? x : T(0);
    }
    if (lane == 31)
        warps[w] = v;
    __syncthreads();
    T before = 0;
    for (int i = 0; i < w; ++i)
        before += warps[i];
    scan[threadIdx.x] = before + v;
    __syncthreads();
}

template <int NT> struct SampleShared {
    PassShared<NT> pass;
    mass_t scan[NT];
    mass_t warps64[NT / 32];
    mass_t goal, slack;
    uint32_t low;   // min_p's lowest key
    int kept;
    int found;      // place of the sampled candidate
};

// The log-probabilities of z: (z - M) / tau - log of the mass it is drawn from, and at 1.
__device__ __forceinline__ float log_share(float z, float M, const Scale &sc, float mass)
{
    float l, e;
    const float x = scaled_diff(z, M, sc, l), ls = logf(mass);
    const float u = two_sum(x, -ls, e);
    return u + (e + l - log_residual(mass, ls));
}

// A mass in units of 2^-43 of the maximum's.
__device__ __forceinline__ mass_t to_mass(float x) { return __float2ull_rn(x * 0x1p43f); }

// e^{(m - M) / tau}, to 2^-22.
__device__ __forceinline__ float share_of(float m, float M, const Scale &sc)
{
    float lo;
    const float e = expf(scaled_diff(m, M, sc, lo));
    return fmaf(e, lo, e);
}

// A row with nothing cut off, in the CTA that has its goal: running masses from the row's first
// entry or, `back`, from its last one, `base` those of the CTAs passed, red[w].s * unit the
// warps'.  Whole numbers, so that only the fp32 sums that they start from are rounded.  True and
// the index in the thread that has it.
template <typename InT, int NT, int kB>
__device__ bool draw_by_index(SampleShared<NT> &sh, const RowPass<InT, NT, kB> &ps, mass_t base,
                              float unit, mass_t goal, bool back, float M, const Scale &sc,
                              unsigned rank, unsigned cs, int &index, float &zi)
{
    constexpr int W = NT / 32, EV = Vec<InT>::kN;
    const int tid = threadIdx.x;
    int w = back ? W - 1 : 0;
    for (int i = 0; i < W - 1; ++i) {
        const mass_t next = base + to_mass(sh.pass.red[w].s * unit);
        if (next > goal)
            break;
        base = next;
        w += back ? -1 : 1;
    }
    const int s0 = ps.seg(w), n = ps.seg(w + 1) - s0;
    const int per = (n + NT - 1) / NT, a0 = s0 + min(n, tid * per), a1 = s0 + min(n, tid * per + per);
    // entries [j0, j1), with the row's ragged ends at the first and the last thread
    int j0 = ps.head + a0 * EV, j1 = ps.head + a1 * EV;
    if (rank == 0 && w == 0 && tid == 0)
        j0 = 0;
    if (rank == cs - 1 && w == W - 1 && tid == NT - 1)
        j1 = ps.V;
    // the sums' own form: a whole offset, and what it is short of M
    const float c = ceilf(M * sc.kappa), f = exp2_accurate(-fmaf(M, sc.kappa, -c));
    auto weight = [&](float z) { return ex2_ftz(fmaf(z, sc.kappa, -c)); };
    float sum = 0.0f, lost = 0.0f;
    auto add = [&](float x) {
        float e;
        sum = two_sum(sum, x, e);
        lost += e;
    };
    for (int j = j0; j < ps.head + a0 * EV; ++j)
        add(weight(to_f32(ps.row[j])));
    for (int v = a0; v < a1; ++v) {
        Vec<InT> x;
        x.q = __ldg(ps.rv + v);
        float p[EV];
#pragma unroll
        for (int k = 0; k < EV; ++k)
            p[k] = weight(x.entry(k));
#pragma unroll
        for (int h = EV / 2; h > 0; h /= 2)
#pragma unroll
            for (int k = 0; k < h; ++k)
                p[k] += p[k + h];
        add(p[0]);
    }
    for (int j = ps.head + a1 * EV; j < j1; ++j)
        add(weight(to_f32(ps.row[j])));
    const mass_t own = to_mass((sum + lost) * f);
    block_scan<NT>(own, sh.scan, sh.warps64);
    mass_t at = base + (back ? sh.scan[NT - 1] - sh.scan[tid] : sh.scan[tid] - own);
    if (!(at <= goal && goal < at + own))
        return false;
    for (int i = 0; i < j1 - j0; ++i) {
        const int j = back ? j1 - 1 - i : j0 + i;
        const float z = to_f32(ps.row[j]);
        const mass_t next = at + to_mass(weight(z) * f);
        if (next > goal) {
            // (512: half a unit for each number made whole on the way; V / 128: 2.4 E of V
            // masses of 2^-32)
            const mass_t open = 512 + ps.V / 128 + (mass_t)(kOpen * (float)goal);
            index = j;
            zi = z;
            // before the first mass there is nothing to be off
            return next - goal > open && (goal - at > open || at == 0);
        }
        at = next;
    }
    return false;
}

// A row with something cut off, in its first CTA: n candidates in `list`, sorted.  whole: they
// are all the row's finite entries.  above: they are all its entries from min_p's key on.
// firm: Z's error is bounded.
// Returns the sampled candidate's place, -1 (left open), or -2 - m for m kept ones that are
// yet to be put in order of their index; the kept mass; in `mass` the running masses.
template <int NT>
__device__ int draw_by_order(SampleShared<NT> &sh, const RowSettings &rs, mass_t *list, int n,
                             mass_t *mass, int V, float M, float Z, bool firm, bool whole,
                             bool above, mass_t &kept_mass)
{
    const int tid = threadIdx.x;
    const Scale &sc = rs.sc;
    if (tid == 0) {
        sh.kept = n;
        sh.found = -1;
    }
    // running masses of the order: each thread has a stretch
    const int per = (n + NT - 1) / NT, i0 = min(n, tid * per), i1 = min(n, i0 + per);
    mass_t sum = 0;
    for (int i = i0; i < i1; ++i) {
        const mass_t m = fixed_mass(key_value((uint32_t)(list[i] >> 32)), M, sc);
        mass[i] = m;
        sum += m;
    }
    mass_t run = sum;
    const int lane = tid & 31, w = tid >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const mass_t x = __shfl_up_sync(0xffffffffu, run, o);
        run += lane >= o ? x : 0;
    }
    __syncthreads();
    if (lane == 31)
        sh.warps64[w] = run;
    __syncthreads();
    run -= sum;
    for (int i = 0; i < w; ++i)
        run += sh.warps64[i];
    for (int i = i0; i < i1; ++i) {
        run += mass[i];
        mass[i] = run;  // inclusive
    }
    __syncthreads();
    int m = n;
    bool open = false, exact = whole;
    if (rs.top_k > 0 && rs.top_k < V) {
        // (a list that ends before top_k entries may yet do, if top_p or min_p ends sooner)
        exact = exact || rs.top_k <= n;
        m = min(n, rs.top_k);
        open = !exact;
    } else {
        open = !whole;
    }
    const bool cut = !open;      // the prefix so far is m entries, known
    if (rs.top_p < 1.0f) {
        // the first place whose running mass reaches the goal
        if (!cut && (!firm || (rs.top_k > 0 && rs.top_k < V)))
            return -1;  // their mass is not known
        if (tid == 0) {  // (fp64 is slow here: one thread)
            const double unit = (double)(1ull << kMassBits);
            sh.goal = cut ? (mass_t)ceil((double)rs.top_p * (double)mass[m - 1])
                          : (mass_t)((double)rs.top_p * (double)Z * unit);
            // (the candidates' masses are exact, Z is not)
            sh.slack = cut ? 0 : (mass_t)((double)kSlack * (double)Z * unit);
        }
        __syncthreads();
        const mass_t goal = sh.goal, slack = sh.slack;
        for (int i = tid; i < m; i += NT) {
            const mass_t c = mass[i], b = i ? mass[i - 1] : 0;
            if (c >= goal && (i == 0 || b < goal)) {
                // not cut: certain only where both sides are away from the goal
                const bool sure = cut || (c - goal > slack && (i == 0 || goal - b > slack));
                sh.kept = sure ? i + 1 : -1;
            }
        }
        __syncthreads();
        const int k = sh.kept;
        if (k < 0)
            return -1;
        if (cut || k < n || mass[n - 1] >= goal) {
            m = k;
            open = false;
        } else if (!(goal - mass[n - 1] > slack)) {
            return -1;
        }  // else the goal lies beyond the list
        __syncthreads();
    }
    if (rs.min_p > 0.0f) {
        for (int i = tid; i < m; i += NT) {
            const bool in = (uint32_t)(list[i] >> 32) >= sh.low;
            const bool next = i + 1 < m && (uint32_t)(list[i + 1] >> 32) >= sh.low;
            if (in && !next)
                sh.kept = i + 1;
        }
        __syncthreads();
        const int k = sh.kept;
        if (k < m || above) {  // the entries that min_p keeps are all here
            m = min(m, k);
            open = false;
        }
    }
    if (open)
        return -1;
    kept_mass = mass[m - 1];
    if (m == 1)
        return 0;
    if (tid == 0)
        sh.goal = min((mass_t)((double)rs.u * (double)kept_mass), kept_mass - 1);
    __syncthreads();
    const mass_t t = sh.goal;
    // running masses by index: for each kept entry those with a lower index
    if (m <= 64) {
        if (tid < m) {
            const uint32_t me = (uint32_t)list[tid];  // larger: a lower index
            mass_t c = 0, own = 0;
            for (int i = 0; i < m; ++i) {
                const mass_t x = mass[i] - (i ? mass[i - 1] : 0);
                c += (uint32_t)list[i] > me ? x : 0;
                own = i == tid ? x : own;
            }
            if (c <= t && c + own > t)
                sh.found = tid;
        }
        __syncthreads();
        return sh.found;
    }
    return -2 - m;
}

template <typename InT, int NT, int kB>
__global__ void __launch_bounds__(NT)
    cis_sample_kernel(const __grid_constant__ SampleArgs a, unsigned cs, int cap)
{
    constexpr int W = NT / 32;
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    __shared__ SampleShared<NT> sh;
    mass_t *list = reinterpret_cast<mass_t *>(dyn_smem);
    mass_t *room = list + cap;  // the candidates of all CTAs
    int *items = reinterpret_cast<int *>(room + cap);
    float *bmax = reinterpret_cast<float *>(items + cap);
    const int64_t t = blockIdx.x / cs;
    const unsigned rank = blockIdx.x - (unsigned)t * cs;
    const int tid = threadIdx.x;
    if (tid == 0)
        allow_next_grid();
    if (a.mask && a.mask[t] == 0) {  // the same branch in every CTA of the row
        if (rank == 0 && tid == 0)
            write_row(a, t, -1, 0.0f, 0.0f);
        return;
    }
    const RowSettings rs = row_settings(a, t);
    if (!rs.ok) {
        if (rank == 0 && tid == 0)
            refuse_row(a, t);
        return;
    }
    const bool by_k = rs.top_k > 0 && rs.top_k < a.V;
    const bool cut = rs.greedy || by_k || rs.top_p < 1.0f || rs.min_p > 0.0f;
    const bool two = a.lp_out != nullptr && rs.sc.hi != 1.0f;
    if (cs > 1)
        cluster_arrive_relaxed();  // waited for before the exchange
    if (tid == 0)
        sh.pass.items = sh.pass.n = 0;
    RowPass<InT, NT, kB> ps(reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V, rank, cs,
                            bmax);
    ExpAcc<false, true> acc;
    acc.k = rs.sc.kappa;
    acc.h = rs.sc.huge;
    ExpAcc<false> raw;
    auto entry = [&](auto &e, float z) {
        e.raise(z);
        if (e.m != -INFINITY)
            e.add_entry(z);
    };
    ps.stream(
        cut,
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
    const int aim = rs.greedy ? 1 : by_k ? min(rs.top_k, kAim) : kAim;
    const int r = (aim + (int)cs - 1) / (int)cs;
    if (cut)
        ps.bound_put(sh.pass, r);
    MaxSumU o = block_exp<NT>(acc, sh.pass.red);  // (its barriers)
    float S1 = two ? block_exp<NT>(raw, sh.pass.red2).s : o.s;
    float bound = cut ? ps.bound_get(sh.pass, r) : -INFINITY;
    float sum_w = 0.0f, sum_p = 0.0f, sum_l = 0.0f;  // the warps' sums, in their own unit
#pragma unroll
    for (int w = 0; w < W; ++w) {
        float e;
        sum_w += sh.pass.red[w].s;  // (as block_exp adds them: o.s has its roundings)
        sum_p = two_sum(sum_p, sh.pass.red[w].s, e);
        sum_l += e;
    }
    float unit = sum_w > 0.0f ? o.s / sum_w : 0.0f;
    float M = o.m, Z = sum_w > 0.0f ? (sum_p + sum_l) * unit : o.s;
    if (cs > 1) {
        exchange(sh.pass, rank, cs, o.m, bound, Z, S1);
        const auto &part = sh.pass.part;
        for (unsigned c = 0; c < cs; ++c) {
            M = fmaxf(M, part[c][0]);
            bound = fminf(bound, part[c][1]);
        }
        Z = S1 = 0.0f;
        float lost = 0.0f;
        for (unsigned c = 0; c < cs; ++c) {  // in rank order
            float e;
            Z = two_sum(Z, part[c][2] * share_of(part[c][0], M, rs.sc), e);
            lost += e;
            S1 += part[c][3] * ex2_ftz((part[c][0] - M) * kLog2e);
        }
        Z += lost;
        unit *= share_of(o.m, M, rs.sc);
    }
    if (!(Z > 0.0f && Z < INFINITY) || !(fabsf(M) < INFINITY)) {  // as every CTA finds
        if (rank == 0 && tid == 0)
            refuse_row(a, t);
        return;
    }
    const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};
    const bool firm = fabsf(M) < 0.5f * rs.sc.huge;
    if (!cut) {
        // The CTA with the goal, from the row's nearer end.
        const bool back = rs.u > 0.5f;
        const mass_t goal = to_mass((back ? 1.0f - rs.u : rs.u) * Z);
        unsigned has = back ? cs - 1 : 0;
        mass_t base = 0;
        for (unsigned i = 0; i + 1 < cs; ++i) {
            const auto &part = sh.pass.part[has];
            const mass_t next = base + to_mass(part[2] * share_of(part[0], M, rs.sc));
            if (next > goal)
                break;
            base = next;
            has += back ? -1 : 1;
        }
        if (rank != has)
            return;
        int j;
        float z;
        __shared__ int done;
        if (tid == 0)
            done = 0;
        __syncthreads();
        if (firm && draw_by_index<InT, NT, kB>(sh, ps, base, unit, goal, back, M, rs.sc, rank, cs,
                                               j, z)) {
            write_row(a, t, j, log_share(z, M, one, S1), log_share(z, M, rs.sc, Z));
            done = 1;
        }
        __syncthreads();
        if (tid == 0 && !done)
            leave_row(a, t, S1, M);
        return;
    }

    // The candidates; what min_p leaves out is none.
    bool above = false;
    if (rs.min_p > 0.0f && !rs.greedy) {
        if (tid == 0)
            sh.low = min_p_key(M, rs.tau, rs.min_p);
        __syncthreads();
        const float least = key_value(sh.low);
        above = bound <= least;
        if (rs.top_p >= 1.0f && (above || !by_k)) {
            // (top_p needs the mass of those that min_p leaves out); with nothing but min_p
            // the kept set is all of them, however many
            bound = least;
            above = true;
        }
    }
    int n = ps.collect(sh.pass, bound, list, items, cap);
    if (cs > 1) {
        n = gather_lists<NT>(sh.pass, rank, cs, list, n, room, cap);
        if (rank != 0)
            return;
        mass_t *swap = list;
        list = room;
        room = swap;
    }
    if (n > cap) {
        if (tid == 0)
            leave_row(a, t, S1, M);
        return;
    }
    sort_list<NT>(list, n);
    int at = 0;
    mass_t kept = (mass_t)1 << kMassBits;
    if (!rs.greedy)
        at = draw_by_order<NT>(sh, rs, list, n, room, (int)a.V, M, Z, firm, bound == -INFINITY,
                               above, kept);
    mass_t pick = at >= 0 ? list[at] : 0;
    if (at < -2) {
        // more than 64 kept: put in order of the index, with their places
        const int m = -2 - at;
        const mass_t t0 = sh.goal;
        for (int i = tid; i < m; i += NT)
            list[i] = (list[i] << 32) | (uint32_t)i;  // (the inverted index: larger is lower)
        __syncthreads();
        sort_list<NT>(list, m);
        const int per = (m + NT - 1) / NT, i0 = min(m, tid * per), i1 = min(m, i0 + per);
        auto own = [&](int i) {
            const uint32_t p = (uint32_t)list[i];
            return room[p] - (p ? room[p - 1] : 0);
        };
        mass_t sum = 0;
        for (int i = i0; i < i1; ++i)
            sum += own(i);
        mass_t run = sum;
        const int lane = tid & 31, w = tid >> 5;
#pragma unroll
        for (int o2 = 1; o2 < 32; o2 <<= 1) {
            const mass_t x = __shfl_up_sync(0xffffffffu, run, o2);
            run += lane >= o2 ? x : 0;
        }
        if (lane == 31)
            sh.warps64[w] = run;
        __syncthreads();
        run -= sum;
        for (int i = 0; i < w; ++i)
            run += sh.warps64[i];
        for (int i = i0; i < i1; ++i) {
            const mass_t next = run + own(i);
            if (run <= t0 && next > t0)
                sh.found = i;
            run = next;
        }
        __syncthreads();
        at = sh.found;
        if (at >= 0) {
            const uint32_t inv = (uint32_t)(list[at] >> 32);
            const int j = (int)(0xffffffffu - inv);
            pick = order_pair(order_key(to_f32(ps.row[j])), (uint32_t)j);
        }
    }
    if (tid == 0) {
        if (at < 0) {
            leave_row(a, t, S1, M);
        } else {
            const float z = key_value((uint32_t)(pick >> 32));
            write_row(a, t, (int32_t)(0xffffffffu - (uint32_t)pick), log_share(z, M, one, S1),
                      rs.greedy ? 0.0f : log_share(z, M, rs.sc, (float)mass_value(kept)));
        }
    }
}

// One row that the first kernel has left, exactly, by the CTAs of a cluster.
template <typename InT, int NT>
__device__ void exact_row(SelectShared<NT> &sh, const SampleArgs &a, int64_t t, int &turn)
{
    RowSelect<InT, NT> rs(sh, reinterpret_cast<const InT *>(a.logits) + t * a.ld, a.V, turn);
    if (!sh.ready) {
        __syncthreads();
        fill_row_table(sh.table);
        if (threadIdx.x == 0)
            sh.ready = true;
        __syncthreads();
    }
    const RowSettings rset = row_settings(a, t);
    const int64_t k = rset.greedy ? 1 : rset.top_k;
    const bool by_k = k > 0 && k < a.V, by_p = rset.top_p < 1.0f && !rset.greedy;
    // The maximum: the first kernel's, where it has left the row, and the least entry is
    // not needed
    float M, bottom = -INFINITY;
    if (a.lps_out && !by_k) {
        M = a.lps_out[t];
    } else {
        uint32_t least;
        M = key_value(rs.max_key(least));
        bottom = key_value(least);
    }
    const Scale &sc = rset.sc;
    const RowMass mass(sh.table, M, rset.tau, sc);
    const float depth = M - 31.0f * rset.tau, floor_z = bottom > depth ? bottom : depth;
    // entries' weights in a selection: 1 each, or the mass of those above zk
    bool count = false;
    float zk = -INFINITY;
    auto approx = [&](float z) {
        return count ? 1.0f : (z > zk ? ex2_ftz((z - M) * sc.kappa) : 0.0f);
    };
    auto weight = [&](float z) {
        return count ? (mass_t)1 : (z > zk ? mass(z) : (mass_t)0);
    };
    Kept kept{0, 0};
    mass_t above, equal, gt, eq, gt0, eq0, target, wkey = 0;
    bool parts = false;
    // top_k first, then top_p: one place for both, as the selection's code is large
#pragma unroll 1
    for (int step = by_k ? 0 : 1; step < (by_p ? 2 : 1); ++step) {
        count = step == 0;
        float goal = (float)k, share = 0.0f, low = M - bottom > 1024.0f ? M - 64.0f : bottom;
        target = (mass_t)k;
        if (!count) {
            low = floor_z;
            if (by_k) {
                rs.kept_mass(kept.key, mass, gt, eq, gt0, eq0);
                target = (mass_t)ceil((double)rset.top_p * (double)(gt + kept.ties * wkey));
                if (target > gt) {  // within the entries at the key
                    if (wkey)
                        kept.ties = min(kept.ties, (target - gt + wkey - 1) / wkey);
                    break;
                }
                goal = (float)mass_value(target);
                zk = key_value(kept.key);
            } else {
                share = rset.top_p;
            }
        }
        kept.key = rs.select(target, goal, share, low, M, approx, weight, above, equal, parts);
        parts = parts && !count;
        wkey = mass(key_value(kept.key));
        kept.ties = count ? target - above : (target - above + wkey - 1) / wkey;
    }
    if (rset.min_p > 0.0f) {
        const uint32_t low = min_p_key(M, rset.tau, rset.min_p);
        if (kept.key < low) {
            kept = Kept{low, ~(mass_t)0};  // all entries at it, too
            wkey = mass(key_value(low));
            parts = false;
        }
    }
    if (parts)
        rs.kept_parts(gt, eq, gt0, eq0);
    else
        rs.kept_mass(kept.key, mass, gt, eq, gt0, eq0);
    const mass_t Z = gt + min(eq, kept.ties) * wkey;
    if (Z == 0 && rs.rank == 0 && threadIdx.x == 0)
        refuse_row(a, t);  // (the maximum is always kept: a mark may not stay in any case)
    target = (mass_t)((double)rset.u * (double)Z);
    // the row's mass at temperature 1: the first kernel's, where it has left the row
    const float S1 = a.lp_out ? a.lp_out[t] : 1.0f;
    int64_t j = 0;
    if (rs.locate(kept, wkey, min(target, Z - 1), gt0, eq0, mass, j) && threadIdx.x == 0) {
        const float z = to_f32(rs.row[j]);
        const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};
        write_row(a, t, (int32_t)j, log_share(z, M, one, S1),
                  rset.greedy ? 0.0f : log_share(z, M, sc, (float)mass_value(Z)));
    }
    __syncthreads();
}

// The rows left, a cluster per row.
template <typename InT>
__global__ void __launch_bounds__(kSelThreads, 2)
    cis_sample_exact_kernel(const __grid_constant__ SampleArgs a)
{
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    SelectShared<kSelThreads> &sh = *reinterpret_cast<SelectShared<kSelThreads> *>(dyn_smem);
    int turn = 0;
    if (threadIdx.x == 0) {
        allow_next_grid();
        sh.ready = false;
    }
    grid_wait();
    RowsLeft<kSelThreads> rows(sh, a.T, gridDim.x / kSelCluster, blockIdx.x / kSelCluster);
    for (;;) {
        const int64_t t = rows.next([&](int64_t i) { return a.ids_out[i] == kTodo; });
        if (t < 0)
            break;
        exact_row<InT>(sh, a, t, turn);
    }
    cg::this_cluster().sync();  // no CTA leaves while a peer reads its shared memory
}

// bf16 rows, exactly, by counting: a row's entries take few values, and how many there are of
// each is all that its filters and masses depend on.  One CTA a row, or two or four where there
// are few rows: one pass counts the values 2^-26 <= |z| < 2^8 and zero, a bin each in shared
// memory (each CTA then adds up all the cluster's counts); 19 bins a thread give the masses in
// the order of the values, the kept set's end and the kept mass; a second pass looks the kept
// entries' masses up, to find the CTA, its warp's stretch, the thread's part and the entry at
// which the running mass passes its goal.  Entries at or below -256 are left out where they
// have no mass; a row with others outside the bins (or with none inside) goes to exact_row: of
// rows of 151,936 entries from a bell of width 2.5 one in 400 (with bins from 2^-17 on every
// third).
//
// Bound: the passes' dependent steps an entry (bin, then an atomic or a lookup in shared memory)
// on the 16 warps that the counts and the registers leave room for: 32,000 and 37,000 of a row's
// 92,000 cycles (151,936 entries), 0.45 instructions a cycle and scheduler.  A call with 64 such
// rows takes 93 us with two CTAs a row and 114 with one.
constexpr int kCountThreads = 512;
constexpr int kLoBits = (127 - 26) << 7, kHiBits = (127 + 8) << 7;  // of bf16 magnitudes
constexpr int kSide = kHiBits - kLoBits;   // bins of either sign
constexpr int kZero = 2 * kSide, kValues = 2 * kSide + 1;
// a thread's bins: an odd number, so that neighbouring threads are on different banks
constexpr int kPer = (kValues + kCountThreads - 1) / kCountThreads | 1;

struct CountShared {
    SelectShared<kCountThreads> select;
    alignas(16) mass_t mass[kValues];  // of one entry of a bin; 0: not kept
    mass_t warps[2][kCountThreads / 32];
    mass_t goal;
    mass_t gt, at;     // mass before the kept set's last bin, of an entry in it
    mass_t ties;
    int end;           // that bin's place in the order (kValues: no last bin)
    int top;
    uint32_t low;      // min_p's lowest key
    bool odd;
    float most;        // the largest entry left out
    int far[kCountThreads / 32];
    int next[kCountThreads / 32];
    bool got;
};
static_assert(sizeof(int) * kValues <= sizeof(float) * kBins * kCountThreads,
              "the counts fit the selection's columns");

// The bin of a bf16's bits; -1: none.
__device__ __forceinline__ int value_bin(uint32_t h)
{
    const uint32_t r = (h & 0x7fffu) - kLoBits;
    return r < (uint32_t)kSide ? (int)(r + (h & 0x8000u ? kSide : 0))
                               : ((h & 0x7fffu) == 0 ? kZero : -1);
}
// The bin at a place of the order (largest value first), and its value's bits.
__device__ __forceinline__ int place_bin(int o)
{
    return o < kSide ? kSide - 1 - o : (o == kSide ? kZero : o - 1);
}
__device__ __forceinline__ float place_value(int o)
{
    if (o == kSide)
        return 0.0f;
    const uint32_t m = o < kSide ? kHiBits - 1 - o : kLoBits + (o - kSide - 1);
    return __uint_as_float((m | (o < kSide ? 0u : 0x8000u)) << 16);
}

// The rows left, one at a time to whichever CTA is free: which rows are left, and so how many
// of a fixed share of them, is up to the data (with fixed shares of 1,024 rows of which half
// were left, the busiest SM had 2.3 times the mean's work: 308 us).  A CTA looks for marks from
// a place of its own on, 8 a thread at a time, and takes the first row by exchanging its mark;
// what a row's outputs are does not depend on the CTA.
struct RowClaims {
    static constexpr int NT = kCountThreads, kN = 8;
    CountShared &sh;
    int64_t T, first, base = 0;

    __device__ __forceinline__ int64_t row(int64_t i) const
    {
        return first + i < T ? first + i : first + i - T;
    }
    __device__ int64_t next(int32_t *marks)
    {
        const int tid = threadIdx.x;
        while (base < T) {
            int best = NT * kN;
#pragma unroll
            for (int k = kN - 1; k >= 0; --k) {
                const int64_t i = base + tid + k * NT;
                if (i < T && __ldcg(marks + row(i)) == kTodo)
                    best = tid + k * NT;
            }
            best = __reduce_min_sync(0xffffffffu, best);
            __syncthreads();
            if ((tid & 31) == 0)
                sh.next[tid >> 5] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NT / 32; ++w)
                best = min(best, sh.next[w]);
            if (best == NT * kN) {  // no mark comes back
                base += NT * kN;
                continue;
            }
            const int64_t t = row(base + best);
            if (tid == 0)
                sh.got = atomicCAS(marks + t, kTodo, kTaken) == kTodo;
            __syncthreads();
            if (sh.got)
                return t;
        }
        return -1;
    }
};

__global__ void __launch_bounds__(kCountThreads, 1)
    cis_sample_counts_kernel(const __grid_constant__ SampleArgs a)
{
    constexpr int NT = kCountThreads, W = NT / 32, EV = 8;
    extern __shared__ __align__(16) uint8_t dyn_smem[];
    CountShared &sh = *reinterpret_cast<CountShared *>(dyn_smem);
    int *count = reinterpret_cast<int *>(sh.select.cols);
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    int turn = 0;
    if (tid == 0) {
        allow_next_grid();
        sh.select.ready = false;
    }
    grid_wait();
    const ClusterPlace cl = cluster_place();
    const int64_t groups = gridDim.x / cl.size, group = blockIdx.x / cl.size;
    RowsLeft<NT> own(sh.select, a.T, groups, group);
    RowClaims any{sh, a.T, group * a.T / groups};
    for (;;) {
        const int64_t t = a.T <= groups
                              ? own.next([&](int64_t i) { return a.ids_out[i] == kTodo; })
                              : any.next(a.ids_out);
        if (t < 0)
            break;
        const RowSettings rset = row_settings(a, t);
        RowSelect<__nv_bfloat16, NT> rs(
            sh.select, reinterpret_cast<const __nv_bfloat16 *>(a.logits) + t * a.ld, a.V, turn);
        const uint4 *rv = reinterpret_cast<const uint4 *>(rs.row + rs.head);
        const uint16_t *bits = reinterpret_cast<const uint16_t *>(rs.row);
        if (!sh.select.ready) {
            __syncthreads();
            fill_row_table(sh.select.table);
            if (tid == 0)
                sh.select.ready = true;
        }
        for (int i = tid; i < kValues; i += NT)
            count[i] = 0;
        if (tid == 0)
            sh.top = kValues;
        __syncthreads();
        // Counts.
        bool odd = false;
        float far = -INFINITY;
        auto add = [&](uint32_t h) {
            const int b = value_bin(h);
            if (b >= 0) {
                atomicAdd(&count[b], 1);
            } else {
                const float z = __uint_as_float(h << 16);
                odd = odd || !(z <= -256.0f);  // small, large, +inf or NaN
                far = fmaxf(far, z);
            }
        };
        // f(bits) for the entries of the warp's stretch, four vectors a lane ahead of their use
        auto stretch = [&](auto f) {
            constexpr int kN = 4;
            const int s1 = rs.seg(w + 1);
            auto load = [&](uint4 (&q)[kN], int v) {
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    q[k] = v + 32 * k < s1 ? __ldg(rv + v + 32 * k) : make_uint4(0, 0, 0, 0);
            };
            uint4 q[kN], next[kN];
            int v = rs.seg(w) + lane;
            load(q, v);
#pragma unroll 1
            for (; v < s1; v += 32 * kN) {
                load(next, v + 32 * kN);
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    if (v + 32 * k < s1) {
                        const uint32_t x[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f(x[i] & 0xffffu);
                            f(x[i] >> 16);
                        }
                    }
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    q[k] = next[k];
            }
        };
        stretch(add);
        const int64_t tail = rs.head + (rs.V - rs.head) / EV * EV;  // the ragged ends
        const bool at_head = cl.rank == 0 && w == 0 && lane < rs.head;
        const bool at_tail = cl.rank == cl.size - 1 && w == W - 1 && lane >= 16 &&
                             tail + lane - 16 < rs.V;
        if (at_head)
            add(bits[lane]);
        if (at_tail)
            add(bits[tail + lane - 16]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            far = fmaxf(far, __shfl_xor_sync(0xffffffffu, far, o));
        if (lane == 0)
            sh.far[w] = __float_as_int(far);
        odd = __syncthreads_or(odd) != 0;
        for (int i = 0; i < W; ++i)
            far = fmaxf(far, __int_as_float(sh.far[i]));
        if (cl.size > 1) {
            // the other CTAs' counts to these, once all have read them
            const cg::cluster_group cluster = cg::this_cluster();
            if (tid == 0) {
                sh.odd = odd;
                sh.most = far;
            }
            cluster.sync();
            int sum[kPer] = {};
            for (unsigned r = 0; r < cl.size; ++r) {
                const int *theirs = cluster.map_shared_rank(count, (int)r);
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    sum[i] += tid + i * NT < kValues ? theirs[tid + i * NT] : 0;
            }
            for (unsigned r = 0; r < cl.size; ++r) {
                const CountShared *peer = cluster.map_shared_rank(&sh, (int)r);
                odd = odd || peer->odd;
                far = fmaxf(far, peer->most);
            }
            cluster.sync();
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (tid + i * NT < kValues)
                    count[tid + i * NT] = sum[i];
            __syncthreads();
        }
        // The maximum.
        const int o0 = min(kValues, tid * kPer), o1 = min(kValues, o0 + kPer);
        for (int o = o0; o < o1; ++o)
            if (count[place_bin(o)] > 0) {
                atomicMin(&sh.top, o);
                break;
            }
        __syncthreads();
        const float M = sh.top < kValues ? place_value(sh.top) : 0.0f;
        if (odd || sh.top == kValues || far >= M - 32.0f * rset.tau) {
            __syncthreads();
            exact_row<__nv_bfloat16>(sh.select, a, t, turn);
            cg::this_cluster().sync();  // before the columns are counts again
            continue;
        }
        // Masses, and this thread's place in their order.
        const RowMass mass(sh.select.table, M, rset.tau, rset.sc);
        mass_t own = 0, n = 0;
        for (int o = o0; o < o1; ++o) {
            const int b = place_bin(o), c = count[b];
            const mass_t m = mass(place_value(o));
            sh.mass[b] = m;
            own += c * m;
            n += c;
        }
        mass_t before = own, place = n;  // inclusive sums, then those before
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const mass_t x = __shfl_up_sync(0xffffffffu, before, o);
            const mass_t y = __shfl_up_sync(0xffffffffu, place, o);
            before += lane >= o ? x : 0;
            place += lane >= o ? y : 0;
        }
        if (lane == 31) {
            sh.warps[0][w] = before;
            sh.warps[1][w] = place;
        }
        __syncthreads();
        mass_t total = 0, all = 0;
        before -= own;
        place -= n;
        for (int i = 0; i < W; ++i) {
            before += i < w ? sh.warps[0][i] : 0;
            place += i < w ? sh.warps[1][i] : 0;
            total += sh.warps[0][i];
            all += sh.warps[1][i];
        }
        // The kept set: bins before `end`, and the first `ties` entries of that bin.
        if (tid == 0) {
            sh.end = kValues;
            sh.ties = 0;
            sh.gt = total;
            sh.at = 0;
        }
        __syncthreads();
        // f(place, mass before it, entries before it, its entries, an entry's mass)
        auto places = [&](auto f) {
            mass_t m = before, c = place;
            for (int o = o0; o < o1; ++o) {
                const int b = place_bin(o), k = count[b];
                f(o, m, c, k, sh.mass[b]);
                m += k * sh.mass[b];
                c += k;
            }
        };
        const int64_t k = rset.greedy ? 1 : rset.top_k;
        if (k > 0 && (mass_t)k < all)
            places([&](int o, mass_t m, mass_t c, int here, mass_t one) {
                if (c < (mass_t)k && c + here >= (mass_t)k) {
                    sh.end = o;
                    sh.ties = (mass_t)k - c;
                    sh.gt = m;
                    sh.at = one;
                }
            });
        __syncthreads();
        if (rset.top_p < 1.0f && !rset.greedy) {
            const mass_t gt = sh.gt, at = sh.at, ties = sh.ties;
            if (tid == 0)  // (fp64 is slow here: one thread)
                sh.goal = (mass_t)ceil((double)rset.top_p * (double)(gt + ties * at));
            __syncthreads();
            const mass_t target = sh.goal;
            if (target <= gt) {
                places([&](int o, mass_t m, mass_t, int here, mass_t one) {
                    if (m < target && m + here * one >= target) {
                        sh.end = o;
                        sh.ties = (target - m + one - 1) / one;
                        sh.gt = m;
                        sh.at = one;
                    }
                });
            } else if (tid == 0 && at) {
                sh.ties = min(ties, (target - gt + at - 1) / at);
            }
            __syncthreads();
        }
        if (rset.min_p > 0.0f) {
            if (tid == 0)
                sh.low = min_p_key(M, rset.tau, rset.min_p);
            const int end = sh.end;
            __syncthreads();
            const uint32_t low = sh.low;
            places([&](int o, mass_t m, mass_t, int, mass_t) {
                if (o <= end && order_key(place_value(o)) < low &&
                    (o == 0 || order_key(place_value(o - 1)) >= low)) {
                    sh.end = o;
                    sh.ties = 0;
                    sh.gt = m;
                    sh.at = 0;
                }
            });
            __syncthreads();
        }
        const int end = sh.end, kbin = end < kValues ? place_bin(end) : -1;
        const mass_t at = sh.at, ties = sh.ties, Z = sh.gt + ties * at;
        __syncthreads();
        if (tid == 0)
            sh.goal = min((mass_t)((double)rset.u * (double)Z), Z - 1);
        for (int o = max(o0, end); o < o1; ++o)  // the rest has no mass
            sh.mass[place_bin(o)] = 0;
        __syncthreads();
        const mass_t goal = sh.goal;
        // The warps' stretches.
        mass_t gt = 0, eq = 0;
        const float least = end < kValues ? place_value(end) : -INFINITY;
        auto look = [&](uint32_t h) {
            if (__uint_as_float(h << 16) >= least) {
                const int b = value_bin(h);
                gt += b >= 0 ? sh.mass[b] : 0;
                eq += b == kbin;
            }
        };
        stretch(look);
        if (at_head)
            look(bits[lane]);
        if (at_tail)
            look(bits[tail + lane - 16]);
        rs.warp_sums(gt, eq);
        if (lane == 0) {
            sh.warps[0][w] = gt;
            sh.warps[1][w] = kbin < 0 ? 0 : eq;
        }
        __syncthreads();
        auto upto = [&](mass_t g, mass_t e) { return g + min(e, ties) * at; };
        mass_t g0 = 0, e0 = 0;
        if (cl.size > 1) {  // the CTAs before this one
            const cg::cluster_group cluster = cg::this_cluster();
            cluster.sync();
            for (unsigned r = 0; r < cl.rank; ++r) {
                const CountShared *peer = cluster.map_shared_rank(&sh, (int)r);
                for (int i = 0; i < W; ++i) {
                    g0 += peer->warps[0][i];
                    e0 += peer->warps[1][i];
                }
            }
            cluster.sync();
        }
        int sw = 0;
        bool here = upto(g0, e0) <= goal;
        for (; sw < W; ++sw) {
            const mass_t g = g0 + sh.warps[0][sw], e = e0 + sh.warps[1][sw];
            if (upto(g, e) > goal)
                break;
            g0 = g;
            e0 = e;
        }
        if (!here || sw == W) {  // in another CTA's part
            if (Z == 0 && cl.rank == 0 && tid == 0)
                refuse_row(a, t);  // (as in exact_row)
            __syncthreads();
            continue;
        }
        // Within the stretch: consecutive entries a thread.
        const int64_t f0 = rs.first(sw), f1 = rs.first(sw + 1);
        const int64_t per = (f1 - f0 + NT - 1) / NT, j0 = min(f1, f0 + tid * per),
                      j1 = min(f1, j0 + per);
        gt = eq = 0;
        for (int64_t j = j0; j < j1; ++j)
            look(bits[j]);
        if (kbin < 0)
            eq = 0;
        mass_t ig = gt, ie = eq;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const mass_t x = __shfl_up_sync(0xffffffffu, ig, o);
            const mass_t y = __shfl_up_sync(0xffffffffu, ie, o);
            ig += lane >= o ? x : 0;
            ie += lane >= o ? y : 0;
        }
        __syncthreads();
        if (lane == 31) {
            sh.warps[0][w] = ig;
            sh.warps[1][w] = ie;
        }
        __syncthreads();
        ig += g0 - gt;
        ie += e0 - eq;
        for (int i = 0; i < w; ++i) {
            ig += sh.warps[0][i];
            ie += sh.warps[1][i];
        }
        if (upto(ig, ie) <= goal && upto(ig + gt, ie + eq) > goal) {
            gt = ig;
            eq = ie;
            int64_t j = j0;
            for (; j < j1; ++j) {
                look(bits[j]);
                if (upto(gt, kbin < 0 ? 0 : eq) > goal)
                    break;
            }
            const float z = __uint_as_float((uint32_t)bits[j] << 16) + 0.0f;
            const Scale one{1.0f, 0.0f, kLog2e, kHugeLogit};
            const float S1 = a.lp_out ? a.lp_out[t] : 1.0f;
            write_row(a, t, (int32_t)j, log_share(z, M, one, S1),
                      rset.greedy ? 0.0f : log_share(z, M, rset.sc, (float)mass_value(Z)));
        }
        __syncthreads();
    }
    cg::this_cluster().sync();  // no CTA leaves while a peer reads its shared memory
}

template <typename InT, int NT, int kB>
cudaError_t launch_fast(const SampleArgs &a, const PassPlan &p, cudaStream_t s)
{
    auto kern = cis_sample_kernel<InT, NT, kB>;
    constexpr size_t lists = kCap * (2 * sizeof(mass_t) + sizeof(int));
    const size_t smem = lists + p.maxima;
    const cudaError_t e = allow_smem(kern, lists + kMostMaxima);
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
    return cudaLaunchKernelEx(&cfg, kern, a, (unsigned)p.cs, kCap);
}

// The exact kernel.
template <typename InT>
cudaError_t launch_exact(const SampleArgs &a, cudaStream_t s)
{
    constexpr size_t smem = sizeof(SelectShared<kSelThreads>);
    const cudaError_t e = allow_smem(cis_sample_exact_kernel<InT>, smem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    // two CTAs an SM are 38 clusters; four times as many share the rows that are left more evenly
    const int64_t groups = a.T < 152 ? a.T : 152;
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
    return cudaLaunchKernelEx(&cfg, cis_sample_exact_kernel<InT>, a);
}

// bf16 rows that the first kernel has left.
inline cudaError_t launch_counts(const SampleArgs &a, cudaStream_t s)
{
    constexpr size_t smem = sizeof(CountShared);
    const cudaError_t e = allow_smem(cis_sample_counts_kernel, smem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    // Few rows: two or four CTAs each, as many as the SMs take (one a SM).
    const int cs = a.T <= 38 ? 4 : a.T <= 76 ? 2 : 1;
    cfg.gridDim = dim3((unsigned)((a.T < 152 ? a.T : 152) * cs));
    cfg.blockDim = dim3(kCountThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cs;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, cis_sample_counts_kernel, a);
}

template <typename InT> cudaError_t launch_sample(const SampleArgs &a, cudaStream_t s)
{
    const PassPlan p = pass_plan(a.T, a.V, (int)sizeof(InT));
    if (a.T * p.cs > 0x7fffffffLL)
        return cudaErrorNotSupported;
    const cudaError_t e = p.nt == 64  ? launch_fast<InT, 64, 1>(a, p, s)
                          : p.kb == 1 ? launch_fast<InT, 256, 1>(a, p, s)
                                      : launch_fast<InT, 256, 4>(a, p, s);
    if (e != cudaSuccess)
        return e;
    // Without a filter a row that is left needs one pass of masses, and eight CTAs are faster at
    // that than one with its counts (T=256, V=151936: 65 us a call against 152).
    if constexpr (sizeof(InT) == 2)
        if (a.top_k || a.top_p || a.min_p)
            return launch_counts(a, s);
    return launch_exact<InT>(a, s);
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
    if (!row_args_ok(logits, dtype, T, V, ld) ||
        !aligned4(u, temperature, top_k, top_p, min_p, ids_out, lp_out, lp_sampled_out, dev_status))
        return CIS_ERR_INVALID_ARG;
    if (T == 0)
        return CIS_OK;
    if (logits == nullptr || u == nullptr || ids_out == nullptr ||
        (lp_out != nullptr && lp_out == lp_sampled_out))
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
                              ? launch_sample<__nv_bfloat16>(a, (cudaStream_t)stream)
                              : launch_sample<float>(a, (cudaStream_t)stream);
    return e == cudaSuccess ? CIS_OK
                            : (e == cudaErrorNotSupported ? CIS_ERR_UNSUPPORTED : CIS_ERR_CUDA);
}
