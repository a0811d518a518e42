"""cis_sample_tokens against its definition in 64 bits: the sampled token (equal, ties to the
lowest index) and its two log-probabilities.

The reference sorts each row stably, takes the kept prefix and the running sums in fp64, and
says how near the decision was: the kernel's masses are right to 2^-34 of each and 2^-44 of
the largest, so a row whose number falls within 2^-32 of a boundary of its kept mass may go to
the neighbour (none of these inputs has one: the test asserts it for its own seeds).  log-probabilities: the row's mass is
summed to 2^-20 (fp32 exponentials, each right to 2^-22), and the result is rounded once.
"""
import math

import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _reference(z, u, tau=None, top_k=None, top_p=None, min_p=None):
    """ids, lp, lp_sampled and the least distance of a decision from its border."""
    T, V = z.shape
    ids, lp, lps, near = [], [], [], 1.0
    x = z.double().cpu()
    get = lambda a, i, d: d if a is None else float(a[i].double())  # noqa: E731
    for i in range(T):
        r, t = x[i], get(tau, i, 1.0)
        v, at = torch.sort(r + 0.0, descending=True, stable=True)
        greedy = t == 0
        s = (v - v[0]) / (1.0 if greedy else t)
        w = s.exp()
        k = int(get(top_k, i, 0))
        n = V if k <= 0 else min(k, V)
        n = 1 if greedy else n
        p = get(top_p, i, 1.0)
        if p < 1:
            c = w[:n].cumsum(0)
            m = int((c < p * c[-1]).sum()) + 1
            near = min(near, float((c - p * c[-1]).abs().min() / c[-1]))
            n = min(n, m)
        lo = get(min_p, i, 0.0)
        if lo > 0:
            n = min(n, int((s >= math.log(lo)).sum()))
        kept = torch.zeros(V, dtype=torch.float64)
        kept[at[:n]] = w[:n]
        c = kept.cumsum(0)
        goal = float(u[i].double()) * float(c[-1])
        j = int((c <= goal).sum())
        edge = c[kept > 0]
        if not greedy and edge.numel() > 1 and goal > 0:
            near = min(near, float((edge - goal).abs().min() / c[-1]))
        ids.append(j)
        lp.append(float((r[j] - v[0]) - torch.logsumexp(r - v[0], 0)))
        lps.append(0.0 if greedy else float((r[j] - v[0]) / t - c[-1].log()))
    f = lambda a: torch.tensor(a, dtype=torch.float64, device=DEV)  # noqa: E731
    return torch.tensor(ids, device=DEV), f(lp), f(lps), near


def _check(z, u, tau=None, top_k=None, top_p=None, min_p=None, on_border=False):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ids, lp, lps = binding.cis_sample_tokens(z, u, temperature=tau, top_k=top_k, top_p=top_p,
                                             min_p=min_p, want_lp_sampled=True, dev_status=st)
    want, wlp, wlps, near = _reference(z, u, tau, top_k, top_p, min_p)
    # of the inputs alone (on a border: the kept entries are equal, their masses exact)
    assert near > 2.0 ** -32 or (on_border and near == 0), near
    assert int(st) == 0
    assert torch.equal(ids.long(), want), (ids.long() != want).nonzero().view(-1)[:5].tolist()
    for a, b in ((lp, wlp), (lps, wlps)):
        big = torch.isinf(b.float())  # (beyond fp32's range)
        assert torch.equal(a[big], b.float()[big])
        far = ((a.double() - b).abs() - 2.0 ** -23 * b.abs())[~big]
        assert bool((far <= 2.0 ** -20).all()), far.max()
    return ids, lp, lps


def _rows(T, V, dtype, g, pad=0, off=0, width=3.0):
    buf = (torch.randn(T * (V + pad) + off, generator=g, device=DEV) * width).to(dtype)
    return buf[off:].view(T, V + pad)[:, :V]


def _full(T, v, dt=torch.float32):
    return torch.full((T,), v, dtype=dt, device=DEV)


SETTINGS = [
    {}, {"tau": 0.7}, {"tau": 0.0}, {"tau": 3.0, "top_k": 5}, {"top_k": 1}, {"top_k": 300},
    {"top_p": 0.9}, {"top_p": 1e-6}, {"top_p": 0.9999, "tau": 2.0}, {"min_p": 0.05},
    {"min_p": 1.0}, {"tau": 0.8, "top_k": 40, "top_p": 0.95, "min_p": 0.01},
    {"top_k": 20, "top_p": 0.5}, {"tau": 1.3, "top_p": 0.97, "min_p": 1e-4},
    {"top_k": 2000, "top_p": 0.99}]


def _named(T, s):
    dt = {"top_k": torch.int32}
    return {k: _full(T, v, dt.get(k, torch.float32)) for k, v in s.items()}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("i", range(len(SETTINGS)))
def test_settings(dtype, i):
    """Every filter alone and together, on rows from one entry to a few CTAs' worth."""
    for T, V, pad, off in ((4, 1, 0, 0), (5, 2, 1, 1), (9, 7, 0, 3), (12, 33, 3, 1),
                           (16, 1000, 8, 0), (8, 4097, 0, 0), (6, 16391, 5, 2)):
        g = _gen(1000 * i + V)
        z = _rows(T, V, dtype, g, pad, off)
        u = torch.rand(T, generator=g, device=DEV)
        _check(z, u, **_named(T, SETTINGS[i]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [0.3, 2.5, 8.0])
def test_large_vocabulary(dtype, width):
    """The workloads' vocabulary: flat rows (wide nuclei), bell-shaped and peaked ones."""
    T, V = 24, 151936
    g = _gen(int(width * 10))
    z = _rows(T, V, dtype, g, width=width)
    u = torch.rand(T, generator=g, device=DEV)
    for s in ({}, {"tau": 0.6, "top_p": 0.95, "top_k": 20}, {"top_p": 0.9}, {"min_p": 0.02},
              {"tau": 1.5, "top_p": 0.8}, {"top_k": 200}, {"top_k": 5000, "top_p": 0.7}):
        _check(z, u, **_named(T, s))


def test_mixed_requests():
    """Every row with settings of its own, masked rows among them."""
    T, V = 64, 5003
    g = _gen(77)
    z = _rows(T, V, torch.float32, g, 1, 1)
    r = [torch.rand(T, generator=g, device=DEV) for _ in range(6)]
    tau = torch.where(r[0] < 0.2, 0.0, 0.3 + r[0])
    k = torch.where(r[1] < 0.5, -1, (1 + 400 * r[2])).int()
    p = torch.where(r[2] < 0.5, 1.0, 0.3 + 0.69 * r[3])
    m = torch.where(r[3] < 0.5, 0.0, r[4])
    ids, lp, lps = _check(z, r[5], tau, k, p, m)
    mask = (r[4] < 0.7).to(torch.uint8) * 3
    got = binding.cis_sample_tokens(z, r[5], tau, k, p, m, mask=mask, want_lp_sampled=True)
    on = mask != 0
    for a, b, off in zip(got, (ids, lp, lps), (-1, 0, 0)):
        assert torch.equal(a[on], b[on]) and bool((a[~on] == off).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties(dtype):
    """Rows of equal entries, of two values, and of both zeros: the lowest index first, and
    the filters' borders inside a run of equal entries."""
    V = 9000
    g = _gen(5)
    z = torch.zeros((6, V), dtype=dtype, device=DEV)
    z[1] = -0.0
    z[2, ::2] = -0.0
    z[3, 4000:] = 1.0
    z[4, 17::1000] = 2.0
    z[5] = 1e30
    u = torch.tensor([0.0, 0.99, 0.3, 0.5, 0.7, 1 - 2.0 ** -24], device=DEV)
    for s in ({}, {"tau": 0.0}, {"top_k": 7}, {"top_k": 300}, {"top_k": 5000},
              {"top_p": 0.3}, {"top_p": 0.30011}, {"min_p": 0.5}, {"top_k": 4500, "top_p": 0.70001}):
        _check(z, u, **_named(6, s), on_border=True)
    ids, _, lps = binding.cis_sample_tokens(z, u, top_k=_full(6, 3, torch.int32),
                                            want_lp_sampled=True)
    assert ids.tolist() == [0, 2, 0, 4001, 2017, 2]
    assert float((lps + math.log(3)).abs().max()) <= 2.0 ** -22


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fill", ["lowest", "neg_inf", -1e30, -1e9])
def test_masked_vocabularies(dtype, fill):
    """Grammar masks of any of the usual values: only live tokens are sampled."""
    V = 20011
    low = {"lowest": torch.finfo(dtype).min, "neg_inf": -math.inf}.get(fill, fill)
    z = torch.full((8, V), low, dtype=dtype, device=DEV)
    live = torch.arange(301, V, 1111, device=DEV)
    z[:, live] = torch.linspace(-2, 3, live.numel(), device=DEV).to(dtype)
    z[6] = low
    z[6, 20010] = -5.0
    z[7] = low
    z[7, 0] = low if fill != "neg_inf" else 0.0
    g = _gen(3)
    u = torch.rand(8, generator=g, device=DEV)
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    for s in ({}, {"top_k": 50}, {"top_p": 0.9}, {"min_p": 0.1}, {"tau": 0.5, "top_p": 0.999},
              {"tau": 0.0}):
        _check(z, u, **_named(8, s))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_sets_with_unusual_values(dtype):
    """Kept sets beyond any list of candidates, with what a count of values has to look out for:
    exact zeros, tiny values of both signs, entries at 256 and above, masked ones at -1e9 and
    -inf, entries near -300 that weigh (a high temperature), a row of one value."""
    T, V = 10, 30001
    g = _gen(57)
    z = _rows(T, V, dtype, g, 3, 1, width=1.0).contiguous()
    z[1, ::3] = 0.0
    z[2, ::5] = 1e-20
    z[2, 1::5] = -1e-30
    z[3] += 300
    z[4, ::2] = -1e9
    z[5, ::2] = -math.inf
    z[6] -= 300
    z[7] = 0.0
    z[8] = -0.0
    z[9, ::4] = z[9, ::4] * 1e-8
    u = torch.rand(T, generator=g, device=DEV)
    for s in ({"top_p": 0.9}, {"top_p": 0.5, "tau": 0.5}, {"top_k": 9001}, {"min_p": 0.02},
              {"top_k": 20000, "top_p": 0.8, "min_p": 1e-3}, {"top_p": 0.95, "tau": 100.0},
              {"top_p": 0.999, "min_p": 0.3, "tau": 2.0}):
        _check(z, u, **_named(T, s), on_border=True)
        mixed = _named(T, s)
        mixed["top_p"] = mixed.get("top_p", _full(T, 1.0))
        mixed["top_p"][:5] = 1.0  # rows without it beside the others
        _check(z, u, **mixed, on_border=True)


def test_extreme_rows():
    """Large magnitudes and temperatures, maxima far apart, rows at the lowest values."""
    V = 3000
    g = _gen(9)
    z = _rows(8, V, torch.float32, g)
    z[0] += 1e6
    z[1] *= 1e30
    z[2] -= 1e9
    z[3] *= 1e-20
    z[4, 5] = 3e38
    z[5] = torch.finfo(torch.float32).min
    u = torch.rand(8, generator=g, device=DEV)
    for t in (1e-3, 0.05, 1.0, 30.0, 1000.0):
        for s in ({}, {"top_p": 0.9}, {"top_k": 12}, {"min_p": 0.3}):
            _check(z, u, **_named(8, {"tau": t, **s}))


def test_rows_that_cannot_be_sampled():
    """NaN, +inf, no finite logit, or a setting out of range: -1, NaN and the status, and the
    other rows as before."""
    T, V = 6, 500
    g = _gen(13)
    z = _rows(T, V, torch.bfloat16, g)
    u = torch.rand(T, generator=g, device=DEV)
    good = binding.cis_sample_tokens(z, u, want_lp_sampled=True)

    def bad(z, u, **kw):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ids, lp, lps = binding.cis_sample_tokens(z, u, want_lp_sampled=True, dev_status=st, **kw)
        assert int(st) == binding.CIS_ERR_BAD_INPUT
        assert int(ids[2]) == -1 and math.isnan(float(lp[2])) and math.isnan(float(lps[2]))
        keep = [0, 1, 3, 4, 5]
        for a, b in zip((ids, lp, lps), good):
            assert torch.equal(a[keep], b[keep])

    for v in (math.nan, math.inf):
        z2 = z.clone()
        z2[2, 77] = v
        bad(z2, u)
    z2 = z.clone()
    z2[2] = -math.inf
    bad(z2, u)
    for v in (-0.1, 1.0, math.nan, math.inf):
        u2 = u.clone()
        u2[2] = v
        bad(z, u2)
    for name, values, off in (("temperature", (-1.0, 1e-4, 2e3, math.nan, math.inf), 1.0),
                              ("top_p", (0.0, -0.5, 1.1, math.nan), 1.0),
                              ("min_p", (-0.1, 1.5, math.nan), 0.0)):
        for v in values:
            s = _full(T, off)
            s[2] = v
            bad(z, u, **{name: s})


@pytest.mark.parametrize("T", [153, 1000, 4700, 9000])
def test_many_rows_with_some_left(T):
    """More rows than CTAs, of which an uneven part, in runs, has a nucleus that no list holds:
    the same as in calls of a few rows, and every seventieth against the reference.  Masked rows
    and rows that cannot be sampled are among them."""
    V = 2501
    g = _gen(T)
    z = _rows(T, V, torch.bfloat16, g, width=0.3)
    i = torch.arange(T, device=DEV)
    peaked = (i // 61) % 3 == 0
    z[peaked, 17] = 14.0
    z[5::977, 3] = math.nan
    mask = (i % 11 != 10).to(torch.uint8)
    u = torch.rand(T, generator=g, device=DEV)
    p, tau = _full(T, 0.93), _full(T, 0.8)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ids, lp, lps = binding.cis_sample_tokens(z, u, temperature=tau, top_p=p, mask=mask,
                                             want_lp_sampled=True, dev_status=st)
    assert int(st) == binding.CIS_ERR_BAD_INPUT
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[5::977] = True
    on = (mask != 0) & ~bad
    assert bool((ids[~on] == -1).all()) and bool(((ids >= 0) & (ids < V))[on].all())
    for n in (30, 100):
        for a in list(range(0, T, n))[:40]:
            c = slice(a, a + n)
            few = binding.cis_sample_tokens(z[c], u[c], temperature=tau[c], top_p=p[c],
                                            mask=mask[c], want_lp_sampled=True)
            assert torch.equal(few[0], ids[c]), (n, a)
            for x, y in zip(few[1:], (lp[c], lps[c])):
                assert bool(((x - y).abs() <= 2.0 ** -19)[on[c]].all())
    r = on.nonzero().view(-1)[::70]
    want, wlp, wlps, near = _reference(z[r], u[r], tau[r], None, p[r])
    assert near > 2.0 ** -32
    assert torch.equal(ids[r].long(), want)
    assert float((lp[r].double() - wlp).abs().max()) <= 2.0 ** -19
    assert float((lps[r].double() - wlps).abs().max()) <= 2.0 ** -19


def test_frequencies():
    """20,000 draws from one small distribution: each count is binomial, so its distance
    from n p is below 5 sqrt(n p (1 - p)) + 1."""
    n = 20000
    g = _gen(21)
    row = torch.tensor([0.1, 2.0, -1.0, 0.5, 1.0, -3.0], device=DEV)
    z = row.expand(n, -1).contiguous()
    ids, _, _ = binding.cis_sample_tokens(z, torch.rand(n, generator=g, device=DEV))
    p = torch.softmax(row.double(), 0)
    c = torch.bincount(ids.long(), minlength=6).double()
    assert bool(((c - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt() + 1).all())


def test_repeats_streams_and_graphs():
    T, V = 40, 30000
    g = _gen(31)
    z = _rows(T, V, torch.bfloat16, g)
    u = torch.rand(T, generator=g, device=DEV)
    kw = dict(top_p=_full(T, 0.9), want_lp_sampled=True)
    a = binding.cis_sample_tokens(z, u, **kw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = binding.cis_sample_tokens(z, u, **kw)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = binding.cis_sample_tokens(z, u, **kw)
    for x in c:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for o in (b, c):
        for x, y in zip(o, a):
            assert torch.equal(x, y)
    assert binding.cis_sample_tokens(z[:0], u[:0])[0].shape == (0,)
    v = binding.cis_sample_tokens(z, u, V=777)[0]
    assert torch.equal(v, binding.cis_sample_tokens(z[:, :777].contiguous(), u)[0])
