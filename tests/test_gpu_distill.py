"""cis_distill_fwd_bwd against its formulas in 64 bits: the divergence of each row, the
gradient and the loss, at the sizes, lists and masks where they can go wrong.

Tolerances.  The kernel forms e^{(z - M) / tau} with the difference, the scale and the product
rounded (2.5 half-steps of |z - M| / tau, and 2^-22 of the exponential's own), sums them (2^-22)
and takes at most eight more roundings to a gradient, so that with c the row's factor
  |gradient's error| <= c (2^-20 (g p + q) + 2^-22 p |z - M| / tau),
g = 1 + q_r / p_r (forward), 2 + |l| + |L| (reverse), 1 (topk); then the output type's rounding.
L is a sum of terms q phi(d), each off by 2^-21 of itself and by the error of its d (2^-21 for
the sums', and 2^-23 |d|) times |q - p|: 2^-20 (sum |q - p| (1 + |d|) + sum q phi(d) + the rest
of the identity).
"""
import math

import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
KINDS = ["forward", "reverse", "topk"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _lists(z, K, tau, g, noise=0.5):
    T, V = z.shape
    x = (z.double() + noise * torch.randn(z.shape, generator=g, device=DEV)) / tau
    k = min(K, V)
    v, i = torch.topk(x, k, dim=1)
    ids = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    lp = torch.zeros((T, K), device=DEV)
    ids[:, :k] = i.int()
    lp[:, :k] = (v - torch.logsumexp(x, 1, keepdim=True)).float()
    return ids, lp


def _reference(z, ids, lp, kind, tau, tail_min=1e-6):
    """(L, tau dL/dz, its tolerance, L's) of every row, by the definitions in 64 bits."""
    T, V = z.shape
    x = z.double() / tau
    p = torch.softmax(x, 1)
    far = x.amax(1, keepdim=True) - x
    q = torch.zeros((T, V + 1), dtype=torch.float64, device=DEV)
    lq = torch.full((T, V + 1), -math.inf, dtype=torch.float64, device=DEV)
    on = (ids >= 0) & (lp > -math.inf)
    at = torch.where(on, ids, V).long()
    a = torch.where(on, lp.double(), -math.inf)
    if kind == "topk":
        a = torch.where(on, a - torch.logsumexp(a, 1, keepdim=True), -math.inf)
    lq.scatter_(1, at, a)
    q.scatter_(1, at, a.exp())
    q, lq = q[:, :V], lq[:, :V]
    inside = torch.zeros((T, V + 1), dtype=torch.bool, device=DEV).scatter_(1, at, on)[:, :V]
    logp = torch.log_softmax(x, 1)
    zero = torch.zeros_like(q)
    pr = p.masked_fill(inside, 0.0).sum(1, keepdim=True)
    qr = 1 - q.sum(1, keepdim=True)
    cut = far.clamp(max=1e4) * p
    if kind == "topk":
        d = torch.where(inside, lq - logp, zero)
        L = torch.where(q > 0, q * d, zero).sum(1)
        grad = torch.where(on.any(1, keepdim=True), p - q, zero)
        tol = 2.0 ** -20 * (p + q) + 2.0 ** -22 * cut
        phi = torch.where(inside, q * d - q + p, zero).sum(1) + pr[:, 0]
        some = (on.any(1)).double()
        tolL = 2.0 ** -20 * ((torch.where(inside, (q - p).abs() * (1 + d.abs()), zero).sum(1)
                              + phi.abs()) + pr[:, 0])
        return L * some, grad, tol, tolL
    if kind == "forward":
        qr = torch.where(qr < tail_min, 0.0, qr)
        Q = q.sum(1, keepdim=True) + qr
        d = torch.where(inside & (q > 0), lq - logp, zero)
        ratio = torch.where(qr > 0, qr / pr, 0.0)
        dr = torch.where(qr > 0, torch.log(ratio), 0.0)
        L = (q * d).sum(1) + (qr * dr)[:, 0]
        grad = torch.where(inside, Q * p - q, p * (Q - ratio))
        grad = torch.where((p == 0) & ~inside, zero, grad)
        tol = 2.0 ** -20 * (p * (1 + torch.where(inside, zero, ratio)) + q) + 2.0 ** -22 * cut
        tol = torch.where((p == 0) & ~inside, zero, tol)
        w = q
    else:
        qr = qr.clamp(min=tail_min)
        l = torch.where(inside, logp - lq, torch.log(pr) - torch.log(qr))
        l = torch.where(p > 0, l, zero)
        L = (p * l).sum(1)
        grad = p * (l - L.view(-1, 1))
        tol = (2.0 ** -20 * p * (2 + l.abs() + L.abs().view(-1, 1)) + 2.0 ** -22 * cut *
               (1 + l.abs() + L.abs().view(-1, 1)))
        d, dr, w = l, torch.where(pr > 0, torch.log(pr / qr), 0.0), p
    gap = torch.where(inside, (q - p).abs() * (1 + d.abs()), zero).sum(1) + (
        (qr - pr).abs() * (1 + dr.abs()))[:, 0]
    return L, grad, tol, 2.0 ** -20 * (gap + L.abs() + w.sum(1) * 2.0 ** -6)


def _check(z, ids, lp, kind, tau=1.0, grad_dtype=None, mask=None, weight=None, coef=1.0,
           dlogits=None, **kw):
    T, V = z.shape
    P = binding.cis_distill_default_params(kind, temperature=tau, coef=coef)
    out = binding.cis_distill_fwd_bwd(z, ids, lp, P, mask=mask, token_weight=weight,
                                      dlogits=dlogits, dlogits_dtype=grad_dtype, **kw)
    L, grad, tol, tolL = _reference(z, ids, lp, kind, tau)
    on = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask != 0
    c = on.double() / max(1, int(on.sum())) * coef
    if weight is not None:
        c = c * weight.double()
    L = torch.where(on, L, 0.0)
    assert binding.device_status(out["workspace"]) == 0
    kl = out["kl"].double()
    assert bool((kl[~on] == 0).all())
    fin = torch.isfinite(L)
    assert torch.equal(torch.isfinite(kl), fin)
    bad = ((kl - L).abs() > tolL + 2.0 ** -24 * L.abs() + 1e-12)[fin]
    assert not bool(bad.any()), (kl - L)[fin].abs().max()
    if bool(fin.all()):
        want = float((c * L).sum())
        assert abs(float(out["loss"]) - want) <= float((c.abs() * (tolL + 1e-12)).sum()) + \
            2.0 ** -23 * float((c * L).abs().sum())
    dz = out["dlogits"]
    g = (grad * (c / tau).view(-1, 1)).masked_fill(~on.view(-1, 1), 0.0)
    t = (tol * (c / tau).abs().view(-1, 1)).masked_fill(~on.view(-1, 1), 0.0)
    t = t + torch.finfo(dz.dtype).eps / 2 * (g.abs() + t) + 2.0 ** -126
    off = (dz.double() - g).abs() - t
    assert not bool((off > 0).any()), (float(off.max()), (off > 0).nonzero()[:4].tolist())
    return out


def _rows(T, V, dtype, g, pad=0, off=0, width=3.0):
    buf = (torch.randn(T * (V + pad) + off, generator=g, device=DEV) * width).to(dtype)
    return buf[off:].view(T, V + pad)[:, :V]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,V,K", [(3, 1, 1), (4, 2, 1), (3, 7, 3), (5, 8, 8), (2, 9, 4),
                                   (2, 31, 40), (3, 100, 1), (7, 1000, 33), (2, 4097, 64),
                                   (3, 16391, 100), (3, 32003, 256), (2, 45001, 17)])
def test_sizes_and_alignments(dtype, kind, T, V, K):
    """Rows that start at every offset from a 16-byte boundary, lists as long as the
    vocabulary and longer, one CTA to three a row."""
    g = _gen(V + K)
    for pad, off in ((0, 0), (3, 1), (8, 5)):
        z = _rows(T, V, dtype, g, pad, off)
        ids, lp = _lists(z, K, 1.0, g)
        _check(z, ids, lp, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_large_rows(kind):
    """The workloads' vocabulary (four CTAs a row in bf16, eight in fp32)."""
    g = _gen(5)
    for dtype in (torch.bfloat16, torch.float32):
        z = _rows(6, 151936, dtype, g)
        z[:, 1000:1040] += 12
        ids, lp = _lists(z, 64, 1.0, g)
        _check(z, ids, lp, kind, grad_dtype=torch.float32)
        _check(z, ids, lp, kind, grad_dtype=torch.bfloat16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tau", [1e-3, 0.05, 0.6, 1.0, 2.5, 40.0, 1000.0])
def test_temperatures(kind, tau):
    g = _gen(11)
    z = _rows(40, 5000, torch.float32, g, width=min(3.0, 3 * tau))
    ids, lp = _lists(z, 50, tau, g, noise=0.5 * min(1.0, tau))
    _check(z, ids, lp, kind, tau=tau, coef=tau * tau)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("above", [60.0, 87.0, 95.0, 104.0, 300.0])
def test_rest_far_below_the_list(kind, dtype, above):
    """A rest whose probability is at, or far below, the end of fp32's range, and a teacher who
    leaves it 0.3: the loss is finite, and the rest's gradients add up to -0.3 c (forward).
    An entry's share of that is e^{(z - max of the rest) / tau} / sum, so its error is that of the
    file's rule with the rest's maximum in M's place."""
    g = _gen(11)
    T, V, K, tau = 5, 5001, 16, 0.5
    z = _rows(T, V, dtype, g, width=0.5)
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:K] for _ in range(T)])
    z.scatter_(1, ids, z.gather(1, ids) + above * tau)
    lp = torch.log_softmax(torch.randn((T, K), generator=g, device=DEV), 1) + math.log(0.7)
    ids = ids.int()
    P = binding.cis_distill_default_params(kind, temperature=tau)
    out = binding.cis_distill_fwd_bwd(z, ids, lp, P, dlogits_dtype=torch.float32)
    L, grad, tol, tolL = _reference(z, ids, lp, kind, tau)
    assert bool(torch.isfinite(L).all())
    assert bool(((out["kl"].double() - L).abs() <= tolL + 2.0 ** -24 * L.abs()).all())
    inside = torch.zeros((T, V), dtype=torch.bool, device=DEV).scatter_(1, ids.long(), True)
    x = (z.double() / tau).masked_fill(inside, -math.inf)
    rest = (x.amax(1, keepdim=True) - x).masked_fill(inside, 0.0)
    tol = torch.where(inside, tol, grad.abs() * (2.0 ** -20 + 2.0 ** -22 * rest) + tol)
    c = 1 / (T * tau)
    off = (out["dlogits"].double() - c * grad).abs() - c * tol * (1 + 2.0 ** -24) \
        - 2.0 ** -24 * c * grad.abs() - 2.0 ** -126
    assert not bool((off > 0).any()), float(off.max())
    if kind == "forward":
        total = out["dlogits"].double().masked_fill(inside, 0.0).sum(1)
        assert bool(((total + 0.3 * c).abs() < 2.0 ** -18 * c).all())


@pytest.mark.parametrize("kind", KINDS)
def test_near_equal_distributions(kind):
    """Divergences far below their terms' size."""
    g = _gen(3)
    for noise in (1e-1, 1e-2, 1e-3):
        z = _rows(64, 3000, torch.float32, g)
        ids, lp = _lists(z, 128, 1.0, g, noise=noise)
        _check(z, ids, lp, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_masks_weights_and_short_lists(kind):
    g = _gen(23)
    T, V, K = 300, 2003, 24
    z = _rows(T, V, torch.bfloat16, g)
    ids, lp = _lists(z, K, 1.0, g)
    n = torch.randint(0, K + 1, (T, 1), generator=g, device=DEV)
    n[::7] = 0  # lists of nothing
    ids[torch.arange(K, device=DEV).view(1, -1) >= n] = -1
    lp[5, 2] = -math.inf  # an empty slot of the other form
    mask = (torch.rand(T, generator=g, device=DEV) > 0.3).to(torch.uint8) * 5
    w = torch.randn(T, generator=g, device=DEV)
    out = _check(z, ids, lp, kind, mask=mask, weight=w, coef=-0.7)
    none = (n.view(-1) == 0) | (mask == 0)
    assert bool((out["kl"][none].abs() <= 1e-12).all())
    assert bool((out["dlogits"][none] == 0).all())
    # no valid token at all
    P = binding.cis_distill_default_params(kind)
    out = binding.cis_distill_fwd_bwd(z, ids, lp, P, mask=torch.zeros_like(mask))
    assert float(out["loss"]) == 0 and not bool(out["dlogits"].any())


@pytest.mark.parametrize("kind", KINDS)
def test_sequence_mean_and_shards(kind):
    """s_t = 1 / (G |y_i|), and the batch's counts handed to the halves of a batch."""
    g = _gen(31)
    T, V, K = 60, 700, 9
    z = _rows(T, V, torch.float32, g)
    ids, lp = _lists(z, K, 1.0, g)
    cu = torch.tensor([0, 10, 10, 35, 60], dtype=torch.int32, device=DEV)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[7:10] = 0
    mask[20:40] = 0
    P = binding.cis_distill_default_params(kind, agg=binding.CIS_AGG_SEQ_MEAN_TOKEN_MEAN)
    out = binding.cis_distill_fwd_bwd(z, ids, lp, P, mask=mask, cu_seqlens=cu)
    L, grad, tol, tolL = _reference(z, ids, lp, kind, 1.0)
    s = torch.zeros(T, dtype=torch.float64, device=DEV)
    for a, b in ((0, 10), (10, 35), (35, 60)):
        s[a:b] = mask[a:b].double() / mask[a:b].sum() / 3
    t = s.view(-1, 1) * (tol + 2.0 ** -23 * grad.abs()) + 2.0 ** -126
    assert bool(((out["dlogits"].double() - s.view(-1, 1) * grad).abs() <= t).all())
    assert abs(float(out["loss"]) - float((s * L).sum())) <= float((s * (tolL + 2.0 ** -23 * L.abs())).sum())
    half = [(0, 10, cu[:2]), (10, 60, (cu[2:] - 10).contiguous())]
    counts = sum(binding.cis_count_valid(b - a, mask[a:b].contiguous(), c) for a, b, c in half)
    Q = binding.with_global_counts(P, counts)
    loss = 0.0
    for a, b, c in half:
        o = binding.cis_distill_fwd_bwd(z[a:b], ids[a:b], lp[a:b], Q, mask=mask[a:b].contiguous(),
                                        cu_seqlens=c)
        assert torch.equal(o["dlogits"], out["dlogits"][a:b])
        loss += float(o["loss"])
    assert abs(loss - float(out["loss"])) <= 1e-12


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fill", ["lowest", "neg_inf", -1e30, -1e9])
def test_masked_vocabularies(dtype, kind, fill):
    """All but a few entries masked by any of the usual values; lists that cover what is
    left, or go beyond it."""
    V = 3001
    low = {"lowest": torch.finfo(dtype).min, "neg_inf": -math.inf}.get(fill, fill)
    z = torch.full((4, V), low, dtype=dtype, device=DEV)
    live = torch.arange(100, 3000, 290, device=DEV)  # 10 tokens
    z[:, live] = torch.linspace(-1, 2, live.numel(), device=DEV).to(dtype)
    ids = torch.full((4, 12), -1, dtype=torch.int32, device=DEV)
    lp = torch.full((4, 12), -math.inf, device=DEV)
    ids[0, :10] = live.int()
    ids[1, :4] = live[:4].int()
    ids[2, :10] = live.flip(0).int()
    ids[3, :1] = live[:1].int()
    share = torch.tensor([0.3, 0.2, 0.15, 0.1, 0.08, 0.06, 0.05, 0.03, 0.02, 0.01], device=DEV)
    lp[0, :10] = share.log()
    lp[1, :4] = share[:4].log()
    lp[2, :10] = share.log()
    lp[3, 0] = math.log(0.9)
    _check(z, ids, lp, kind)
    if fill == "neg_inf":
        # a listed token that the student has at -inf: infinite, or 0 where p weighs
        ids[1, 4], lp[1, 4] = 50, math.log(0.01)
        out = _check(z, ids, lp, kind)
        assert math.isinf(float(out["kl"][1])) == (kind != "reverse")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_a_value(dtype, kind):
    """NaN, +inf or no finite logit: that row is NaN and its neighbours are as before."""
    g = _gen(41)
    z = _rows(6, 600, dtype, g)
    ids, lp = _lists(z, 8, 1.0, g)
    P = binding.cis_distill_default_params(kind)
    good = binding.cis_distill_fwd_bwd(z, ids, lp, P)
    z2 = z.clone()
    z2[0, 300] = math.nan
    z2[1, int(ids[1, 3])] = math.nan
    z2[2, 17 if 17 not in ids[2].tolist() else 18] = math.inf
    z2[3] = -math.inf
    out = binding.cis_distill_fwd_bwd(z2, ids, lp, P)
    assert bool(out["kl"][:4].isnan().all()) and bool(out["dlogits"][:4].isnan().any(1).all())
    assert torch.equal(out["dlogits"][4:], good["dlogits"][4:])
    assert torch.equal(out["kl"][4:], good["kl"][4:])
    assert math.isnan(float(out["loss"]))


def test_bad_lists():
    """Ids out of range or twice in a row: that row's status, NaN and zeros."""
    g = _gen(43)
    z = _rows(6, 600, torch.bfloat16, g)
    ids, lp = _lists(z, 40, 1.0, g)
    for kind in KINDS:
        P = binding.cis_distill_default_params(kind)
        good = binding.cis_distill_fwd_bwd(z, ids, lp, P)
        for bad in (600, -2, 2 ** 31 - 1, -2 ** 31, int(ids[2, 7])):
            i2 = ids.clone()
            i2[2, 33] = bad
            out = binding.cis_distill_fwd_bwd(z, i2, lp, P)
            assert binding.device_status(out["workspace"]) == binding.CIS_ERR_BAD_TOKEN_ID
            assert math.isnan(float(out["kl"][2])) and not bool(out["dlogits"][2].any())
            keep = [0, 1, 3, 4, 5]
            assert torch.equal(out["dlogits"][keep], good["dlogits"][keep])
            l2 = lp.clone()
            l2[2, 33] = -math.inf  # the same id in an empty slot
            out = binding.cis_distill_fwd_bwd(z, i2, l2, P)
            assert binding.device_status(out["workspace"]) == 0


@pytest.mark.parametrize("kind", KINDS)
def test_gradient_against_differences(kind):
    """(L(z + h e_j) - L(z - h e_j)) / 2h with h = 2^-6: each L is off by its tolerance, and
    the third derivative is at most (2 + |l| + |L|) p / 1 per entry, times h^2 / 6."""
    g = _gen(47)
    V, h = 23, 2.0 ** -6
    z = _rows(1, V, torch.float32, g, width=1.5).contiguous()
    ids, lp = _lists(z, 6, 1.0, g)
    P = binding.cis_distill_default_params(kind)
    dz = binding.cis_distill_fwd_bwd(z, ids, lp, P)["dlogits"][0].double()
    both = torch.cat([z + h * torch.eye(V, device=DEV), z - h * torch.eye(V, device=DEV)])
    rep = lambda x: x.expand(2 * V, -1).contiguous()  # noqa: E731
    kl = binding.cis_distill_fwd_bwd(both, rep(ids), rep(lp), P, want_grad=False)["kl"].double()
    step = (both[:V].double() - both[V:].double()).diagonal()
    diff = (kl[:V] - kl[V:]) / step
    L, grad, tol, tolL = _reference(both, rep(ids), rep(lp), kind, 1.0)
    p = torch.softmax(z.double(), 1)[0]
    size = 6 + float(L.abs().max()) + (float((grad / torch.softmax(both.double(), 1)).abs().max())
                                       if kind == "reverse" else 0)
    bound = (tolL[:V] + tolL[V:]) / step + p * size * h * h / 6 + 1e-7
    assert bool(((diff - dz).abs() <= bound).all()), ((diff - dz).abs() - bound).max()


def test_loss_alone_and_given_buffers():
    g = _gen(53)
    T, V = 50, 4100
    z = _rows(T, V, torch.bfloat16, g)
    ids, lp = _lists(z, 20, 1.0, g)
    P = binding.cis_distill_default_params("forward")
    out = binding.cis_distill_fwd_bwd(z, ids, lp, P)
    alone = binding.cis_distill_fwd_bwd(z, ids, lp, P, want_grad=False)
    assert alone["dlogits"] is None
    assert torch.equal(alone["kl"], out["kl"]) and torch.equal(alone["loss"], out["loss"])
    # rows with a stride of their own, lists as views of longer ones, V below the rows' length
    wide = torch.full((T, V + 11), 7.0, dtype=torch.float32, device=DEV)
    l2 = torch.full((T, 33), 0, dtype=torch.int32, device=DEV)
    p2 = torch.zeros((T, 33), device=DEV)
    l2[:, 5:25], p2[:, 5:25] = ids, lp
    ws = torch.empty(binding.cis_distill_workspace_size(T), dtype=torch.uint8, device=DEV)
    o2 = binding.cis_distill_fwd_bwd(z, l2[:, 5:25], p2[:, 5:25], P, dlogits=wide[:, 3:3 + V],
                                     workspace=ws)
    assert o2["workspace"] is ws and torch.equal(o2["kl"], out["kl"])
    assert torch.equal(wide[:, 3:3 + V].to(torch.bfloat16), out["dlogits"])
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + V:] == 7).all())
    short = binding.cis_distill_fwd_bwd(z, ids.clamp(max=3999) * 0 - 1, lp, P, V=4000)
    assert short["dlogits"].shape == (T, 4000)
    empty = binding.cis_distill_fwd_bwd(z[:0], ids[:0], lp[:0], P)
    assert float(empty["loss"]) == 0 and empty["dlogits"].shape == (0, V)


def test_repeats_streams_and_graphs():
    """Bit-identical on every call, on another stream, and replayed from a graph."""
    g = _gen(59)
    z = _rows(128, 9000, torch.bfloat16, g)
    ids, lp = _lists(z, 30, 1.0, g)
    P = binding.cis_distill_default_params("reverse")
    a = binding.cis_distill_fwd_bwd(z, ids, lp, P)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = binding.cis_distill_fwd_bwd(z, ids, lp, P)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = binding.cis_distill_fwd_bwd(z, ids, lp, P)
    for x in c.values():
        x.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for o in (b, c):
        for k in ("dlogits", "kl", "loss"):
            assert torch.equal(o[k], a[k])
