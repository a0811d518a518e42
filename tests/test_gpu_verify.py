"""cis_verify_tokens against its definition in 64 bits.

Tokens and counts are equal: the reference says how near its decisions were to their borders,
and the test asserts that none of its inputs is within 2^-33.  The kernel's masses are right to
2^-35 of each: u q against p is off by twice that, relative to the larger (the sums of both rows
and, in fp64, the two entries), and a running sum of p - q and its goal by twice that each, relative
to the rows' masses of 1.  log-probabilities: the row's mass is summed to
6 x 2^-20 (fp32 exponentials, each right to 2^-22, as the sampler's), and the difference from it is
rounded to fp32 once or twice: 8 x 2^-20 + 2^-22 |lp|.
"""
import math

import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
BF, F32 = torch.bfloat16, torch.float32
BAD_ID, BAD_INPUT = binding.CIS_ERR_BAD_TOKEN_ID, binding.CIS_ERR_BAD_INPUT
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _reference(z, ids, cu, u, u_last, D, zd=None, tau=None, tau_d=None, mask=None):
    """tokens, kept, lp, lps, and the least distance of a decision from its border."""
    B, near = len(cu) - 1, 1.0
    tok = torch.full((B, D + 1), -1)
    kept = torch.full((B,), -1)
    lp, lps = torch.zeros(B, D + 1).double(), torch.zeros(B, D + 1).double()
    for b in range(B):
        if mask is not None and not mask[b]:
            continue
        t = 1.0 if tau is None else float(tau[b].double())
        td = 1.0 if tau_d is None else float(tau_d[b].double())
        n = cu[b + 1] - cu[b]
        for i in range(n + 1):
            x = z[cu[b] + b + i].double()
            p = torch.softmax(x / t, 0) if t > 0 else torch.zeros_like(x)
            if t == 0:
                p[int((x == x.max()).nonzero()[0])] = 1.0
            q, token = None, None
            if i < n:
                d, r = int(ids[cu[b] + i]), float(u[cu[b] + i].double())
                if zd is None or t == 0 or td == 0:
                    q = torch.zeros_like(p)
                    q[d] = 1.0
                else:
                    q = torch.softmax(zd[cu[b] + i].double() / td, 0)
                if t > 0:
                    a, c = r * float(q[d]), float(p[d])
                    near = min(near, abs(a - c) / max(a, c) if max(a, c) > 0 else 1.0)
                if (float(p[d]) > 0 if t == 0 else r * float(q[d]) < float(p[d])):
                    token = d
            if token is None:
                m = p if q is None else (p - q).clamp(min=0)
                near = min(near, abs(float(m.sum()) * 2.0 ** 32 - 1))
                m = m if float(m.sum()) * 2.0 ** 32 > 1 else p
                c = m.cumsum(0)
                goal = float(u_last[b].double()) * float(c[-1])
                token = int((c <= goal).sum())
                if t == 0:
                    token = int(p.argmax())
                else:
                    near = min(near, float((c - goal)[m > 0].abs().min()) or 1.0)
                kept[b] = i
            tok[b, i] = token
            lp[b, i] = torch.log_softmax(x, 0)[token]
            lps[b, i] = torch.log_softmax(x / t, 0)[token] if t > 0 else 0.0
            if kept[b] >= 0:
                break
    return tok, kept, lp, lps, near


def _close(got, want):
    got, want = got.double().cpu(), want.cpu()
    assert ((got - want).abs() <= 8 * 2.0 ** -20 + 2.0 ** -22 * want.abs()).all()


def _check(z, ids, cu, u, ul, D, zd=None, tau=None, tau_d=None, mask=None, V=None):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd, temperature=tau,
                                    draft_temperature=tau_d, mask=mask, V=V, want_lp_sampled=True,
                                    dev_status=st)
    cut = (lambda x: x) if V is None else (lambda x: None if x is None else x[:, :V])
    want = _reference(cut(z), ids.cpu(), cu.tolist(), u.cpu(), ul.cpu(), D, cut(zd), tau, tau_d,
                      mask)
    assert want[4] > 2.0 ** -33
    assert int(st) == 0
    assert got[0].cpu().tolist() == want[0].tolist() and got[1].cpu().tolist() == want[1].tolist()
    _close(got[2], want[2])
    _close(got[3], want[3])
    again = binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd, temperature=tau,
                                      draft_temperature=tau_d, mask=mask, V=V,
                                      want_lp_sampled=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    return got


def _case(B, D, V, dtype, seed, ragged=True, noise=0.8, pad=0, width=2.5):
    g = _gen(seed)
    n = torch.full((B,), D)
    if ragged and B > 1:
        n = torch.randint(0, D + 1, (B,), generator=torch.Generator().manual_seed(seed))
        n[0] = D
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = n.cumsum(0)
    N = int(cu[-1])
    of = torch.repeat_interleave(torch.arange(B), n)
    row = (torch.arange(N) + of).to(DEV)
    full = width * torch.randn(N + B, V + pad, generator=g, device=DEV)
    full[:, ::max(V // 37, 1)] += 4.0
    fd = full[row] + noise * torch.randn(N, V + pad, generator=g, device=DEV)
    z, zd = full.to(dtype), fd.to(dtype)
    ids = torch.empty(N, dtype=torch.int32, device=DEV)
    if N:
        e = torch.empty(N, V, device=DEV).exponential_(generator=g)
        ids = (zd[:, :V].float() - torch.log(e)).argmax(1).int()
    u = torch.rand(N, generator=g, device=DEV)
    ul = torch.rand(B, generator=g, device=DEV)
    if pad:
        z[:, V:], zd[:, V:] = float("nan"), float("nan")
    return z, zd, ids, cu.to(DEV), u, ul


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,D,V", [(1, 0, 1), (1, 1, 1), (1, 1, 2), (3, 2, 7), (1, 4, 1000),
                                   (5, 3, 1001), (2, 64, 130), (40, 3, 515), (1, 4, 32003),
                                   (7, 5, 8192), (3, 2, 40001), (160, 2, 2048), (320, 1, 300),
                                   (1, 16, 4099), (2, 1, 151936)])
def test_drafts_of_a_model(B, D, V, dtype):
    z, zd, ids, cu, u, ul = _case(B, D, V, dtype, B * 7 + D * 3 + V)
    _check(z, ids, cu, u, ul, D, zd=zd)
    tau = torch.full((B,), 0.7, device=DEV)
    tau_d = 0.5 + torch.rand(B, generator=_gen(V), device=DEV)
    _check(z, ids, cu, u, ul, D, zd=zd, tau=tau, tau_d=tau_d)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,D,V", [(1, 1, 1), (3, 2, 7), (1, 4, 32003), (40, 3, 515),
                                   (3, 2, 40001)])
def test_drafts_that_were_looked_up(B, D, V, dtype):
    z, zd, ids, cu, u, ul = _case(B, D, V, dtype, B + D + V, width=1.0)
    N = ids.numel()
    if N:  # half of them the target's likeliest
        of = torch.repeat_interleave(torch.arange(B, device=DEV), (cu[1:] - cu[:-1]).long())
        best = z[torch.arange(N, device=DEV) + of].float().argmax(1).int()
        z[torch.arange(N, device=DEV) + of, best.long()] += 6.0
        ids = torch.where(torch.rand(N, generator=_gen(1), device=DEV) < 0.5, best, ids)
    _check(z, ids, cu, u, ul, D)
    _check(z, ids, cu, u, ul, D, zd=zd, tau_d=torch.zeros(B, device=DEV))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_settings_of_their_own(dtype):
    """Temperatures from 0 to 20, masked requests, more slots than drafts, rows of a wider tensor."""
    B, D, V = 48, 6, 3001
    z, zd, ids, cu, u, ul = _case(B, D, V, dtype, 5, pad=3)
    tau = 0.3 + 1.2 * torch.rand(B, generator=_gen(2), device=DEV)
    tau[::5] = 0.0
    tau[1], tau[2] = 20.0, 0.05
    tau_d = 0.5 + torch.rand(B, generator=_gen(3), device=DEV)
    tau_d[::7] = 0.0
    mask = (torch.rand(B, generator=_gen(4), device=DEV) > 0.2).to(torch.uint8)
    mask[:3] = 1
    tok, kept, lp, lps = _check(z, ids, cu, u, ul, D + 2, zd=zd, tau=tau, tau_d=tau_d, mask=mask,
                                V=V)
    off = mask == 0
    assert (tok[off] == -1).all() and (kept[off] == -1).all() and (lp[off] == 0).all()
    _check(z[:, :V], ids, cu, u, ul, D, tau=tau, mask=mask)


def test_ties_and_forbidden_tokens():
    """-inf in either row, rows of equal logits, and the first of equal maxima."""
    V, g = 4003, _gen(6)
    z = torch.randn(6, V, generator=g, device=DEV)
    zd = z[[0, 1, 3, 4]] + 0.5 * torch.randn(4, V, generator=g, device=DEV)
    z[:, 100:3000] = -INF            # the target forbids them
    zd[0, 3000:] = -INF              # the draft forbids what the target wants
    zd[2:, 50:] = -INF
    z[3:] = torch.where(z[3:] > -INF, torch.zeros_like(z[3:]), z[3:])
    cu = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    for seed in range(12):
        r = _gen(seed)
        u, ul = torch.rand(4, generator=r, device=DEV), torch.rand(2, generator=r, device=DEV)
        ids = torch.randint(0, V, (4,), generator=r, device=DEV).int()
        ids[2] = seed
        for t in (None, torch.tensor([0.8, 0.0], device=DEV), torch.tensor([0.0, 1.5], device=DEV)):
            _check(z, ids, cu, u, ul, 2, zd=zd, tau=t)
            _check(z, ids, cu, u, ul, 2, tau=t)


def test_the_same_distribution_keeps_everything():
    """u q < q for every u below 1, down to the last bit."""
    B, D, V = 3, 4, 5003
    z, _, _, cu, _, ul = _case(B, D, V, F32, 8, ragged=False)
    of = torch.repeat_interleave(torch.arange(B, device=DEV), (cu[1:] - cu[:-1]).long())
    zd = z[torch.arange(B * D, device=DEV) + of].clone()
    u = torch.full((B * D,), 1.0 - 2.0 ** -24, device=DEV)
    ids = torch.randint(0, V, (B * D,), generator=_gen(1), device=DEV).int()
    got = binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd)
    assert (got[1] == D).all() and torch.equal(got[0][:, :D].flatten(), ids)
    # all of p on one token, looked up
    z[:] = -INF
    z[:, 17] = 3.0
    ids[:] = 17
    got = binding.cis_verify_tokens(z, ids, cu, u, ul, D)
    assert (got[1] == D).all() and (got[0] == 17).all()
    assert (got[2] == 0).all()


def test_decisions_next_to_their_border():
    """u a step of fp32 on either side of p / q: what fp32 sums cannot tell, whole numbers do."""
    V, g = 20011, _gen(3)
    n = 24
    z = 2.0 * torch.randn(2 * n, V, generator=g, device=DEV)
    zd = z[::2] + 0.3 * torch.randn(n, V, generator=g, device=DEV)
    p, q = torch.softmax(z[::2].double(), 1), torch.softmax(zd.double(), 1)
    ids = ((p < q) & (p > 1e-7)).float().multinomial(1, generator=g).view(-1)
    ratio = (p / q).gather(1, ids[:, None]).view(-1)
    u = ratio.float()
    below, above = u.double() < ratio, u.double() > ratio
    cu = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    ul = torch.rand(n, generator=g, device=DEV)
    for k in (-1, 0, 1):
        v = (u.view(torch.int32) + k).view(F32)
        side = v.double() < ratio
        clear = (v.double() / ratio - 1).abs() > 2.0 ** -34
        got = binding.cis_verify_tokens(z, ids.int(), cu, v, ul, 1, draft_logits=zd)
        assert torch.equal((got[1] == 1)[clear], side[clear]) and clear.sum() >= n - 1
    assert below.any() and above.any()


def _one(n=2, V=300):
    g = _gen(1)
    z = torch.randn(n + 1, V, generator=g, device=DEV)
    zd = z[:n] - 0.1
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    ids = torch.arange(n, device=DEV).int()
    return z, zd, ids, cu, torch.full((n,), 0.5, device=DEV), torch.full((1,), 0.5, device=DEV)


def _status(*a, **k):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = binding.cis_verify_tokens(*a, want_lp_sampled=True, dev_status=st, **k)
    return int(st), out


def _refused(res, bit):
    st, (tok, kept, lp, lps) = res
    assert st == bit and (tok == -1).all() and (kept == -1).all()
    assert lp.isnan().all() and lps.isnan().all()


@pytest.mark.parametrize("bad", [math.nan, INF])
def test_rows_that_cannot_be_used(bad):
    z, zd, ids, cu, u, ul = _one()
    u[:] = 0.0  # everything is kept
    ok = _status(z, ids, cu, u, ul, 2, draft_logits=zd)
    assert ok[0] == 0 and int(ok[1][1]) == 2
    for t in (z, zd):
        for i in range(len(t)):
            keep = t[i, 7].clone()
            t[i, 7] = bad
            _refused(_status(z, ids, cu, u, ul, 2, draft_logits=zd), BAD_INPUT)
            t[i, 7] = keep
    z[1] = -INF
    _refused(_status(z, ids, cu, u, ul, 2, draft_logits=zd), BAD_INPUT)
    # a row behind the last token is not looked at
    z[0, int(ids[0])] = -INF
    st, out = _status(z, ids, cu, u, ul, 2, draft_logits=zd)
    assert st == 0 and int(out[1]) == 0
    zd[1], ids[1], u[1] = bad, -5, 3.0
    st, again = _status(z, ids, cu, u, ul, 2, draft_logits=zd)
    assert st == 0 and all(torch.equal(a, b) for a, b in zip(out, again))


def test_drafts_and_numbers_out_of_range():
    z, zd, ids, cu, u, ul = _one()
    u[:] = 0.0
    for bad in (-1, 300, 1 << 30, -(1 << 31)):
        x = ids.clone()
        x[1] = bad
        _refused(_status(z, x, cu, u, ul, 2, draft_logits=zd), BAD_ID)
        _refused(_status(z, x, cu, u, ul, 2), BAD_ID)
    for bad in (-0.25, 1.0, math.nan):
        x = u.clone()
        x[1] = bad
        _refused(_status(z, ids, cu, x, ul, 2, draft_logits=zd), BAD_INPUT)
        _refused(_status(z, ids, cu, u, ul * 0 + bad, 2, draft_logits=zd), BAD_INPUT)
    for bad in (-1.0, 1e-4, 1e4, math.nan, INF):
        t = torch.full((1,), bad, device=DEV)
        _refused(_status(z, ids, cu, u, ul, 2, draft_logits=zd, temperature=t), BAD_INPUT)
        _refused(_status(z, ids, cu, u, ul, 2, draft_logits=zd, draft_temperature=t), BAD_INPUT)
    for bad in ([0, 3], [-1, 2], [2, 0], [1, 1 << 30]):
        x = torch.tensor(bad, dtype=torch.int32, device=DEV)
        _refused(_status(z, ids, x, u, ul, 2, draft_logits=zd), BAD_INPUT)
    # more drafts than a request may have, in one request of two: the other one is served
    z2 = torch.cat([z, z[:1]])
    x = torch.tensor([0, 2, 2], dtype=torch.int32, device=DEV)
    st, (tok, kept, lp, _) = _status(z2, ids, x, u, ul.repeat(2), 1, draft_logits=zd)
    assert st == BAD_INPUT and kept.tolist() == [-1, 0] and int(tok[1, 0]) >= 0
    assert lp[0].isnan().all() and lp[1].isfinite().all()


@pytest.mark.parametrize("tau", [1.0, 1e-3, 1e3])
def test_offsets_that_decrease(tau):
    """The request whose range is none is refused; those that come to share a row with another one
    get some tokens of the vocabulary, and requests before them their own."""
    B, D, V, N = 5, 6, 2051, 9
    z, zd, ids, _, u, ul = _case(B, D, V, F32, 31, ragged=False)
    z, zd, ids, u = z[:N + B], zd[:N], ids[:N], u[:N]
    t = torch.tensor([1.0, 1.0, 1.0, tau, 1.0], device=DEV)
    good = torch.tensor([0, 3, 6, 8, 8, N], dtype=torch.int32, device=DEV)
    bad = torch.tensor([0, 3, 8, 5, 9, 9], dtype=torch.int32, device=DEV)
    for q in (zd, None):
        k = dict(draft_logits=q, temperature=t)
        st, (tok, kept, _, _) = _status(z, ids, bad, u, ul, D, **k)
        assert st & BAD_INPUT and kept[2] == -1 and (tok[2] == -1).all()
        assert (tok >= -1).all() and (tok < V).all() and (kept >= -1).all() and (kept <= D).all()
        want = _status(z, ids, good, u, ul, D, **k)[1]
        assert torch.equal(tok[0], want[0][0]) and kept[0] == want[1][0]


def test_refusals():
    z, zd, ids, cu, u, ul = _one()
    f = binding.cis_verify_tokens
    for bad in (lambda: f(z[:2], ids, cu, u, ul, 2), lambda: f(z, ids, cu, u[:1], ul, 2),
                lambda: f(z, ids.long(), cu, u, ul, 2), lambda: f(z, ids, cu.long(), u, ul, 2),
                lambda: f(z, ids, cu, u, ul.repeat(2), 2), lambda: f(z, ids, cu, u, ul, 65),
                lambda: f(z, ids, cu, u, ul, -1), lambda: f(z, ids, cu, u, ul, 1),
                lambda: f(z, ids, cu, u, ul, 2, draft_logits=zd[:1]),
                lambda: f(z, ids, cu, u, ul, 2, draft_logits=zd.bfloat16()),
                lambda: f(z, ids, cu, u, ul, 2, V=301), lambda: f(z.t(), ids, cu, u, ul, 2),
                lambda: f(z, ids, cu, u, ul, 2, temperature=ul.double()),
                lambda: f(z, ids.cpu(), cu, u, ul, 2)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        f(z.half(), ids, cu, u, ul, 2)


def test_guard_bands_and_no_requests():
    """The C call writes its outputs and its workspace's bytes, and nothing else."""
    B, D, V = 5, 3, 2050
    z, zd, ids, cu, u, ul = _case(B, D, V, BF, 12)
    pad, n = 32, B * (D + 1)
    L, p = binding.lib(), binding._ptr
    big = {k: torch.full((m + 2 * pad,), 77, dtype=d, device=DEV)
           for k, m, d in (("tok", n, torch.int32), ("kept", B, torch.int32), ("lp", n, F32),
                           ("lps", n, F32))}
    v = {k: x[pad:-pad] for k, x in big.items()}
    need = binding.cis_verify_workspace_size(B, V, D)
    ws = torch.full((need + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    assert L.cis_verify_tokens(p(z), 1, B, ids.numel(), V, V, p(ids), p(cu), D, p(zd), V, p(u),
                               p(ul), None, None, None, p(v["tok"]), p(v["kept"]), p(v["lp"]),
                               p(v["lps"]), None, p(ws), need, binding._stream()) == 0
    torch.cuda.synchronize()
    for x in big.values():
        assert (x[:pad] == 77).all() and (x[-pad:] == 77).all()
    assert (ws[need:] == 0x5A).all()
    want = binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd, want_lp_sampled=True)
    for a, b in zip(("tok", "kept", "lp", "lps"), want):
        assert torch.equal(v[a], b.flatten())
    none = binding.cis_verify_tokens(z[:0], ids[:0], cu[:1], u[:0], ul[:0], D)
    assert none[0].shape == (0, D + 1) and none[1].shape == (0,)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1e-3, 1.0, 300.0, 1e4, 1e7, 1e30])
def test_extreme_logits_and_temperatures(size, dtype):
    """Rows around +-size, temperatures at both ends of their range."""
    B, D, V = 12, 2, 777
    z, zd, ids, cu, u, ul = _case(B, D, V, dtype, 3)
    z, zd = (z.float() * size).to(dtype), (zd.float() * size).to(dtype)
    z[::2] -= 20 * size
    for t in (1e-3, 1.0, 1e3):
        tau = torch.full((B,), t, device=DEV)
        _check(z, ids, cu, u, ul, D, zd=zd, tau=tau, tau_d=tau)
        _check(z, ids, cu, u, ul, D, tau=tau)


def test_outputs_that_are_not_asked_for():
    z, zd, ids, cu, u, ul = _case(5, 3, 4001, BF, 9)
    tau = torch.full((5,), 0.6, device=DEV)
    full = binding.cis_verify_tokens(z, ids, cu, u, ul, 3, draft_logits=zd, temperature=tau,
                                     want_lp_sampled=True)
    for lp in (False, True):
        for lps in (False, True):
            got = binding.cis_verify_tokens(z, ids, cu, u, ul, 3, draft_logits=zd, temperature=tau,
                                            want_lp=lp, want_lp_sampled=lps)
            assert (got[2] is not None) == lp and (got[3] is not None) == lps
            assert all(a is None or torch.equal(a, b) for a, b in zip(got, full))


def test_rows_far_apart():
    """Row strides whose offsets pass 2^31 elements."""
    z, zd, ids, cu, u, ul = _case(2, 1, 4001, BF, 4, ragged=False)
    ld = 1_300_000_001
    far = torch.empty(5 * ld, dtype=BF, device=DEV)
    z2, zd2 = far[:4 * ld].view(4, ld)[:, :4001], far[2 * ld + 7000:4 * ld + 7000]
    zd2 = zd2.view(2, ld)[:, :4001]
    z2.copy_(z)
    zd2.copy_(zd)
    got = binding.cis_verify_tokens(z2, ids, cu, u, ul, 1, draft_logits=zd2)
    want = binding.cis_verify_tokens(z, ids, cu, u, ul, 1, draft_logits=zd)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))


@pytest.mark.parametrize("B,D,V", [(1, 0, 3), (1, 4, 40001), (7, 64, 300), (64, 4, 20000),
                                   (130, 3, 2500), (700, 2, 300), (33, 1, 151936)])
@pytest.mark.parametrize("two", [True, False])
def test_workspace_is_as_long_as_it_says(B, D, V, two):
    z, zd, ids, cu, u, ul = _case(B, D, V, BF, B + V, ragged=False)
    need = binding.cis_verify_workspace_size(B, V, D)
    ws = torch.full((need + 65536,), 0x5A, dtype=torch.uint8, device=DEV)
    L, p = binding.lib(), binding._ptr
    tok = torch.empty(B, D + 1, dtype=torch.int32, device=DEV)
    kept = torch.empty(B, dtype=torch.int32, device=DEV)
    for n in (ids.numel(), 0):  # as many drafts as there may be, and none
        c = cu if n else torch.zeros_like(cu)
        assert L.cis_verify_tokens(p(z), 1, B, n, V, V, p(ids), p(c), D, p(zd) if two else None, V,
                                   p(u), p(ul), None, None, None, p(tok), p(kept), None, None,
                                   None, p(ws), need, binding._stream()) == 0
        torch.cuda.synchronize()
        assert (ws[need:] == 0x5A).all() and (kept >= 0).all()


def test_two_graphs_with_a_workspace_each():
    """Captured on streams of their own and replayed at once, on new inputs."""
    B, D, V = 6, 4, 32000
    sets = [list(_case(B, D, V, BF, s, ragged=False)) for s in (1, 2)]
    graphs, outs = [], []
    for z, zd, ids, cu, u, ul in sets:
        ws = torch.empty(binding.cis_verify_workspace_size(B, V, D), dtype=torch.uint8, device=DEV)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd,
                                                  workspace=ws))
        graphs.append((g, s, ws))
    for seed in (11, 21):
        for k, x in enumerate(sets):
            for a, b in zip(x, _case(B, D, V, BF, seed + k, ragged=False)):
                a.copy_(b)
        torch.cuda.synchronize()
        for g, s, _ in graphs:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (z, zd, ids, cu, u, ul), got in zip(sets, outs):
            want = binding.cis_verify_tokens(z, ids, cu, u, ul, D, draft_logits=zd)
            assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))


def _nearly_equal_rows(B, V, dtype, seed):
    """Requests of one draft, rejected.  Near the end are five likely tokens, of which the second is
    a bf16 step (0.125) below the first in p and the draft; in the draft's row the two change places.
    Token 0, of 1.7e-4 to 1.9e-4 of the mass, is a step higher there, so that p is above q in all the
    others' equal logits by 2.2e-5 to 2.6e-5 of itself.  The other entries are 0 in both rows and have
    e^-31.2 to e^-32.4 of the mass: 0.2 to 0.9 units of 2^-60 are left of each."""
    g = torch.Generator().manual_seed(seed)
    z = torch.zeros(2 * B, V)
    x = 31.2 + 1.2 * torch.rand(B, 1, generator=g)
    share = 0.2 + torch.rand(B, 5, generator=g)
    top = (x + torch.log(share / share.sum(1, keepdim=True))).bfloat16().float()
    top[:, 1] = top[:, 0] - 0.125
    z[::2, V - 40:V - 15:5] = top
    z[::2, 0] = (torch.logsumexp(top, 1) + math.log(1.8e-4)).bfloat16().float()
    z[1::2] = z[::2]
    assert (z >= 0).all() and (z[:, z[0] != 0] >= 16).all() and (z < 31.875).all()
    zd = z[::2].clone()
    zd[:, V - 40], zd[:, V - 35] = z[::2, V - 35], z[::2, V - 40]
    zd[:, 0] += 0.125
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    ids = torch.full((B,), V - 35, dtype=torch.int32, device=DEV)
    u = torch.full((B,), 1.0 - 2.0 ** -24, device=DEV)
    return z.to(DEV, dtype), zd.to(DEV, dtype), ids, cu, u


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(300, 32000), (30, 151936)])
def test_little_is_left_of_many_entries(B, V, dtype):
    """What is left of such entries is lost in whole numbers, and must not come out below 0."""
    z, zd, ids, cu, u = _nearly_equal_rows(B, V, dtype, V)
    ul = 0.01 + 0.98 * torch.rand(B, generator=_gen(V), device=DEV)
    _, kept, _, _ = _check(z, ids, cu, u, ul, 1, zd=zd)
    assert (kept == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(300, 32000), (30, 151936)])
def test_the_first_of_what_is_left(B, V, dtype):
    """u_last = 0: the first entry of which something is left, wherever the sums say that it begins;
    not one which p has no more of than q."""
    z, zd, ids, cu, u = _nearly_equal_rows(B, V, dtype, V + 1)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    tok, kept, _, _ = binding.cis_verify_tokens(z, ids, cu, u, torch.zeros(B, device=DEV), 1,
                                                draft_logits=zd, dev_status=st)
    assert int(st) == 0 and (kept == 0).all()
    j = tok[:, :1].long()
    p, q = (torch.log_softmax(x.double(), 1).gather(1, j) for x in (z[::2], zd))
    assert (p > q).all()
