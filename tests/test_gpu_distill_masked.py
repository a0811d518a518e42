"""cis_distill_fwd_bwd where the student masks tokens that the teacher lists (logits at the type's
lowest value, -1e30, -1e9 or -inf), and where the rest is masked as a whole, at several
temperatures: the divergence and the gradient against the definitions in 64 bits.

Tolerances are those of the distillation's other tests: a gradient is off by
c (2^-20 p (2 + |l| + |L|) + 2^-22 p |z - M| / tau (1 + |l| + |L|)) under reverse,
c (2^-20 (p + q) + 2^-22 p |z - M| / tau) otherwise, and L by
2^-20 (sum |q - p| (1 + |d|) + |L| + 2^-6), each with the output's rounding.
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


def _reverse(z, ids, lp, tau, tail_min=1e-6):
    """L, tau dL/dz and their tolerances, outcome by outcome; ids without empty slots."""
    x = z.double() / tau
    top = x.amax(1, keepdim=True)
    logZ = torch.logsumexp(x - top, 1, keepdim=True)
    logp = x - top - logZ
    p = logp.exp()
    inside = torch.zeros_like(x, dtype=torch.bool).scatter_(1, ids.long(), True)
    a = torch.zeros_like(x).scatter_(1, ids.long(), lp.double())
    pr = p.masked_fill(inside, 0.0).sum(1, keepdim=True)
    qr = (1 - lp.double().exp().sum(1, keepdim=True)).clamp(min=tail_min)
    l = torch.where(inside, logp - a, pr.log() - qr.log())
    l = torch.where(p > 0, l, 0.0)
    L = (p * l).sum(1, keepdim=True)
    grad = p * (l - L)
    size = l.abs() + L.abs()
    cut = (top - x).clamp(max=1e4) * p
    tol = 2.0 ** -20 * p * (2 + size) + 2.0 ** -22 * cut * (1 + size)
    q = torch.where(inside, a.exp(), 0.0)
    gap = torch.where(inside, (q - p).abs() * (1 + l.abs()), 0.0).sum(1)
    lr = torch.where(pr > 0, (pr / qr).log(), 0.0)
    gap = gap + ((pr - qr).abs() * (1 + lr.abs()))[:, 0]
    return L[:, 0], grad, tol, 2.0 ** -20 * (gap + L[:, 0].abs() + 2.0 ** -6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fill", ["lowest", -1e30, -1e9, -1e4])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("first", [True, False])
def test_reverse_with_listed_tokens_that_the_student_masks(dtype, fill, tau, first):
    """A grammar masks the student and not the teacher, whose list then has masked tokens at any
    place; the live ones' gradients and the rest's are what they are without them.  The last
    rows' rest is masked as a whole."""
    T, V, K = 6, 3001, 40
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    z = (torch.randn((T, V), generator=g, device=DEV) * 2).to(dtype)
    low = torch.finfo(dtype).min if fill == "lowest" else fill
    order = torch.stack([torch.randperm(V, generator=g, device=DEV) for _ in range(T)])
    ids = order[:, :K]
    off = ids[:, :3] if first else ids[:, -3:]
    z.scatter_(1, off, low)
    z[1].scatter_(0, ids[1, :K - 1], low)  # one live token
    live = ids[4:, 5:20]  # rows whose only live tokens are listed
    keep = z[4:].gather(1, live)
    z[4:] = low
    z[4:].scatter_(1, live, keep)
    lp = torch.log_softmax(torch.randn((T, K), generator=g, device=DEV), 1) + math.log(0.9)
    P = binding.cis_distill_default_params("reverse", temperature=tau)
    out = binding.cis_distill_fwd_bwd(z, ids.int(), lp, P, dlogits_dtype=torch.float32)
    L, grad, tol, tolL = _reverse(z, ids, lp, tau)
    assert bool(torch.isfinite(L).all())
    kl = out["kl"].double()
    assert bool(((kl - L).abs() <= tolL + 2.0 ** -24 * L.abs()).all()), (kl, L)
    c = 1 / (T * tau)
    off = (out["dlogits"].double() - c * grad).abs() - c * tol * (1 + 2.0 ** -24) \
        - 2.0 ** -24 * c * grad.abs() - 2.0 ** -126
    assert not bool((off > 0).any()) and not bool(off.isnan().any()), float(off.max())


@pytest.mark.parametrize("tau", [0.5, 1.0])
def test_reverse_with_a_token_that_the_teacher_all_but_excludes(tau):
    """A listed log-probability of -1e9, on the student's likeliest token and on an unlikely one:
    the gradients of the other outcomes keep their precision."""
    T, V, K = 4, 2003, 20
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    z = torch.randn((T, V), generator=g, device=DEV)
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:K] for _ in range(T)])
    lp = torch.log_softmax(torch.randn((T, K), generator=g, device=DEV), 1) + math.log(0.8)
    z[0, ids[0, 4]] = 8.0
    z[1, ids[1, 4]] = -30.0
    z[2].scatter_(0, ids[2], -40.0)  # the list all but nothing, its largest the excluded one
    z[2, ids[2, 4]] = -25.0
    lp[:3, 4] = -1e9
    P = binding.cis_distill_default_params("reverse", temperature=tau)
    out = binding.cis_distill_fwd_bwd(z, ids.int(), lp, P)
    L, grad, tol, tolL = _reverse(z, ids, lp, tau)
    assert bool(((out["kl"].double() - L).abs() <= tolL + 2.0 ** -24 * L.abs()).all())
    c = 1 / (T * tau)
    off = (out["dlogits"].double() - c * grad).abs() - c * tol * (1 + 2.0 ** -24) \
        - 2.0 ** -24 * c * grad.abs() - 2.0 ** -126
    assert not bool((off > 0).any()) and not bool(off.isnan().any()), float(off.max())


@pytest.mark.parametrize("kind", ["forward", "topk"])
@pytest.mark.parametrize("fill", ["lowest", -1e9])
def test_other_kinds_with_listed_tokens_that_the_student_masks(kind, fill):
    """L is the masked tokens' share times how far they are masked; the gradients are p - q."""
    T, V, K, tau = 5, 3001, 30, 1.0
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    z = torch.randn((T, V), generator=g, device=DEV) * 2
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:K] for _ in range(T)])
    low = torch.finfo(torch.float32).min if fill == "lowest" else fill
    z.scatter_(1, ids[:, :2], low)
    lp = torch.log_softmax(torch.randn((T, K), generator=g, device=DEV), 1) + math.log(0.9)
    P = binding.cis_distill_default_params(kind, temperature=tau)
    out = binding.cis_distill_fwd_bwd(z, ids.int(), lp, P)
    x = z.double() / tau
    logp = x - x.amax(1, keepdim=True)
    logp = logp - torch.logsumexp(logp, 1, keepdim=True)
    p = logp.exp()
    a = lp.double()
    if kind == "topk":
        a = a - torch.logsumexp(a, 1, keepdim=True)
    q = torch.zeros_like(p).scatter_(1, ids, a.exp())
    inside = torch.zeros_like(p, dtype=torch.bool).scatter_(1, ids, True)
    qr = 1 - a.exp().sum(1, keepdim=True) if kind == "forward" else torch.zeros((T, 1), device=DEV)
    pr = p.masked_fill(inside, 0.0).sum(1, keepdim=True)
    L = (a.exp() * (a - logp.gather(1, ids))).sum(1)
    if kind == "forward":
        L = L + (qr * (qr / pr).log())[:, 0]
    assert bool(((out["kl"].double() - L).abs() <= 2.0 ** -20 * L.abs()).all())
    ratio = qr / pr
    grad = torch.where(inside, p - q, p * (1 - ratio))
    top = x.amax(1, keepdim=True)
    tol = 2.0 ** -20 * (p * (1 + torch.where(inside, torch.zeros_like(p), ratio)) + q) \
        + 2.0 ** -22 * (top - x).clamp(max=1e4) * p
    off = (out["dlogits"].double() - grad / T).abs() - tol / T * (1 + 2.0 ** -24) \
        - 2.0 ** -24 * grad.abs() / T - 2.0 ** -126
    assert not bool((off > 0).any()), float(off.max())
