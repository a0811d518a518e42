"""cis_distill_fwd_bwd with lists that hold nearly all of the teacher's probability: the rest's q_r
is 1 less their sum, down to 2e-6, and the divergence and the rest's gradients have its precision.

q_r is taken from the given log-probabilities in 64 bits.  Tolerances are those of the
distillation's other tests, of the rest's own size: L is off by 2^-20 (sum |q - p| (1 + |d|) + L +
2^-6), the rest's gradient by c 2^-20 (Q p_r + q_r) of an entry's share of p_r (forward), or
c 2^-20 p_r (2 + |l_r| + |L|) of it (reverse), and 2^-22 |z - max of the rest| / tau of itself.
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


@pytest.mark.parametrize("kind", ["forward", "reverse"])
@pytest.mark.parametrize("K", [1, 20, 256])
@pytest.mark.parametrize("share", [3e-6, 2e-5, 1e-3])
def test_rest_that_the_teacher_all_but_excludes(kind, K, share):
    T, V = 200, 1003
    g = torch.Generator(device=DEV)
    g.manual_seed(K)
    z = torch.randn((T, V), generator=g, device=DEV)
    ids = torch.stack([torch.randperm(V, generator=g, device=DEV)[:K] for _ in range(T)])
    z.scatter_(1, ids, z.gather(1, ids) + 14 * torch.rand((T, 1), generator=g, device=DEV))
    a = torch.log_softmax(2 * torch.randn((T, K), generator=g, device=DEV, dtype=torch.float64), 1)
    lp = (a + math.log1p(-share)).float()
    q = lp.double().exp()
    qr = 1 - q.sum(1)
    assert float(qr.min()) > 2e-6  # above tail_min in every row (of the inputs alone)
    P = binding.cis_distill_default_params(kind)
    out = binding.cis_distill_fwd_bwd(z, ids.int(), lp, P)
    logp = torch.log_softmax(z.double(), 1)
    p = logp.exp()
    inside = torch.zeros_like(p, dtype=torch.bool).scatter_(1, ids, True)
    rest = logp.masked_fill(inside, -math.inf)
    lpr = torch.logsumexp(rest, 1)
    pr, part = lpr.exp(), torch.softmax(rest, 1)
    pk, d = p.gather(1, ids), lp.double() - logp.gather(1, ids)
    dr = qr.log() - lpr
    if kind == "forward":
        L = (q * d).sum(1) + qr * dr
        grad, size = pr - qr, pr + qr
    else:
        L = -(pk * d).sum(1) - pr * dr
        grad, size = pr * (-dr - L), pr * (2 + dr.abs() + L.abs())
    gap = ((q - pk).abs() * (1 + d.abs())).sum(1) + (qr - pr).abs() * (1 + dr.abs())
    off = (out["kl"].double() - L).abs() - 2.0 ** -20 * (gap + L.abs() + 2.0 ** -6)
    assert not bool((off > 0).any()), float(off.max())
    far = (rest.amax(1, keepdim=True) - rest).masked_fill(inside, 0.0)
    got = (out["dlogits"].double() * T).masked_fill(inside, 0.0)
    want = part * grad.view(-1, 1)
    tol = 2.0 ** -20 * part * size.view(-1, 1) + 2.0 ** -22 * far * want.abs() + 2.0 ** -24 * want.abs()
    off = (got - want).abs() - tol - 2.0 ** -126 * T
    assert not bool((off > 0).any()), float((off / want.abs().clamp(min=1e-30)).max())
