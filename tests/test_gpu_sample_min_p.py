"""cis_sample_tokens with min_p = 1, which keeps a row's maxima alone, against counting them."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [0.0, 1.5, -2.0, 100.0])
def test_min_p_of_one(dtype, M):
    """min_p = 1 keeps the maxima alone, also where they are zeros of either sign: rows of
    maxima, more of them than any list holds, and rows less their maximum with a wide set."""
    T, V = 6, 9001
    g = _gen(19)
    z = (torch.randn((T, V), generator=g, device=DEV) * 0.5).clamp(max=0.0).to(dtype) + M
    z[0] = M
    z[1, ::3] = M - 1
    z[2, ::2] = M
    z[3] = M - 1
    z[3, 5000:] = M
    if M == 0.0:
        z[0] = -0.0
        z[2, ::4] = -0.0
        z[4:, 7] = -1e-20  # (bf16 rows with such a value are not counted)
    assert bool((z.float().amax(1) == M).all())
    u = torch.rand(T, generator=g, device=DEV)
    one = torch.ones(T, device=DEV)
    top = z.float() == M
    n = top.sum(1)
    j = (u.double() * n.double()).floor().long()  # the j-th maximum
    want = (top.cumsum(1) == (j + 1).view(-1, 1)).float().argmax(1)
    edge = (u.double() * n.double()).frac()
    assert bool((torch.minimum(edge, 1 - edge) / n > 2.0 ** -32).all())
    for kw in ({}, {"top_p": one * 0.999}, {"top_k": (one * 9000).int()},
               {"top_k": (one * 8000).int(), "top_p": one * 0.9995},
               {"temperature": one * 0.8}, {"temperature": one * 40.0, "top_p": one * 0.9999}):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ids, lp, lps = binding.cis_sample_tokens(z, u, min_p=one, want_lp_sampled=True,
                                                 dev_status=st, **kw)
        # (a nucleus or a top_k below the number of maxima: the rows it cuts among them)
        k = kw["top_k"].long() if "top_k" in kw else n
        full = (n <= k) & (n.double() <= 0.9 * V)
        if "top_p" not in kw:
            full = n <= k
        assert int(st) == 0
        assert torch.equal(ids.long()[full], want[full]), kw
        assert float((lps.double() + n.double().log())[full].abs().max()) <= 2.0 ** -20
        raw = torch.log_softmax(z.double(), 1).gather(1, want.view(-1, 1)).view(-1)
        assert float((lp.double() - raw)[full].abs().max()) <= 2.0 ** -19
        assert bool((ids >= 0).all())
