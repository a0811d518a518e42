"""cis_topk_logprobs against a stable sort and fp64 log-softmaxes.

Tokens have to be equal (ties to the lowest index).  Log-probabilities: the row's sum is right
to 2^-20 relative (fp32 exponentials, each to 2^-22, and their sums), and the difference is
rounded once: 2^-20 + 2^-23 |lp|; the logsumexp likewise.
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


def _rows(T, V, dtype, g, pad=0, off=0, width=3.0):
    buf = (torch.randn(T * (V + pad) + off, generator=g, device=DEV) * width).to(dtype)
    return buf[off:].view(T, V + pad)[:, :V]


def _check(z, K, tau=1.0, mask=None):
    T, V = z.shape
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ids, lp, lse = binding.cis_topk_logprobs(z, K, temperature=tau, mask=mask, want_lse=True,
                                             dev_status=st)
    x = z.double() + 0.0
    v, at = torch.sort(x, dim=1, descending=True, stable=True)
    n = min(K, V)
    top = v[:, :1]  # sums are taken from the maximum, whatever its size
    rest = torch.logsumexp((x - top) / tau, 1)
    e = rest + top.view(-1) / tau
    want = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    wlp = torch.full((T, K), -math.inf, dtype=torch.float64, device=DEV)
    want[:, :n] = at[:, :n].int()
    wlp[:, :n] = (v[:, :n] - top) / tau - rest.view(-1, 1)
    want[wlp == -math.inf] = -1
    if mask is not None:
        off = mask == 0
        want[off], wlp[off], e[off] = -1, -math.inf, 0.0
    assert int(st) == 0
    assert torch.equal(ids, want), (ids != want).nonzero()[:5].tolist()
    fin = torch.isfinite(wlp.float())  # (values beyond fp32's range are infinite in it)
    assert torch.equal(torch.isfinite(lp), fin) and bool((lp[~fin] == -math.inf).all())
    far = (lp.double() - wlp)[fin].abs()
    assert bool((far <= 2.0 ** -20 + 2.0 ** -23 * wlp[fin].abs()).all()), far.max()
    big = torch.isinf(e.float())
    assert torch.equal(lse[big], e.float()[big])
    assert bool(((lse.double() - e).abs() <= 2.0 ** -20 + 2.0 ** -23 * e.abs())[~big].all())
    return ids, lp, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,K", [(3, 1, 1), (3, 1, 5), (4, 2, 1), (5, 7, 7), (4, 8, 3),
                                   (3, 33, 200), (6, 255, 256), (5, 1000, 1), (6, 1000, 100),
                                   (4, 4097, 256), (3, 16391, 17), (3, 32003, 128),
                                   (2, 60001, 33)])
def test_sizes_and_alignments(dtype, T, V, K):
    g = _gen(V + K)
    for pad, off in ((0, 0), (3, 1), (8, 5)):
        _check(_rows(T, V, dtype, g, pad, off), K)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K", [1, 20, 64, 256])
def test_large_vocabulary(dtype, K):
    """Bell-shaped rows (in bf16 many equal entries), flat and peaked ones."""
    g = _gen(K)
    for width in (0.2, 3.0, 12.0):
        _check(_rows(9, 151936, dtype, g, width=width), K)


@pytest.mark.parametrize("tau", [1e-3, 0.3, 2.0, 1000.0])
def test_temperature_and_mask(tau):
    g = _gen(7)
    T = 200
    z = _rows(T, 3001, torch.float32, g)
    mask = (torch.rand(T, generator=g, device=DEV) > 0.4).to(torch.uint8) * 9
    _check(z, 30, tau, mask)
    _check(z, 30, tau, torch.zeros_like(mask))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_and_order(dtype):
    """Equal entries, sorted and reversed rows, both zeros, the largest ones side by side."""
    V = 9001
    z = torch.zeros((8, V), dtype=dtype, device=DEV)
    z[1] = -0.0
    z[2, ::3] = -0.0
    z[3] = torch.linspace(-8, 8, V, device=DEV).to(dtype)
    z[4] = torch.linspace(8, -8, V, device=DEV).to(dtype)
    z[5, 5000:5300] = 4.0
    z[6, 1::30] = 1.0
    z[7] = torch.finfo(dtype).min
    for K in (1, 2, 100, 256):
        _check(z, K)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fill", ["lowest", "neg_inf", -1e30, -1e9])
def test_masked_vocabularies(dtype, fill):
    V = 20011
    low = {"lowest": torch.finfo(dtype).min, "neg_inf": -math.inf}.get(fill, fill)
    z = torch.full((4, V), low, dtype=dtype, device=DEV)
    live = torch.arange(301, V, 1111, device=DEV)
    z[:3, live] = torch.linspace(-2, 3, live.numel(), device=DEV).to(dtype)
    z[3, 7] = -4.0
    for K in (1, 5, live.numel(), 40, 256):
        _check(z, K)


def test_rows_without_a_value():
    g = _gen(13)
    z = _rows(6, 700, torch.float32, g)
    good = binding.cis_topk_logprobs(z, 9, want_lse=True)
    z2 = z.clone()
    z2[0, 3] = math.nan
    z2[1, 699] = math.inf
    z2[2] = -math.inf
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ids, lp, lse = binding.cis_topk_logprobs(z2, 9, want_lse=True, dev_status=st)
    assert int(st) == binding.CIS_ERR_BAD_INPUT
    assert bool((ids[:3] == -1).all()) and bool(lp[:3].isnan().all()) and bool(lse[:3].isnan().all())
    for a, b in zip((ids, lp, lse), good):
        assert torch.equal(a[3:], b[3:])


def test_extreme_rows():
    g = _gen(9)
    z = _rows(6, 3000, torch.float32, g)
    z[0] += 1e6
    z[1] *= 1e30
    z[2] -= 1e9
    z[3] *= 1e-20
    z[4, 5] = 3e38
    for tau in (1e-3, 1.0, 50.0):
        _check(z, 64, tau)


def test_repeats_streams_and_graphs():
    g = _gen(31)
    z = _rows(100, 30000, torch.bfloat16, g)
    a = binding.cis_topk_logprobs(z, 50, want_lse=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = binding.cis_topk_logprobs(z, 50, want_lse=True)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = binding.cis_topk_logprobs(z, 50, want_lse=True)
    for x in c:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for o in (b, c):
        for x, y in zip(o, a):
            assert torch.equal(x, y)
    assert binding.cis_topk_logprobs(z[:0], 3)[0].shape == (0, 3)
    v = binding.cis_topk_logprobs(z, 9, V=777)
    assert torch.equal(v[0], binding.cis_topk_logprobs(z[:, :777].contiguous(), 9)[0])
