"""Host-side checks of the sampling, list and distillation calls: what the C ABI and the binding
refuse before any GPU work, and what they answer without any.  No kernel is launched."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2609_32444_gb300 import binding as b
    from paper_2609_32444_gb300 import build
    build.build()
    b.lib()
    return b


FAKE, OTHER, WS = (ctypes.c_void_p(x) for x in (0x10000, 0x4000000, 0x20000))
INVALID, UNSUPPORTED = 1, 2


def _sample(b, **over):
    a = dict(z=FAKE, dt=1, T=4, V=8, ld=8, u=FAKE, ids=FAKE)
    a.update(over)
    return b.lib().cis_sample_tokens(a["z"], a["dt"], a["T"], a["V"], a["ld"], a["u"], None, None,
                                     None, None, None, a["ids"], a.get("lp"), a.get("lps"), None,
                                     None)


def _topk(b, **over):
    a = dict(z=FAKE, dt=1, T=4, V=8, ld=8, K=3, tau=1.0, ids=FAKE, lp=FAKE)
    a.update(over)
    return b.lib().cis_topk_logprobs(a["z"], a["dt"], a["T"], a["V"], a["ld"], a["K"], a["tau"],
                                     None, a["ids"], a["lp"], None, None, None)


def _distill(b, params=(), **over):
    a = dict(z=FAKE, dt=1, T=4, V=8, ld=8, ids=FAKE, lp=FAKE, K=3, ldt=3, cu=None, B=0, dz=OTHER,
             dzt=1, ldo=8, ws=WS, nws=1 << 20)
    a.update(over)
    P = b.cis_distill_default_params()
    for k, v in dict(params).items():
        setattr(P, k, v)
    return b.lib().cis_distill_fwd_bwd(
        a["z"], a["dt"], a["T"], a["V"], a["ld"], a["ids"], a["lp"], a["K"], a["ldt"], None, None,
        a["cu"], a["B"], ctypes.byref(P), a["dz"], a["dzt"], a["ldo"], None, None, a["ws"],
        a["nws"], None)


ROWS = [dict(T=-1), dict(V=0), dict(V=-3), dict(ld=7), dict(dt=2), dict(dt=-1), dict(z=None),
        dict(z=ctypes.c_void_p(0x10001)), dict(dt=0, z=ctypes.c_void_p(0x10002)),
        dict(T=1 << 31), dict(V=1 << 31, ld=1 << 31)]


ODD = ctypes.c_void_p(0x30002)


@pytest.mark.parametrize("over", ROWS + [dict(u=None), dict(ids=None), dict(lp=OTHER, lps=OTHER),
                                         dict(u=ODD), dict(ids=ODD), dict(lp=ODD), dict(lps=ODD)])
def test_sample_refuses(binding, over):
    assert _sample(binding, **over) == INVALID


@pytest.mark.parametrize("over", ROWS + [
    dict(ids=None), dict(lp=None), dict(K=0), dict(K=257), dict(K=-1), dict(tau=0.0),
    dict(ids=ODD), dict(lp=ODD), dict(tau=-1.0), dict(tau=9e-4), dict(tau=1001.0), dict(tau=float("nan")),
    dict(tau=float("inf"))])
def test_topk_refuses(binding, over):
    assert _topk(binding, **over) == INVALID


@pytest.mark.parametrize("over", ROWS + [
    dict(ids=None), dict(lp=None), dict(K=0), dict(K=257), dict(K=4), dict(ldo=7), dict(dzt=3),
    dict(dz=ctypes.c_void_p(0x4000001)), dict(dz=ctypes.c_void_p(0x10010)), dict(ws=None),
    dict(ws=ctypes.c_void_p(0x20040)), dict(nws=64), dict(ids=ODD), dict(lp=ODD), dict(cu=ODD),
    dict(params=dict(kind=3)), dict(params=dict(kind=-1)), dict(params=dict(agg=2)),
    dict(params=dict(agg=1)), dict(params=dict(temperature=0.0)),
    dict(params=dict(temperature=float("nan"))), dict(params=dict(coef=float("inf"))),
    dict(params=dict(tail_min=0.0)), dict(params=dict(tail_min=0.6)),
    dict(params=dict(tail_min=float("nan")))])
def test_distill_refuses(binding, over):
    assert _distill(binding, **over) == INVALID


def test_rows_that_are_too_long(binding):
    n = 1 << 20
    assert _sample(binding, V=n + 1, ld=n + 1) == UNSUPPORTED
    assert _topk(binding, V=n + 1, ld=n + 1) == UNSUPPORTED
    far = ctypes.c_void_p(0x40000000)
    assert _distill(binding, V=819208, ld=819208, ldo=819208, dz=far) == UNSUPPORTED
    assert _distill(binding, dt=0, V=409608, ld=409608, ldo=409608, dz=far) == UNSUPPORTED
    n = 1 << 28
    assert _distill(binding, T=n, V=1, ld=1, ldo=1, dz=far, nws=1 << 40) == UNSUPPORTED


def test_no_rows_is_no_work(binding):
    assert _sample(binding, T=0, z=None, u=None, ids=None) == 0
    assert _topk(binding, T=0, z=None, ids=None, lp=None) == 0


def test_defaults_and_sizes(binding):
    P = binding.cis_distill_default_params()
    assert (P.kind, P.agg, P.temperature, P.coef, P.tail_min) == (0, 0, 1.0, 1.0, 1e-6)
    assert binding.cis_distill_default_params("topk", coef=2.0).coef == 2.0
    with pytest.raises(TypeError):
        binding.cis_distill_default_params("forward", lam=1.0)
    with pytest.raises(KeyError):
        binding.cis_distill_default_params("backward")
    L = binding.lib()
    assert L.cis_distill_default_params(None) == INVALID
    assert L.cis_distill_workspace_size(-1, ctypes.byref(ctypes.c_size_t())) == INVALID
    assert L.cis_distill_workspace_size(4, None) == INVALID
    assert binding.cis_distill_workspace_size(1000) >= 1000 * 12
    assert binding.status_string(16).startswith("CIS_ERR_BAD_INPUT")


def test_host_tensors_are_refused(binding):
    z, u = torch.zeros(4, 8), torch.zeros(4)
    ids, lp = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for f in (lambda: binding.cis_sample_tokens(z, u), lambda: binding.cis_topk_logprobs(z, 2),
              lambda: binding.cis_distill_fwd_bwd(z, ids, lp,
                                                  binding.cis_distill_default_params())):
        with pytest.raises(ValueError, match="libcis takes CUDA tensors"):
            f()
