"""Host-side refusals of the calls around the LM head's decoding step.  No call gets as far as
the GPU: every argument set but the last of each list is refused by the host's checks."""
import ctypes
import os
import shutil

import pytest
import torch

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not os.path.exists("/usr/local/cuda/bin/nvcc"),
                                reason="needs nvcc to build libcis")

P = 4096  # stands for an aligned device pointer; never followed


@pytest.fixture(scope="module")
def binding():
    from paper_2609_32444_gb300 import build, binding as b
    build.build()
    b.lib()
    return b


def _call(f, names, base, **over):
    d = dict(zip(names, base))
    for k, v in over.items():
        assert k in d
        d[k] = v
    return f(*[d[k] for k in names])


FWD = ("x", "dtype", "T", "H", "ld_x", "r", "ld_r", "w", "wdt", "eps", "mask", "h", "y", "q", "s",
       "stream")
FWD_OK = (P, 1, 4, 64, 64, None, 0, P, 0, 1e-6, None, None, P, None, None, None)


@pytest.mark.parametrize("over,rc", [
    (dict(x=None), 1), (dict(w=None), 1), (dict(T=-1), 1), (dict(H=0), 1), (dict(ld_x=63), 1),
    (dict(dtype=2), 1), (dict(wdt=5), 1), (dict(eps=0.0), 1), (dict(eps=float("nan")), 1),
    (dict(y=None), 1), (dict(q=P), 1), (dict(s=P), 1), (dict(r=P, ld_r=63), 1), (dict(x=P + 1), 1),
    (dict(w=P + 2), 1), (dict(y=P + 1), 1), (dict(q=P, s=P + 2), 1), (dict(dtype=0, h=P + 2), 1),
    (dict(H=16385, ld_x=16385), 2), (dict(T=0), 0)])
def test_norm_refusals(binding, over, rc):
    assert _call(binding.lib().cis_rmsnorm_fwd, FWD, FWD_OK, **over) == rc


BWD = ("dy", "h", "dtype", "T", "H", "ld_dy", "ld_h", "w", "wdt", "dh", "ld_dh", "eps", "mask",
       "dx", "dw", "ws", "nws", "stream")
BWD_OK = (P, P, 1, 4, 64, 64, 64, P, 0, None, 0, 1e-6, None, P, P, P, 1 << 20, None)


@pytest.mark.parametrize("over,rc", [
    (dict(dy=None), 1), (dict(h=None), 1), (dict(dx=None), 1), (dict(dw=None), 1),
    (dict(ws=None), 1), (dict(ws=P + 64), 1), (dict(nws=1023), 1), (dict(ld_dy=1), 1),
    (dict(ld_h=1), 1), (dict(dh=P, ld_dh=9), 1), (dict(dx=P + 1), 1), (dict(dw=P + 2), 1),
    (dict(eps=1.5), 1), (dict(T=1 << 31), 1), (dict(H=20000, ld_dy=20000, ld_h=20000), 2)])
def test_norm_gradient_refusals(binding, over, rc):
    assert _call(binding.lib().cis_rmsnorm_bwd, BWD, BWD_OK, **over) == rc


def test_norm_workspace(binding):
    n = ctypes.c_size_t()
    f = binding.lib().cis_rmsnorm_bwd_workspace_size
    assert f(4, 64, None) == 1 and f(-1, 64, ctypes.byref(n)) == 1
    assert f(4, 0, ctypes.byref(n)) == 1 and f(4, 16385, ctypes.byref(n)) == 2
    sizes = [binding.cis_rmsnorm_bwd_workspace_size(T, 64) for T in (0, 1, 5, 1000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] >= 256 and sizes[2] >= 5 * 64 * 4


HEAD = ("x", "xs", "w", "ws", "T", "H", "V", "z", "dtype", "ld", "status", "stream")
HEAD_OK = (P, P, P, P, 4, 64, 100, P, 1, 100, None, None)


@pytest.mark.parametrize("over,rc", [
    (dict(x=None), 1), (dict(xs=None), 1), (dict(w=None), 1), (dict(ws=None), 1),
    (dict(z=None), 1), (dict(T=-1), 1), (dict(H=0), 1), (dict(V=0), 1), (dict(ld=99), 1),
    (dict(dtype=3), 1), (dict(x=P + 8), 1), (dict(w=P + 1), 1), (dict(z=P + 1), 1),
    (dict(xs=P + 2), 1), (dict(status=P + 1), 1), (dict(H=24), 2), (dict(T=0, x=None), 0)])
def test_logits_refusals(binding, over, rc):
    assert _call(binding.lib().cis_lmhead_logits, HEAD, HEAD_OK, **over) == rc


VER = ("z", "dtype", "B", "N", "V", "ld", "ids", "cu", "D", "zd", "ldd", "u", "ul", "tau", "taud",
       "mask", "tok", "kept", "lp", "lps", "status", "ws", "nws", "stream")
VER_OK = (P, 1, 2, 6, 100, 100, P, P, 3, P, 100, P, P, None, None, None, P, P, None, None, None, P,
          1 << 20, None)


@pytest.mark.parametrize("over,rc", [
    (dict(z=None), 1), (dict(ids=None), 1), (dict(cu=None), 1), (dict(u=None), 1),
    (dict(ul=None), 1), (dict(tok=None), 1), (dict(kept=None), 1), (dict(ws=None), 1),
    (dict(ws=P + 128), 1), (dict(nws=255), 1), (dict(B=-1), 1), (dict(B=(1 << 20) + 1), 1),
    (dict(N=-1), 1), (dict(N=7), 1), (dict(V=0), 1), (dict(ld=99), 1), (dict(ldd=99), 1),
    (dict(D=-1), 1), (dict(D=65), 1), (dict(dtype=7), 1), (dict(z=P + 1), 1), (dict(zd=P + 1), 1),
    (dict(u=P + 2), 1), (dict(kept=P + 1), 1), (dict(lp=P, lps=P), 1),
    (dict(V=(1 << 20) + 1, ld=1 << 21, ldd=1 << 21), 2), (dict(B=0, N=0, z=None, ids=None), 0)])
def test_verification_refusals(binding, over, rc):
    assert _call(binding.lib().cis_verify_tokens, VER, VER_OK, **over) == rc


def test_verification_workspace(binding):
    n = ctypes.c_size_t()
    f = binding.lib().cis_verify_workspace_size
    assert f(1, 100, 4, None) == 1 and f(-1, 100, 4, ctypes.byref(n)) == 1
    assert f(1, 0, 4, ctypes.byref(n)) == 1 and f(1, 100, 65, ctypes.byref(n)) == 1
    # 32 bytes for each row and stretch at least
    for B, V, D in ((0, 10, 0), (1, 151936, 4), (64, 151936, 4), (256, 1000, 16), (3, 1 << 20, 64)):
        assert binding.cis_verify_workspace_size(B, V, D) >= 32 * B * (D + 1)


def test_host_tensors_are_refused(binding):
    x, w = torch.zeros(2, 64), torch.ones(64)
    q = x.to(torch.float8_e4m3fn)
    for call in (lambda: binding.cis_rmsnorm_fwd(x, w), lambda: binding.cis_rmsnorm_bwd(x, x, w),
                 lambda: binding.cis_lmhead_logits(q, w[:2], q, w[:2]),
                 lambda: binding.cis_verify_tokens(x, w[:1].int(), w[:2].int(), w[:1], w[:1], 1)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
