"""The calls around the LM head's step together, as an engine and a trainer make them.

Serving: norm with the residual to 8 bits, 8-bit logits, drafts sampled from a draft's logits,
their verification; the log-probabilities that it records are those of the forward call.
Training: the same norm before the fused LM head, its gradient from the head's.
"""
import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _e4m3(x):
    s = x.abs().amax(1) / 448
    return (x / s[:, None]).to(torch.float8_e4m3fn), s


def test_speculative_step():
    B, D, H, V = 6, 3, 512, 4001
    g = _gen(1)
    W, Ws = _e4m3(torch.randn(V, H, generator=g, device=DEV) / H ** 0.5)
    Wd, Wds = _e4m3(W.float() * Ws[:, None] + 0.01 * torch.randn(V, H, generator=g, device=DEV))
    norm = 1 + 0.1 * torch.randn(H, generator=g, device=DEV)
    x = (3 * torch.randn(B * (D + 1), H, generator=g, device=DEV)).to(BF)
    r = torch.randn(B * (D + 1), H, generator=g, device=DEV).to(BF)
    n = binding.cis_rmsnorm_fwd(x, norm, residual=r, want_y=False, want_q=True)
    z = binding.cis_lmhead_logits(n["q"], n["scale"], W, Ws)
    zd = binding.cis_lmhead_logits(n["q"], n["scale"], Wd, Wds)
    rows = torch.arange(B * (D + 1), device=DEV).view(B, D + 1)[:, :D].flatten()
    zd = zd[rows].contiguous()
    tau = torch.full((B,), 0.8, device=DEV)
    ids, _, _ = binding.cis_sample_tokens(zd, torch.rand(B * D, generator=g, device=DEV),
                                          temperature=tau.repeat_interleave(D))
    cu = torch.arange(0, B * D + 1, D, dtype=torch.int32, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    tok, kept, lp, lps = binding.cis_verify_tokens(
        z, ids, cu, torch.rand(B * D, generator=g, device=DEV),
        torch.rand(B, generator=g, device=DEV), D, draft_logits=zd, temperature=tau,
        draft_temperature=tau, want_lp_sampled=True, dev_status=st)
    assert int(st) == 0 and (kept >= 0).all() and kept.sum() > 0
    # what was recorded is what the forward call says of the same rows and tokens
    there = tok >= 0
    assert torch.equal(there.sum(1).int(), kept + 1)
    want = binding.cis_token_logprobs(z, tok.flatten().clamp(min=0))
    tol = 16 * 2.0 ** -20 + 2.0 ** -21 * want.abs()
    assert ((lp.flatten() - want).abs() <= tol)[there.flatten()].all()
    flat = torch.log_softmax(z.double() / 0.8, 1).gather(1, tok.flatten().clamp(min=0).long()[:, None])
    assert ((lps.flatten() - flat.view(-1)).abs() <= 16 * 2.0 ** -20 +
            2.0 ** -21 * flat.view(-1).abs())[there.flatten()].all()


def test_norm_around_the_fused_head():
    """Gradients through norm and head against the chain of their formulas in 64 bits, on the
    operands as they were rounded between the calls."""
    T, H, V, eps = 96, 256, 1000, 1e-6
    g = _gen(2)
    x, r, up = (torch.randn(T, H, generator=g, device=DEV).to(BF) for _ in range(3))
    norm = 1 + 0.1 * torch.randn(H, generator=g, device=DEV)
    W = (torch.randn(V, H, generator=g, device=DEV) / H ** 0.5).to(BF)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV).int()
    adv = torch.randn(T, generator=g, device=DEV)
    mask = (torch.rand(T, generator=g, device=DEV) > 0.25).to(torch.uint8)
    lpi = torch.full((T,), -6.5, device=DEV)
    P = binding.cis_default_params("none")
    n = binding.cis_rmsnorm_fwd(x, norm, residual=r, mask=mask)
    head = binding.cis_lmhead_fused(n["y"], W, ids, lpi, adv, P, mask=mask, grad_dtype=BF)
    back = binding.cis_rmsnorm_bwd(head["dhidden"], n["h"], norm, dh=up, mask=mask)
    on = mask != 0
    y, h = n["y"].double(), n["h"].double()
    z = y @ W.double().t()
    p = torch.softmax(z, 1)
    p[torch.arange(T), ids.long()] -= 1.0
    dz = p * (adv.double() * on / on.sum())[:, None]
    dy = dz @ W.double()
    size = dz.abs() @ W.double().abs()
    assert ((head["dhidden"].double() - dy).abs()[on] <=
            2.0 ** -8 * dy.abs()[on] + 2.0 ** -7 * size[on]).all()
    dy = head["dhidden"].double()
    rstd = torch.rsqrt(h.pow(2).mean(1, keepdim=True) + eps)
    gr = dy * norm.double()
    c = rstd.pow(2) * (gr * h).mean(1, keepdim=True)
    dx = (up.double() + rstd * (gr - h * c)) * on[:, None]
    tol = 2.0 ** -8 * dx.abs() + 1e-5 * (up.double().abs() + rstd * (gr.abs() + (h * c).abs()))
    assert ((back["dx"].double() - dx).abs() <= tol).all()
    per = (dy * h * rstd) * on[:, None]
    assert ((back["dweight"].double() - per.sum(0)).abs() <= 1e-5 * per.abs().sum(0)).all()


@pytest.mark.parametrize("plain", [True, False])
def test_native_calls_are_the_python_ones(plain, monkeypatch):
    """Both parts of the binding make the same calls."""
    T, H, V, D = 8, 256, 515, 3
    g = _gen(3)
    x, r = (torch.randn(T, H, generator=g, device=DEV).to(BF) for _ in range(2))
    norm = torch.ones(H, device=DEV)
    W, Ws = _e4m3(torch.randn(V, H, generator=g, device=DEV))
    u, ul = torch.rand(6, generator=g, device=DEV), torch.rand(2, generator=g, device=DEV)
    cu = torch.tensor([0, 3, 6], dtype=torch.int32, device=DEV)

    def calls():
        n = binding.cis_rmsnorm_fwd(x, norm, residual=r, want_q=True)
        b = binding.cis_rmsnorm_bwd(x, n["h"], norm, dh=r)
        z = binding.cis_lmhead_logits(n["q"], n["scale"], W, Ws)
        ids = z.float().argmax(1).int()[:6].contiguous()
        v = binding.cis_verify_tokens(z, ids, cu, u, ul, D, want_lp_sampled=True)
        return [n[k] for k in n] + [b[k] for k in b] + [z, *v]

    binding.lib()
    first = calls()
    if not plain:
        monkeypatch.setattr(binding, "_native", binding._PythonCalls())
    second = calls()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8))
               for a, b in zip(first, second))
