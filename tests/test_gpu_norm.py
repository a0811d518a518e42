"""cis_rmsnorm_fwd and cis_rmsnorm_bwd against their formulas in 64 bits.

Tolerances, with u = 2^-24 (an fp32 rounding, relative): a row's sum of at most 16384 squares
goes through 32 additions in a thread, 5 and 4 across lanes and warps, each square rounded
once: 42 u, 21 u of its root; with the mean, eps, the root and the division 25 u.  An entry of
y takes h's rounding, the weight's and r's product: 28 u, then one rounding to the type, half
a step.  In the gradient the two sums are right to 42 u of the sum of their terms' sizes, c to
42 + 2 x 25 + 3 u of the same, and the rest adds 5 roundings: 100 u of the sizes added up.
dweight: 28 u a term, and the additions of a thread's rows and of the CTAs' sums.
"""
import math

import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
U = 2.0 ** -24
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


def _rand(T, H, g, dtype, scale=1.0, pad=0):
    """[T, H] rows; pad: columns behind them, which no call may touch."""
    x = (torch.randn((T, H + pad), generator=g, device=DEV) * scale).to(dtype)
    x[:, ::17] *= 11.0
    x[:, H:] = float("nan")
    return x[:, :H]


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _check_fwd(out, x, w, r, mask, eps, dtype):
    T, H = x.shape
    h = x.double() + (0 if r is None else r.double())
    on = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask != 0
    h[~on] = 0
    y = h * torch.rsqrt(h.pow(2).mean(1, keepdim=True) + eps) * w.double()
    if r is None:
        assert out["h"] is None
    else:
        tol = (_half(dtype) + U) * h.abs() + torch.finfo(dtype).tiny
        assert ((out["h"].double() - h).abs() <= tol).all()
    if out["y"] is not None:
        tol = (_half(dtype) + 29 * U) * y.abs() + torch.finfo(dtype).tiny
        assert ((out["y"].double() - y).abs() <= tol).all()
    if out["q"] is not None:
        sc = y.abs().amax(1).clamp(min=2.0 ** -100) / 448
        got = out["scale"].double()
        assert (out["scale"][~on] == 0).all() and (out["q"].float()[~on] == 0).all()
        assert ((got - sc)[on].abs() <= 31 * U * sc[on]).all()
        v = y / sc[:, None]
        # half a step of 3 mantissa bits; below 2^-6 the step is 2^-9
        tol = (2.0 ** -4 + 62 * U) * v.abs()
        tol = torch.where(v.abs() < 2.0 ** -6, 2.0 ** -10 + 62 * U * v.abs(), tol)
        assert ((out["q"].double() - v).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H", [(1, 1), (1, 64), (5, 63), (7, 256), (3, 264), (33, 512), (4, 519),
                                 (2, 1000), (9, 2048), (6, 2531), (3, 4096), (2, 8191), (3, 8192),
                                 (2, 8200), (1, 16383), (1, 16384), (1300, 128), (700, 777)])
def test_forward(T, H, dtype):
    g = _gen(T * 31 + H)
    x, r = _rand(T, H, g, dtype), _rand(T, H, g, dtype, 0.7)
    mask = (torch.rand(T, generator=g, device=DEV) > 0.3).to(torch.uint8)
    for w in ((1 + 0.2 * torch.randn(H, generator=g, device=DEV)).to(d) for d in (BF, F32)):
        for res, m, want_y, want_q in ((r, None, True, True), (None, mask, True, False),
                                       (r, mask, False, True), (None, None, False, True)):
            out = binding.cis_rmsnorm_fwd(x, w, residual=res, eps=1e-6, mask=m, want_y=want_y,
                                          want_q=want_q)
            assert (out["y"] is not None) == want_y and (out["q"] is not None) == want_q
            _check_fwd(out, x, w, res, m, 1e-6, dtype)


def _check_bwd(out, dy, h, w, dh, mask, eps, dtype):
    T, H = h.shape
    h, dy, w = h.double(), dy.double(), w.double()
    d = torch.zeros_like(h) if dh is None else dh.double()
    if mask is not None:
        off = mask == 0
        h, dy, d = (v.masked_fill(off[:, None], 0.0) for v in (h, dy, d))
    r = torch.rsqrt(h.pow(2).mean(1, keepdim=True) + eps)
    g = dy * w
    c = r * r * (g * h).mean(1, keepdim=True)
    size_c = r * r * (g * h).abs().mean(1, keepdim=True)
    dx = d + r * (g - h * c)
    if mask is not None:
        dx[off] = 0
    size = d.abs() + r * (g.abs() + h.abs() * size_c)
    tol = 100 * U * size + _half(dtype) * dx.abs() + torch.finfo(dtype).tiny
    assert ((out["dx"].double() - dx).abs() <= tol).all()
    per = dy * h * r
    adds = 28 + 4 + 32 + 5 + T / 100  # a term; R warps; the second kernel; a CTA's rows
    tol = adds * U * per.abs().sum(0) + torch.finfo(F32).tiny
    assert ((out["dweight"].double() - per.sum(0)).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H", [(1, 1), (1, 64), (5, 63), (7, 256), (3, 264), (33, 512), (4, 519),
                                 (2, 1000), (9, 2048), (6, 2531), (3, 4096), (2, 8191), (3, 8192),
                                 (2, 8200), (1, 16383), (2, 16384), (3100, 128), (1700, 777),
                                 (900, 2048)])
def test_backward(T, H, dtype):
    g = _gen(T * 37 + H)
    h, dy, dh = (_rand(T, H, g, dtype, s) for s in (1.0, 1e-3, 1e-3))
    mask = (torch.rand(T, generator=g, device=DEV) > 0.3).to(torch.uint8)
    for w in ((1 + 0.2 * torch.randn(H, generator=g, device=DEV)).to(d) for d in (BF, F32)):
        for d, m in ((dh, mask), (None, None), (None, mask)):
            out = binding.cis_rmsnorm_bwd(dy, h, w, dh=d, eps=1e-6, mask=m)
            _check_bwd(out, dy, h, w, d, m, 1e-6, dtype)


def _masks(T, g):
    """Rows masked at random, with three quarters of them masked one after another, and none."""
    mask = (torch.rand(T, generator=g, device=DEV) > 0.3).to(torch.uint8)
    block = mask.clone()
    block[T // 8:T // 8 + 3 * T // 4] = 0
    return mask, block, None


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H", [(110000, 128), (30000, 259), (30000, 520), (28000, 2048),
                                 (14000, 2531), (14000, 4096), (7000, 8192), (7000, 16384),
                                 (7000, 8207)])
def test_forward_many_rows(T, H, dtype):
    """Some 10 rows or more for each group of threads that is there at a time (152 SMs, 2048 threads each)."""
    g = _gen(T + H)
    x, r = _rand(T, H, g, dtype), _rand(T, H, g, dtype, 0.7)
    w = 1 + 0.2 * torch.randn(H, generator=g, device=DEV)
    for m in _masks(T, g):
        out = binding.cis_rmsnorm_fwd(x, w, residual=r, mask=m, want_q=True)
        _check_fwd(out, x, w, r, m, 1e-6, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H", [(30000, 128), (30000, 512), (30000, 511), (8000, 777), (8000, 1024),
                                 (8000, 2048), (4000, 4096), (4000, 2531), (2000, 8192),
                                 (2000, 16384), (2000, 16383)])
def test_backward_many_rows(T, H, dtype):
    """Some 12 rows for each group of threads that is there at a time (152 SMs, 512 threads each): the
    rows copied ahead come round, in each number of stages, and rows from the ninth on have their
    mask read later; a block of masked rows is longer than what is known of the mask ahead."""
    g = _gen(T + H)
    h, dy, dh = (_rand(T, H, g, dtype, s) for s in (1.0, 1e-3, 1e-3))
    w = 1 + 0.2 * torch.randn(H, generator=g, device=DEV)
    for m in _masks(T, g):
        for d in (dh, None):
            out = binding.cis_rmsnorm_bwd(dy, h, w, dh=d, mask=m)
            _check_bwd(out, dy, h, w, d, m, 1e-6, dtype)
            again = binding.cis_rmsnorm_bwd(dy, h, w, dh=d, mask=m)
            assert torch.equal(out["dx"], again["dx"])
            assert torch.equal(out["dweight"], again["dweight"])


def test_backward_against_differences():
    """Along random directions, of the forward call's formula in 64 bits."""
    g = _gen(5)
    T, H, eps, step = 6, 96, 1e-6, 1e-5
    h, dy, dh = (_rand(T, H, g, F32) for _ in range(3))
    w = 1 + 0.2 * torch.randn(H, generator=g, device=DEV)

    def value(x, v):
        y = x * torch.rsqrt(x.pow(2).mean(1, keepdim=True) + eps) * v
        return (dy.double() * y).sum() + (dh.double() * x).sum()

    out = binding.cis_rmsnorm_bwd(dy, h, w, dh=dh, eps=eps)
    x, v = h.double(), w.double()
    for _ in range(5):
        a = torch.randn(T, H, generator=g, device=DEV, dtype=torch.float64)
        b = torch.randn(H, generator=g, device=DEV, dtype=torch.float64)
        num = (value(x + step * a, v) - value(x - step * a, v)) / (2 * step)
        size = (out["dx"].double() * a).abs().sum()
        assert abs(float(num - (out["dx"].double() * a).sum())) <= 1e-6 * float(size)
        num = (value(x, v + step * b) - value(x, v - step * b)) / (2 * step)
        size = (out["dweight"].double() * b).abs().sum()
        assert abs(float(num - (out["dweight"].double() * b).sum())) <= 1e-6 * float(size)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pad", [1, 8])
def test_strided_rows(dtype, pad):
    """Rows of a wider tensor: their stride, odd or not, is the call's; what lies between is NaN."""
    T, H = 19, 1024
    g = _gen(pad)
    x, r, dy = (_rand(T, H, g, dtype, pad=p) for p in (pad, 2 * pad, 3 * pad))
    w = 1 + 0.2 * torch.randn(H, generator=g, device=DEV)
    _check_fwd(binding.cis_rmsnorm_fwd(x, w, residual=r, want_q=True), x, w, r, None, 1e-6, dtype)
    _check_bwd(binding.cis_rmsnorm_bwd(dy, x, w, dh=r), dy, x, w, r, None, 1e-6, dtype)


def test_rows_far_apart():
    """A row stride whose offsets pass 2^31 elements."""
    T, H, ld = 3, 700, 1_300_000_001
    g = _gen(4)
    x = torch.empty(T * ld, dtype=BF, device=DEV).view(T, ld)[:, :H]
    x.copy_(_rand(T, H, g, BF))
    w = torch.randn(H, generator=g, device=DEV)
    got, near = binding.cis_rmsnorm_fwd(x, w, residual=x), x.contiguous()
    assert torch.equal(got["y"], binding.cis_rmsnorm_fwd(near, w, residual=near)["y"])
    got = binding.cis_rmsnorm_bwd(x, x, w, dh=x)
    want = binding.cis_rmsnorm_bwd(near, near, w, dh=near)
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])


def test_unaligned_base():
    """A row tensor that starts off 16 bytes, and weights too."""
    T, H = 5, 512
    g = _gen(3)
    flat = torch.randn(T * H + 1, generator=g, device=DEV).to(BF)[1:].view(T, H)
    w = torch.randn(H + 1, generator=g, device=DEV)[1:]
    _check_fwd(binding.cis_rmsnorm_fwd(flat, w, residual=flat, want_q=True), flat, w, flat, None,
               1e-6, BF)
    _check_bwd(binding.cis_rmsnorm_bwd(flat, flat, w), flat, flat, w, None, None, 1e-6, BF)


def test_special_rows():
    """Rows of zeros, of tiny numbers, with NaN or infinity; NaN and infinity behind the mask."""
    H = 300
    x = torch.randn(6, H, generator=_gen(9), device=DEV)
    x[1] = 0.0
    x[2] = 1e-30
    x[3, 7] = float("nan")
    x[4, 7] = float("inf")
    x[5] = float("nan")
    mask = torch.tensor([1, 1, 1, 1, 1, 0], dtype=torch.uint8, device=DEV)
    w = torch.ones(H, device=DEV)
    out = binding.cis_rmsnorm_fwd(x, w, mask=mask, want_q=True)
    assert (out["y"][1] == 0).all() and (out["q"].float()[1] == 0).all()
    assert float(out["scale"][1]) == pytest.approx(2.0 ** -100 / 448, rel=1e-6)
    assert out["y"][2].double().sub(1e-27).abs().max() <= 31 * U * 1e-27 + 0.0
    assert (out["q"].float()[2] == 448).all()
    assert out["y"][3].isnan().all() and out["scale"][3].isnan()
    assert out["q"].float()[3].isnan().all()
    assert out["y"][4, 7].isnan() and out["scale"][4].isnan()
    assert (out["y"][5] == 0).all() and out["scale"][5] == 0 and (out["q"].float()[5] == 0).all()
    got = binding.cis_rmsnorm_bwd(x, x, w, dh=x, mask=mask)
    assert (got["dx"][5] == 0).all() and got["dx"][3].isnan().all()
    got = binding.cis_rmsnorm_bwd(x[[0, 5]], x[[0, 5]], w, mask=mask[[0, 5]])
    assert got["dweight"].isfinite().all()


def test_no_rows():
    w = torch.ones(64, device=DEV)
    x = torch.empty((0, 64), device=DEV)
    out = binding.cis_rmsnorm_fwd(x, w, residual=x, want_q=True)
    assert out["h"].shape == (0, 64) and out["q"].shape == (0, 64) and out["scale"].shape == (0,)
    got = binding.cis_rmsnorm_bwd(x, x, w)
    assert got["dx"].shape == (0, 64) and (got["dweight"] == 0).all()
    mask = torch.zeros(9, dtype=torch.uint8, device=DEV)
    x = torch.full((9, 64), math.nan, device=DEV)
    got = binding.cis_rmsnorm_bwd(x, x, w, mask=mask)
    assert (got["dx"] == 0).all() and (got["dweight"] == 0).all()


def test_graph_replay_and_repeat():
    """Captured on a stream of its own; replays on other inputs equal direct calls, bit for bit."""
    T, H = 700, 1024
    g = _gen(11)
    x, r, dy = (_rand(T, H, g, BF) for _ in range(3))
    w = torch.randn(H, generator=g, device=DEV)
    ws = torch.empty(binding.cis_rmsnorm_bwd_workspace_size(T, H), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        f = binding.cis_rmsnorm_fwd(x, w, residual=r, want_q=True)
        b = binding.cis_rmsnorm_bwd(dy, f["h"], w, dh=dy, workspace=ws)
    for seed in (1, 2):
        for t in (x, r, dy):
            t.copy_(_rand(T, H, _gen(seed), BF))
        graph.replay()
        torch.cuda.synchronize()
        f1 = binding.cis_rmsnorm_fwd(x, w, residual=r, want_q=True)
        b1 = binding.cis_rmsnorm_bwd(dy, f1["h"], w, dh=dy)
        for k in f:
            assert torch.equal(f[k].view(torch.uint8), f1[k].view(torch.uint8))
        for k in b:
            assert torch.equal(b[k].view(torch.uint8), b1[k].view(torch.uint8))


@pytest.mark.parametrize("H", [64, 513, 2048])
def test_guard_bands(H):
    """The C calls write their outputs and nothing else, the workspace's end too."""
    T, pad = 37, 64
    g = _gen(H)
    x, r = _rand(T, H, g, BF), _rand(T, H, g, BF)
    w = torch.randn(H, generator=g, device=DEV)

    def buf(n, dtype):
        b = torch.full((n + 2 * pad,), 0x5A, dtype=torch.uint8, device=DEV) if \
            dtype == torch.uint8 else torch.full((n + 2 * pad,), 7.0, device=DEV).to(dtype)
        return b, b[pad:pad + n]

    def clean(b, n):
        return torch.equal(b[:pad], b.new_full((pad,), b[0].item())) and \
            torch.equal(b[pad + n:], b.new_full((pad,), b[0].item()))

    L, p = binding.lib(), binding._ptr
    bufs = {k: (buf(n, d), n) for k, n, d in (("h", T * H, BF), ("y", T * H, BF),
                                              ("q", T * H, torch.uint8), ("s", T, F32),
                                              ("dx", T * H, BF), ("dw", H, F32))}
    v = {k: b[0][1] for k, b in bufs.items()}
    s = binding._stream()
    assert L.cis_rmsnorm_fwd(p(x), 1, T, H, H, p(r), H, p(w), 0, 1e-6, None, p(v["h"]), p(v["y"]),
                             p(v["q"]), p(v["s"]), s) == 0
    n = binding.cis_rmsnorm_bwd_workspace_size(T, H)
    ws = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    assert L.cis_rmsnorm_bwd(p(x), p(r), 1, T, H, H, H, p(w), 0, None, 0, 1e-6, None, p(v["dx"]),
                             p(v["dw"]), p(ws), n, s) == 0
    torch.cuda.synchronize()
    assert (ws[n:] == 0x5A).all()
    for (whole, _), n in bufs.values():
        assert clean(whole, n)
    want = binding.cis_rmsnorm_fwd(x, w, residual=r, want_q=True)
    assert torch.equal(v["h"].view(T, H), want["h"]) and torch.equal(v["y"].view(T, H), want["y"])
    assert torch.equal(v["q"], want["q"].view(torch.uint8).flatten())
    assert torch.equal(v["s"], want["scale"])


def test_refusals():
    x, w = torch.randn(4, 64, device=DEV), torch.ones(64, device=DEV)
    fwd, bwd = binding.cis_rmsnorm_fwd, binding.cis_rmsnorm_bwd
    for bad in (lambda: fwd(x.half(), w), lambda: fwd(x, w.double()),
                lambda: fwd(x.double(), w)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: fwd(x.t(), w), lambda: fwd(x, w[:63]), lambda: fwd(x[0], w),
                lambda: fwd(x, w, residual=x.bfloat16()), lambda: fwd(x, w, residual=x[:3]),
                lambda: fwd(x, w, mask=torch.ones(4, device=DEV)),
                lambda: fwd(x, w, want_y=False), lambda: fwd(x.cpu(), w), lambda: fwd(x, w.cpu()),
                lambda: bwd(x[:3], x, w), lambda: bwd(x, x, w, dh=x.bfloat16()),
                lambda: bwd(x, x, w, mask=torch.ones(3, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fwd(x, w, eps=0.0), lambda: fwd(x, w, eps=2.0),
                lambda: bwd(x, x, w, eps=math.nan),
                lambda: fwd(torch.empty(1, 16385, device=DEV), torch.ones(16385, device=DEV))):
        with pytest.raises(binding.CisError):
            bad()
