"""cis_lmhead_logits against its formula in 64 bits.

Products of two e4m3 numbers are exact in fp32.  The tensor cores' fp32 sum of H of them is taken
to be off by no more than one rounding, 2^-23 (they cut off rather than round) of the sum of the
products' sizes, for each of the H / 32 steps and 3 more inside a step: (H / 32 + 3) 2^-23 of it.  The
scales add 2 roundings, and the result's type half a step.
"""
import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
E4 = torch.float8_e4m3fn
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _rows(T, H, g):
    x = torch.randn((T, H), generator=g, device=DEV)
    x[:, ::29] *= 9.0
    s = x.abs().amax(1) / 448
    return (x / s[:, None]).to(E4), s


def _check(z, x, xs, w, ws):
    dtype, H = z.dtype, x.shape[1]
    a, b = x.double(), w.double()
    sc = xs.double()[:, None] * ws.double()[None]
    want, size = (a @ b.t()) * sc, (a.abs() @ b.abs().t()) * sc
    tol = (H / 32 + 3) * 2.0 ** -23 * size + (torch.finfo(dtype).eps / 2 + 2.0 ** -23) * want.abs()
    # (a result below the accumulator's error keeps at most that error)
    assert ((z.double() - want).abs() <= tol * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H,V", [
    (1, 16, 1), (1, 128, 127), (2, 144, 128), (3, 2048, 1000), (15, 512, 129), (16, 256, 256),
    (17, 1040, 2049), (31, 128, 640), (33, 384, 513), (64, 2048, 4100), (65, 640, 1001),
    (128, 256, 384), (129, 272, 1026), (200, 512, 999), (255, 128, 130), (256, 1024, 2048),
    (257, 256, 515), (320, 2048, 3001), (333, 128, 770), (512, 256, 777), (513, 144, 300),
    (1000, 128, 1111), (2048, 256, 1025), (1, 8192, 2000), (40, 8176, 20005)])
def test_logits(T, H, V, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + H + V)
    x, xs = _rows(T, H, g)
    w, ws = _rows(V, H, g)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    z = binding.cis_lmhead_logits(x, xs, w, ws, logits_dtype=dtype, dev_status=st)
    assert z.shape == (T, V) and z.dtype == dtype and int(st) == 0
    _check(z, x, xs, w, ws)
    z2 = binding.cis_lmhead_logits(x, xs, w, ws, logits_dtype=dtype)
    assert torch.equal(z, z2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H,V", [
    (3, 128, 60001), (64, 272, 60000), (65, 144, 60001), (192, 128, 60003), (256, 384, 60000),
    (257, 128, 60002), (320, 128, 60000), (320, 1040, 60001), (600, 128, 50003), (2048, 128, 20003)])
def test_several_tiles_a_cta(T, H, V, dtype):
    """3 tiles or more for each of up to 152 CTAs or 76 pairs: the accumulators and the ring come round, the
    third accumulator too (257 to 320 tokens), with several token tiles for a vocabulary tile
    (above 320)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T + H + V)
    x, xs = _rows(T, H, g)
    w, ws = _rows(V, H, g)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    z = binding.cis_lmhead_logits(x, xs, w, ws, logits_dtype=dtype, dev_status=st)
    _check(z, x, xs, w, ws)
    for _ in range(4):
        again = binding.cis_lmhead_logits(x, xs, w, ws, logits_dtype=dtype, dev_status=st)
        assert torch.equal(z, again)
    assert int(st) == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,ld,off", [(5, 300, 301, 1), (37, 254, 256, 0), (37, 255, 257, 3),
                                        (300, 512, 520, 8), (20, 128, 128, 1)])
def test_rows_of_a_wider_buffer(T, V, ld, off, dtype):
    """Rows that are not aligned; what lies between and around them stays as it was."""
    H = 192
    g = torch.Generator(device=DEV)
    g.manual_seed(T + V)
    x, xs = _rows(T, H, g)
    w, ws = _rows(V, H, g)
    flat = torch.full((off + T * ld + 64,), 7.0, dtype=dtype, device=DEV)
    out = flat[off:off + T * ld].view(T, ld)
    z = binding.cis_lmhead_logits(x, xs, w, ws, logits=out)
    assert z.data_ptr() == out.data_ptr()
    _check(out[:, :V], x, xs, w, ws)
    assert (out[:, V:] == 7).all() and (flat[:off] == 7).all() and (flat[off + T * ld:] == 7).all()


@pytest.mark.parametrize("T", [3, 70])
def test_rows_far_apart(T):
    """A row stride whose offsets pass 2^31 elements."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    x, xs = _rows(T, 128, g)
    w, ws = _rows(300, 128, g)
    ld = 2_500_000_001 // (T - 1) + 1
    out = torch.empty(T * ld, dtype=BF, device=DEV).view(T, ld)
    binding.cis_lmhead_logits(x, xs, w, ws, logits=out)
    assert torch.equal(out[:, :300], binding.cis_lmhead_logits(x, xs, w, ws))


def test_special_values():
    """A NaN spoils its row or column alone; zero scales give zeros; 448s add up exactly."""
    T, H, V = 20, 512, 300
    x, w = torch.full((T, H), 448.0, device=DEV).to(E4), torch.full((V, H), 448.0, device=DEV).to(E4)
    xs, ws = torch.ones(T, device=DEV), torch.ones(V, device=DEV)
    xs[3], ws[5] = 0.0, 2.0
    x.view(torch.uint8)[7, 100] = 0x7F
    w.view(torch.uint8)[9, 200] = 0xFF
    z = binding.cis_lmhead_logits(x, xs, w, ws, logits_dtype=F32)
    nan = torch.zeros(T, V, dtype=torch.bool, device=DEV)
    nan[7], nan[:, 9] = True, True
    assert torch.equal(z.isnan(), nan)
    want = (448.0 * 448 * H) * xs[:, None] * ws[None]
    assert torch.equal(z[~nan], want[~nan])


def test_no_rows():
    w, ws = _rows(64, 128, torch.Generator(device=DEV))
    z = binding.cis_lmhead_logits(w[:0], ws[:0], w, ws)
    assert z.shape == (0, 64)


def test_captured_on_its_own_stream():
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, xs = _rows(24, 512, g)
    w, ws = _rows(3000, 512, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        z = binding.cis_lmhead_logits(x, xs, w, ws)
    for _ in range(2):
        a, b = _rows(24, 512, g)
        x.copy_(a)
        xs.copy_(b)
        graph.replay()
        assert torch.equal(z, binding.cis_lmhead_logits(x, xs, w, ws))
    torch.cuda.synchronize()


def test_two_streams_at_once():
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    w, ws = _rows(5000, 256, g)
    xs = [_rows(T, 256, g) for T in (1, 90)]
    want = [binding.cis_lmhead_logits(*x, w, ws) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(binding.cis_lmhead_logits(*xs[i], w, ws))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(z, want[i]) for z in got[i])


def test_norm_then_logits():
    """The 8-bit norm's rows as they are: z stands for y W^T to the two roundings to 8 bits."""
    T, H, V = 33, 1024, 2000
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    x, r = (torch.randn((T, H), generator=g, device=DEV).to(BF) for _ in range(2))
    weight = torch.ones(H, device=DEV)
    w, ws = _rows(V, H, g)
    n = binding.cis_rmsnorm_fwd(x, weight, residual=r, want_y=False, want_q=True)
    z = binding.cis_lmhead_logits(n["q"], n["scale"], w, ws, logits_dtype=F32)
    _check(z, n["q"], n["scale"], w, ws)
    y = binding.cis_rmsnorm_fwd(x, weight, residual=r)["y"].double()
    W = w.double() * ws.double()[:, None]
    # each entry of q is off by half a step: 2^-4 of itself, or 2^-10 of the row's scale
    off = 2.0 ** -4 * y.abs() + 2.0 ** -10 * n["scale"].double()[:, None]
    tol = off @ W.abs().t() + 2.0 ** -8 * (y.abs() @ W.abs().t())
    assert ((z.double() - y @ W.t()).abs() <= tol).all()


def test_refusals():
    g = torch.Generator(device=DEV)
    x, xs = _rows(4, 64, g)
    w, ws = _rows(9, 64, g)
    f = binding.cis_lmhead_logits
    for bad in (lambda: f(x.float(), xs, w, ws), lambda: f(x, xs[:3], w, ws),
                lambda: f(x, xs, w[:, :48], ws), lambda: f(x[:, :48].contiguous(), xs, w, ws),
                lambda: f(x, xs, w, ws.double()), lambda: f(x.cpu(), xs, w, ws),
                lambda: f(x, xs, w, ws, logits=torch.empty(4, 8, device=DEV)),
                lambda: f(x, xs, w, ws, dev_status=torch.zeros(1, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        f(x, xs, w, ws, logits_dtype=torch.float16)
    y, ys = _rows(4, 72, g)
    with pytest.raises(binding.CisError):
        f(y, ys, y, ys)
