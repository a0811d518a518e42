"""cis_sample_tokens where a decision is close: numbers a few steps of fp32 to either side of an
entry's running mass, nuclei that end a few steps from top_p, the same rows in calls of any size.

The masses that decide are right to 2^-34 of each, so a number farther than 2^-32 of the row's
mass from every border has one answer, whatever the path and the number of CTAs a row.  The
inputs are chosen by their distance in 64 bits; those within 2^-32 are given another number.
"""
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


def _near(x, g, lo=0.0, hi=1.0):
    """Numbers at x (fp64, in (0, 1)), each moved by 2^-24 to 2^-15 to either side, as fp32."""
    d = 2.0 ** -(15 + 9 * torch.rand(x.shape, generator=g, device=DEV, dtype=torch.float64))
    up = torch.rand(x.shape, generator=g, device=DEV) < 0.5
    return (x + torch.where(up, d, -d)).clamp(lo, hi).float()


def _rows(n, V, dtype, width, g, tilt=0.0):
    x = torch.randn((n, V), generator=g, device=DEV) * width
    return (x - tilt * torch.arange(V, device=DEV) / V).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,width,tilt", [(151936, 1.0, 0.0), (151936, 2.5, 0.0),
                                          (32003, 2.5, 0.0), (32003, 0.2, 12.0),
                                          (2001, 1.0, 0.0), (300, 2.0, 0.0)])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_draws_next_to_an_entrys_running_mass(dtype, V, width, tilt, tau):
    """Nothing cut off: u over [0, 1), and as many in its last and its first parts, near the
    running masses of entries that are taken in proportion to their mass."""
    n, each = 8, 256
    g = _gen(V + int(10 * width))
    base = _rows(n, V, dtype, width, g, tilt)
    t = torch.full((n * each,), tau, device=DEV)
    x = base.double() / float(t[0])  # (the temperature is fp32)
    c = torch.cumsum(torch.exp(x - x.amax(1, keepdim=True)), 1)
    c = (c / c[:, -1:]).contiguous()
    r = torch.rand((n, each), generator=g, device=DEV, dtype=torch.float64)
    part = torch.arange(each, device=DEV) % 4
    r = torch.where(part == 1, 1 - 0.05 * r, torch.where(part == 2, 0.05 * r, r))
    r = torch.where(part == 3, 1 - 2.0 ** -10 * r, r)
    at = torch.searchsorted(c, r).clamp(max=V - 1)
    u = _near(c.gather(1, at), g, 0.0, 1 - 2.0 ** -24)

    def token(u):
        v = u.double()
        j = torch.searchsorted(c, v, right=True).clamp(max=V - 1)
        below = torch.where(j > 0, c.gather(1, (j - 1).clamp(min=0)), -1.0)
        return j, torch.minimum(c.gather(1, j) - v, v - below)

    for _ in range(20):
        want, gap = token(u)
        u = torch.where(gap <= 2.0 ** -32, torch.rand((n, each), generator=g, device=DEV) * 0.99, u)
    want, gap = token(u)
    assert float(gap.min()) > 2.0 ** -32  # of the inputs alone
    z = base.repeat_interleave(each, 0)
    u, want = u.view(-1), want.view(-1)
    for T in (n * each, 700, 256, 24, 1):
        for a in range(0, min(n * each, 40 * T), T):
            s = slice(a, a + T)
            ids = binding.cis_sample_tokens(z[s], u[s], temperature=None if tau == 1.0 else t[s])[0]
            off = (ids != want[s]).nonzero().view(-1)
            assert off.numel() == 0, (T, off.numel(), u[s][off][:4].tolist(),
                                      gap.view(-1)[s][off][:4].tolist())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,width", [(151936, 2.5), (32003, 3.0), (5003, 3.0)])
def test_nuclei_that_end_next_to_top_p(dtype, V, width):
    """top_p within 2^-24 to 2^-15 of the mass of a prefix.  The rows rise, so that u = 0 samples
    the last kept entry, whose log-probability tells the kept mass."""
    n, each = 8, 128
    g = _gen(V)
    base = torch.sort(_rows(n, V, torch.float32, width, g), dim=1)[0]  # the largest come last
    base += torch.linspace(0, 1e-3, V, device=DEV)
    base = base.to(dtype)
    x = base.double()
    w = torch.exp(x - x[:, -1:]).flip(1)
    c = torch.cumsum(w, 1)  # mass of the k + 1 largest
    # (equal entries are taken by index: an order of values alone has the same masses)
    share = (c / c[:, -1:]).contiguous()
    k = torch.randint(2, 200, (n, each), generator=g, device=DEV)
    p = _near(share.gather(1, k), g, 1e-6, 1 - 2.0 ** -24)

    def kept(p):
        v = p.double()
        m = torch.searchsorted(share, v)  # the first place whose mass is at least p
        below = torch.where(m > 0, share.gather(1, (m - 1).clamp(min=0)), -1.0)
        return m + 1, torch.minimum(share.gather(1, m) - v, v - below)

    for _ in range(20):
        m, gap = kept(p)
        p = torch.where(gap <= 2.0 ** -32, 0.1 + 0.3 * torch.rand((n, each), generator=g, device=DEV),
                        p)
    m, gap = kept(p)
    assert float(gap.min()) > 2.0 ** -32
    z = base.repeat_interleave(each, 0)
    u = torch.zeros(n * each, device=DEV)  # the first by index: the last of the order's values
    _, _, lps = binding.cis_sample_tokens(z, u, top_p=p.view(-1), want_lp_sampled=True)
    # its log-probability tells the kept mass, whose neighbours differ by far more than fp32's
    # step: the k-th of at most 200 entries has over 2^-14 of it (asserted)
    row = torch.arange(n, device=DEV).repeat_interleave(each)
    mm = m.view(-1)
    mass = c[row, mm - 1]
    assert float((w[row, mm - 1] / mass).min()) > 2.0 ** -14
    assert float((w[row, mm] / mass).min()) > 2.0 ** -14
    want = (w[row, mm - 1] / mass).log()
    off = ((lps.double() - want).abs() > 2.0 ** -19).nonzero().view(-1)
    assert off.numel() == 0, (off.numel(), gap.view(-1)[off][:4].tolist())
