"""Sampling, a teacher's lists and the two losses run together, as a step of on-policy
distillation does; the calls' native part against the Python one; what the binding refuses;
guard bands around every output."""
import contextlib
import ctypes
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


class _Python:
    def __getattr__(self, name):
        return lambda *a: None


@contextlib.contextmanager
def _python_only():
    kept = binding._native
    binding._native = _Python()
    try:
        yield
    finally:
        binding._native = kept


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def test_a_step_of_on_policy_distillation():
    """Tokens and their log-probabilities from the student's logits; the policy pass takes them
    as they are (on policy: weight 1, no truncation); the teacher's lists; the student towards
    them.  A logit step against the gradient lowers the divergence by |gradient|^2 times the
    step, to second order: L's curvature along it is at most (1 + max |l|) / T."""
    T, V, K = 96, 5003, 40
    g = _gen(1)
    student = (torch.randn((T, V), generator=g, device=DEV) * 2.5).to(torch.bfloat16)
    teacher = (student.float() + 0.7 * torch.randn((T, V), generator=g, device=DEV)).to(torch.bfloat16)
    mask = (torch.rand(T, generator=g, device=DEV) > 0.2).to(torch.uint8)
    u = torch.rand(T, generator=g, device=DEV)
    ids, lp, lps = binding.cis_sample_tokens(student, u, mask=mask, want_lp_sampled=True)
    on = mask != 0
    assert bool((ids[on] >= 0).all()) and bool((ids[~on] == -1).all())
    assert float((lp - lps)[on].abs().max()) <= 2.0 ** -19  # nothing cut off
    again = binding.cis_token_logprobs(student, ids, mask=mask)
    assert float((again - lp)[on].abs().max()) <= 4e-5
    adv = torch.randn(T, generator=g, device=DEV)
    out = binding.cis_loss_fwd_bwd(student, ids, lp, adv, binding.cis_default_params("cis"),
                                   mask=mask)
    st = binding.decode_stats(out["stats"])
    assert st["status"] == 0 and st["n_truncated"] == 0 and st["max_abs_logk"] <= 4e-5
    tids, tlp, lse = binding.cis_topk_logprobs(teacher, K, mask=mask, want_lse=True)
    for kind in ("forward", "reverse", "topk"):
        P = binding.cis_distill_default_params(kind)
        d = binding.cis_distill_fwd_bwd(student.float(), tids, tlp, P, mask=mask)
        assert binding.device_status(d["workspace"]) == 0
        assert bool((d["kl"][on] > 0).all()) and bool((d["kl"][~on] == 0).all())
        dz = d["dlogits"].double()
        step = 0.01 * T
        after = binding.cis_distill_fwd_bwd((student.double() - step * dz).float(), tids, tlp, P,
                                            mask=mask, want_grad=False)
        gain = float(d["loss"]) - float(after["loss"])
        first = step * float(dz.square().sum())
        worst = float((dz.abs() * on.sum()).max())  # max_j |dL/dz_j| of a row
        curve = 0.5 * step * step * float(dz.square().sum()) * (2 + 4 * worst + 40) / float(on.sum())
        assert abs(gain - first) <= curve + 1e-6 * float(d["loss"]), (kind, gain, first, curve)


def test_teacher_equal_to_student_has_no_gradient():
    """Lists of the student's own log-probabilities: the divergences are 0 but for the lists'
    rounding to fp32 (2^-24 |lp| of each p, squared in L), and the gradients are of that size."""
    T, V = 20, 3001
    z = torch.randn((T, V), generator=_gen(2), device=DEV) * 3
    ids, lp, _ = binding.cis_topk_logprobs(z, 100)
    for kind in ("forward", "reverse"):
        d = binding.cis_distill_fwd_bwd(z, ids, lp, binding.cis_distill_default_params(kind))
        assert float(d["kl"].abs().max()) <= 1e-10
        assert float((d["dlogits"] * T).abs().max()) <= 4e-6


def _cases():
    g = _gen(3)
    T, V, K = 50, 777, 9
    z = torch.randn((T, V), generator=g, device=DEV)
    ids, lp, _ = binding.cis_topk_logprobs(z, K)
    u = torch.rand(T, generator=g, device=DEV)
    return z, ids, lp, u


def _same(a, b):
    if isinstance(a, dict):
        assert list(a) == list(b)
        a = {k: v for k, v in a.items() if k != "workspace"}
        return all(_same(a[k], b[k]) for k in a)
    if isinstance(a, tuple):
        return len(a) == len(b) and all(_same(x, y) for x, y in zip(a, b))
    return (a is None and b is None) or (a.dtype == b.dtype and torch.equal(a, b))


def test_native_and_python_calls_agree():
    z, ids, lp, u = _cases()
    T = z.shape[0]
    m = torch.ones(T, dtype=torch.uint8, device=DEV)
    m[3:9] = 0
    cu = torch.tensor([0, 20, 50], dtype=torch.int32, device=DEV)
    P = binding.cis_distill_default_params("reverse", agg=1)
    f = torch.full((T,), 0.8, device=DEV)
    k = torch.full((T,), 12, dtype=torch.int32, device=DEV)
    wide = torch.zeros((T, 800), device=DEV)
    calls = [
        lambda: binding.cis_sample_tokens(z, u),
        lambda: binding.cis_sample_tokens(z, u, f, k, f, f, m, 700, False, True),
        lambda: binding.cis_topk_logprobs(z, 5),
        lambda: binding.cis_topk_logprobs(z, 5, 0.5, m, 600, True),
        lambda: binding.cis_topk_logprobs(z, 5, 2),  # (a whole number for the temperature)
        lambda: binding.cis_distill_fwd_bwd(z, ids, lp, P, f, m, cu),
        lambda: binding.cis_distill_fwd_bwd(z, ids, lp, binding.cis_distill_default_params(),
                                            dlogits_dtype=torch.bfloat16),
        lambda: {k: v.clone() if v is not None else v for k, v in binding.cis_distill_fwd_bwd(
            z, ids[:, :4], lp[:, :4], P, cu_seqlens=cu, dlogits=wide.zero_()[:, 1:778],
            want_grad=False).items()}]
    for i, call in enumerate(calls):
        a = call()
        with _python_only():
            b = call()
        assert _same(a, b), i


def test_binding_refuses():
    """Wrong kinds, types, shapes and strides: the same error from both parts."""
    z, ids, lp, u = _cases()
    P = binding.cis_distill_default_params()
    sample, topk, distill = (binding.cis_sample_tokens, binding.cis_topk_logprobs,
                             binding.cis_distill_fwd_bwd)
    k = torch.ones(50, dtype=torch.int32, device=DEV)
    calls = [
        lambda: sample(z.half(), u), lambda: sample(z, u[:-1]), lambda: sample(z, u.double()),
        lambda: sample(z.t(), u), lambda: sample(z, u.cpu()), lambda: sample(z, u, top_k=u),
        lambda: sample(z, u, temperature=k), lambda: sample(z, u, V=778),
        lambda: sample(z, u, V=0), lambda: sample(z, u, mask=u), lambda: sample(z[0], u),
        lambda: sample(z, u, dev_status=k.byte()), lambda: sample(z, u, dev_status=k[:0]),
        lambda: topk(z, 3, dev_status=u), lambda: topk(z, 2.5),
        lambda: distill(z, ids, lp, P, workspace=torch.zeros(
            1, dtype=torch.uint8, device=DEV).expand(1 << 20)),
        lambda: topk(z, 0), lambda: topk(z, 257), lambda: topk(z, 3, 0.0),
        lambda: topk(z, 3, math.nan), lambda: topk(z, 3, V=1000), lambda: topk(z.int(), 3),
        lambda: distill(z, ids.long(), lp, P), lambda: distill(z, ids, lp.double(), P),
        lambda: distill(z, ids[:-1], lp, P), lambda: distill(z, ids, lp[:, :-1], P),
        lambda: distill(z, ids, lp.cpu(), P), lambda: distill(z, ids.t(), lp.t(), P),
        lambda: distill(z, ids, lp, P, V=900), lambda: distill(z, ids, lp, P, u[:-1]),
        lambda: distill(z, ids, lp, P, dlogits=z), lambda: distill(z, ids[:, :0], lp[:, :0], P),
        lambda: distill(z, ids, lp, P, dlogits_dtype=torch.float16),
        lambda: distill(z, ids, lp, P, dlogits=torch.empty((50, 8), device=DEV)),
        lambda: distill(z, ids, lp, binding.cis_default_params("cis")),
        lambda: distill(z, ids, lp, binding.cis_distill_default_params(agg=1)),
        lambda: distill(z, ids, lp, P, cu_seqlens=u)]
    for i, f in enumerate(calls):
        errors = []
        for python in (False, True):
            with _python_only() if python else contextlib.nullcontext():
                with pytest.raises(Exception) as e:
                    f()
                errors.append((type(e.value), str(e.value)))
        assert errors[0] == errors[1], (i, errors)


class _Guarded:
    """nbytes of device memory with 4096 known bytes on either side."""

    def __init__(self, nbytes):
        self.n = nbytes
        self.buf = torch.full((nbytes + 8192 + 1024,), 0xA5, dtype=torch.uint8, device=DEV)
        self.at = 4096 + (-(self.buf.data_ptr() + 4096)) % 1024
        self.ptr = ctypes.c_void_p(self.buf.data_ptr() + self.at)

    def ok(self):
        b = self.buf.cpu()
        return bool((b[:self.at] == 0xA5).all()) and bool((b[self.at + self.n:] == 0xA5).all())


@pytest.mark.parametrize("T,V,K", [(3, 1, 1), (5, 33, 40), (70, 1001, 7), (9, 20003, 256),
                                   (2, 151936, 64)])
@pytest.mark.parametrize("bf16", [True, False])
def test_calls_write_only_their_outputs(T, V, K, bf16):
    g = _gen(T)
    z = (torch.randn((T, V), generator=g, device=DEV) * 3).to(torch.bfloat16 if bf16 else
                                                              torch.float32)
    u = torch.rand(T, generator=g, device=DEV)
    p = torch.full((T,), 0.95, device=DEV)
    L, code = binding.lib(), int(bf16)
    P = ctypes.c_void_p
    s = P(torch.cuda.current_stream().cuda_stream)
    ptr = lambda t: P(t.data_ptr())  # noqa: E731
    out = [_Guarded(4 * T) for _ in range(4)]
    assert L.cis_sample_tokens(ptr(z), code, T, V, V, ptr(u), None, None, ptr(p), None, None,
                               out[0].ptr, out[1].ptr, out[2].ptr, out[3].ptr, s) == 0
    assert all(x.ok() for x in out)
    lists = [_Guarded(4 * T * K), _Guarded(4 * T * K), _Guarded(4 * T)]
    assert L.cis_topk_logprobs(ptr(z), code, T, V, V, K, 1.0, None, lists[0].ptr, lists[1].ptr,
                               lists[2].ptr, None, s) == 0
    assert all(x.ok() for x in lists)
    params = binding.cis_distill_default_params()
    n = binding.cis_distill_workspace_size(T)
    for dz_code, size in ((0, 4), (1, 2)):
        d = [_Guarded(T * (V + 3) * size), _Guarded(4 * T), _Guarded(8), _Guarded(n)]
        before = d[0].buf.clone()
        assert L.cis_distill_fwd_bwd(ptr(z), code, T, V, V, lists[0].ptr, lists[1].ptr, K, K,
                                     None, None, None, 0, ctypes.byref(params), d[0].ptr, dz_code,
                                     V + 3, d[1].ptr, d[2].ptr, d[3].ptr, n, s) == 0
        assert all(x.ok() for x in d)
        view = lambda b: b[d[0].at:d[0].at + d[0].n].view(T, (V + 3) * size)  # noqa: E731
        assert torch.equal(view(d[0].buf)[:, V * size:], view(before)[:, V * size:])


def test_two_graphs_and_two_streams_at_once():
    """Calls in flight together share nothing: two captured steps replayed on two streams give
    what the calls alone do."""
    g = _gen(5)
    zs = [(torch.randn((40, 9001), generator=g, device=DEV) * 3).to(torch.bfloat16)
          for _ in range(2)]
    u = torch.rand(40, generator=g, device=DEV)
    p = torch.full((40,), 0.9, device=DEV)
    P = binding.cis_distill_default_params("forward")

    def step(z):
        ids, lp, _ = binding.cis_topk_logprobs(z, 20)
        return (ids, lp) + binding.cis_sample_tokens(z, u, top_p=p, want_lp_sampled=True) + tuple(
            binding.cis_distill_fwd_bwd(z, ids, lp, P)[k] for k in ("dlogits", "kl", "loss"))

    want = [[x.clone() for x in step(z)] for z in zs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for z in zs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(z))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 819200), (torch.float32, 409600),
                                     (torch.bfloat16, (1 << 20) - 3), (torch.float32, 1 << 20)])
def test_longest_rows(dtype, V):
    """The longest rows of each call: tokens against a stable sort, masses against fp64."""
    T, K = 2, 256
    z = (torch.randn((T, V), generator=_gen(V), device=DEV) * 2).to(dtype)
    x = z.double()
    ids, lp, lse = binding.cis_topk_logprobs(z, K, want_lse=True)
    v, at = torch.sort(x, dim=1, descending=True, stable=True)
    e = torch.logsumexp(x, 1)
    assert torch.equal(ids.long(), at[:, :K])
    assert float((lse.double() - e).abs().max()) <= 2.0 ** -18
    assert float((lp.double() - (v[:, :K] - e.view(-1, 1))).abs().max()) <= 2.0 ** -18
    u = torch.tensor([0.25, 0.9], device=DEV)
    for p in (None, torch.full((T,), 0.7, device=DEV)):
        got, glp, glps = binding.cis_sample_tokens(z, u, top_p=p, want_lp_sampled=True)
        w = torch.exp(v - v[:, :1])
        c = w.cumsum(1)
        n = torch.full((T,), V, device=DEV) if p is None else (
            (c < p.double().view(-1, 1) * c[:, -1:]).sum(1) + 1)
        keep = torch.arange(V, device=DEV).view(1, -1) < n.view(-1, 1)
        m = torch.zeros_like(w).scatter_(1, at, w * keep)
        r = m.cumsum(1)
        j = (r <= u.double().view(-1, 1) * r[:, -1:]).sum(1)
        assert torch.equal(got.long(), j)
        zj = x.gather(1, j.view(-1, 1)).view(-1)
        assert float((glp.double() - (zj - e)).abs().max()) <= 2.0 ** -18
        assert float((glps.double() - (zj - v[:, 0] - r[:, -1].log())).abs().max()) <= 2.0 ** -18
    P = binding.cis_distill_default_params("forward")
    if V * T * z.element_size() <= 2 * 819200 * 2:
        d = binding.cis_distill_fwd_bwd(z, ids, lp, P, dlogits_dtype=torch.float32)
        assert float(d["kl"].abs().max()) <= 1e-9  # the row's own lists
        assert float((d["dlogits"] * T).abs().max()) <= 4e-6
    else:
        with pytest.raises(binding.CisError):
            binding.cis_distill_fwd_bwd(z, ids, lp, P)
