"""Calls of several sizes from several threads at once, each on a stream of its own: a kernel's
shared memory is granted for its largest call, so that none takes another's away.  The calls go
to the C entry points, with arguments made beforehand, to be in the library most of the time."""
import ctypes
import threading

import pytest
import torch

from paper_2609_32444_gb300 import binding

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]

DEV = torch.device("cuda")
BF16 = 1


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_32444_gb300 import build
    build.build()
    binding.lib()


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


class _Call:
    """One entry point's call on a stream: the tensors it takes, its outputs, its arguments."""

    def __init__(self, V, stream, T=2):
        g = torch.Generator(device=DEV)
        g.manual_seed(V)
        self.T, self.V = T, V
        self.z = (torch.randn((T, V), generator=g, device=DEV) * 3).to(torch.bfloat16)
        self.f = torch.full((T,), 0.5, device=DEV)
        self.ids = torch.zeros((T, 256), dtype=torch.int32, device=DEV)
        self.lp = torch.zeros((T, 256), device=DEV)
        self.stream = ctypes.c_void_p(stream.cuda_stream)
        self.fn, self.args, self.out = self.make()

    def __call__(self):
        return self.fn(*self.args)


class _Sample(_Call):
    def make(self):
        return (binding.lib().cis_sample_tokens,
                (_ptr(self.z), BF16, self.T, self.V, self.V, _ptr(self.f), None, None,
                 _ptr(self.f), None, None, _ptr(self.ids), _ptr(self.lp), None, None, self.stream),
                (self.ids, self.lp))


class _Topk(_Call):
    def make(self):
        K = 256 if self.V > 6000 else 3
        return (binding.lib().cis_topk_logprobs,
                (_ptr(self.z), BF16, self.T, self.V, self.V, K, ctypes.c_double(1.0), None,
                 _ptr(self.ids), _ptr(self.lp), None, None, self.stream), (self.ids, self.lp))


class _Distill(_Call):
    def make(self):
        self.P = binding.cis_distill_default_params()
        ids, lp, _ = binding.cis_topk_logprobs(self.z, 8)
        self.ids[:, :8], self.lp[:, :8] = ids, lp
        self.dz = torch.zeros((self.T, self.V), dtype=torch.bfloat16, device=DEV)
        n = binding.cis_distill_workspace_size(self.T)
        self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        return (binding.lib().cis_distill_fwd_bwd,
                (_ptr(self.z), BF16, self.T, self.V, self.V, _ptr(self.ids), _ptr(self.lp), 8, 256,
                 None, None, None, 0, ctypes.byref(self.P), _ptr(self.dz), BF16, self.V, None, None,
                 _ptr(self.ws), n, self.stream), (self.dz,))


class _Loss(_Call):
    def make(self):
        L, T, V = binding.lib(), self.T, self.V
        self.P = binding.cis_default_params("cis")
        self.dz = torch.zeros((T, V), dtype=torch.bfloat16, device=DEV)
        self.tok = torch.ones(T, dtype=torch.int32, device=DEV)
        n = binding.cis_loss_workspace_size(T, V)
        self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        return (L.cis_loss_fwd_bwd,
                (_ptr(self.z), BF16, T, V, V, _ptr(self.tok), _ptr(self.f), None, _ptr(self.f), None,
                 None, 0, ctypes.byref(self.P), _ptr(self.dz), BF16, V, None, None, None, None, None,
                 None, _ptr(self.ws), n, self.stream), (self.dz,))


class _Bins(_Call):
    def make(self):
        n = 40 if self.V > 2000 else 3
        edges = (ctypes.c_double * (n + 1))(*[-10 + 20 * i / n for i in range(n + 1)])
        self.key = self.z.float().view(-1)
        values = (ctypes.c_void_p * 1)(self.key.data_ptr())
        need = ctypes.c_size_t(0)
        L, N = binding.lib(), self.key.numel()
        assert L.cis_binned_sums_workspace_size(N, n, 1, ctypes.byref(need)) == 0
        self.ws = torch.zeros(need.value, dtype=torch.uint8, device=DEV)
        counts = torch.zeros(n, dtype=torch.int64, device=DEV)
        sums = torch.zeros(n, dtype=torch.float64, device=DEV)
        return (L.cis_binned_sums,
                (_ptr(self.key), None, N, edges, n, values, 1, _ptr(counts), _ptr(sums),
                 _ptr(self.ws), need.value, self.stream), (counts, sums))


# the same kernel in both sizes
@pytest.mark.parametrize("kind,small,large", [(_Sample, 5000, 32000), (_Topk, 5000, 7000),
                                              (_Distill, 1000, 16000), (_Loss, 1000, 16000),
                                              (_Bins, 2000, 4000)])
def test_sizes_at_once(kind, small, large):
    n = 6
    streams = [torch.cuda.Stream() for _ in range(n)]
    # (sampling: rows enough for one CTA each, whose shared memory goes by the row's length)
    calls = [kind(large if i % 2 else small, s, 320 if kind is _Sample and i % 2 else 2)
             for i, s in enumerate(streams)]
    torch.cuda.synchronize()
    for c in calls:
        assert c() == 0
    torch.cuda.synchronize()
    want = [[x.clone() for x in c.out] for c in calls]
    codes, gate = [set() for _ in calls], threading.Barrier(n)

    def run(i):
        call, seen = calls[i], codes[i]
        gate.wait()
        for _ in range(3000):
            seen.add(call())

    threads = [threading.Thread(target=run, args=(i,)) for i in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert codes == [{0}] * n
    for c, w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(c.out, w))
