"""What the performance of the calls around the LM head's decoding step is measured on.

A rollout engine that proposes several tokens at a time ends each step with three calls: the
final norm with the residual's addition, whose output may be 8 bits wide (cis_rmsnorm_fwd), the
LM head on it (cis_lmhead_logits), and the verification of the proposed tokens against those
logits (cis_verify_tokens).  Training has the same norm before the fused LM head, and its
gradient after it (cis_rmsnorm_bwd).  Sizes are those of the synthetic workloads, the tests and
the benchmark, with odd ones beside them.

Families (a case's "family"):
  norm    h = x + residual and its root-mean-square norm, in bf16 / fp32 or in e4m3 with a
          scale a row.
  back    the norm's gradients, with the gradient that arrives by the residual stream added.
  logits  logits from e4m3 hidden states and weights with a scale a row of each.
  verify  which drafted tokens are kept, the token after them, and their log-probabilities.

Where `own` is false, `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False  # set by whoever measures: true takes the library's calls

DEV = "cuda"
EPS = 1e-6
FLOOR = 2.0 ** -100  # the least largest value that a row's 8-bit scale is made for


def _norm(T, H, dtype="bf16", out="same", residual=True, wide=False, pad=0.0):
    return {"family": "norm", "T": T, "H": H, "dtype": dtype, "out": out, "residual": residual,
            "wide": wide, "pad": pad}


def _back(T, H, dtype="bf16", residual=True, wide=False, pad=0.0):
    return {"family": "back", "T": T, "H": H, "dtype": dtype, "residual": residual, "wide": wide,
            "pad": pad}


def _logits(T, H, V, out="bf16"):
    return {"family": "logits", "T": T, "H": H, "V": V, "out": out}


def _verify(B, D, V, dtype="bf16", draft="model", tau=1.0, ragged=False, mixed=False):
    return {"family": "verify", "B": B, "D": D, "V": V, "dtype": dtype, "draft": draft,
            "tau": tau, "ragged": ragged, "mixed": mixed}


def listed():
    return [
        # one request's decoding step before an 8-bit LM head: the call's own cost
        dict(_norm(1, 2048, out="e4m3"), name="norm_one"),
        # a speculative step of 64 requests with 5 positions each
        dict(_norm(320, 4096, out="e4m3"), name="norm_step"),
        # a training batch before the fused LM head, 40% padding
        dict(_norm(16384, 2048, pad=0.4), name="norm_train"),
        # its gradient, joined with the one of the residual stream
        dict(_back(16384, 2048, pad=0.4), name="back_train"),
        # fp32 rows of no alignment, without a residual stream
        dict(_back(3001, 2531, "f32", residual=False, wide=True), name="back_odd"),
        # one request's token
        dict(_logits(1, 2048, 151936), name="logits_one"),
        # a speculative step of 64 requests with 5 positions each
        dict(_logits(320, 2048, 151936), name="logits_step"),
        # scoring a rollout's tokens on a vocabulary that tokens were added to
        dict(_logits(2048, 2048, 32003, "f32"), name="logits_score"),
        # one request, four tokens from a small model
        dict(_verify(1, 4, 151936, tau=0.6), name="verify_one"),
        # a rollout batch at the model's own distribution
        dict(_verify(64, 4, 151936), name="verify_step"),
        # requests with settings and numbers of drafts of their own, some greedy, some idle
        dict(_verify(128, 8, 32003, "f32", ragged=True, mixed=True), name="verify_mixed"),
        # drafts looked up in the prompt: no distribution of theirs
        dict(_verify(96, 3, 151936, draft="lookup", ragged=True), name="verify_lookup"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.random()
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind < 0.45:
        H = _log_int(rng, 64, 8192)
        H = H if rng.random() < 0.25 else -(-H // 64) * 64  # most hidden sizes are round
        T = _log_int(rng, 1, min(16384, 33554432 // H))
        pad, residual, wide = rng.choice([0.0, 0.25, 0.4]), rng.random() < 0.8, rng.random() < 0.3
        if kind < 0.27:
            return _norm(T, H, dtype, rng.choice(["e4m3", "e4m3", "same"]), residual, wide, pad)
        return _back(T, H, dtype, residual, wide, pad)
    V = _log_int(rng, 1000, 151936)
    V = V if rng.random() < 0.3 else -(-V // 8) * 8  # most vocabularies are padded
    if kind < 0.7:
        H = 16 * _log_int(rng, 8, 512)
        T = _log_int(rng, 1, min(2048, 90000000000 // (H * V)))
        return _logits(T, H, V, rng.choice(["bf16", "bf16", "f32"]))
    D = _log_int(rng, 1, 16)
    B = _log_int(rng, 1, min(256, 96000000 // (2 * (D + 1) * V)))
    return _verify(B, D, V, dtype, rng.choice(["model", "model", "lookup"]),
                   rng.choice([1.0, round(rng.uniform(0.3, 1.5), 2)]), rng.random() < 0.5,
                   rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _mask(T, pad, g):
    """A padded batch: responses of up to 256 tokens of which the last ones are padding."""
    if pad == 0:
        return None
    at = torch.arange(T, device=DEV)
    keep = 1 - pad * 2 * torch.rand(T // 256 + 1, generator=g, device=DEV)
    return ((at % 256).float() < 256 * keep[at // 256]).to(torch.uint8)


def _hidden(T, H, g, dtype):
    """Hidden states: a few channels are far larger than the others, as a model's are."""
    wide = torch.exp(0.4 * torch.randn(H, generator=g, device=DEV))
    wide[torch.rand(H, generator=g, device=DEV) < 0.004] *= 12.0
    return (torch.randn((T, H), generator=g, device=DEV) * wide).to(dtype)


def _e4m3(x):
    """Rows in 8 bits, and their scales."""
    scale = x.abs().amax(1).clamp(min=FLOOR) / 448.0
    return (x / scale.view(-1, 1)).to(torch.float8_e4m3fn), scale


def _rows(T, V, g):
    """Rows of logits: a bell of width 2 to 3, and a head of 256 tokens that fall off with the
    logarithm of their rank, as high above the bell as the row is confident."""
    width = 2.0 + torch.rand((T, 1), generator=g, device=DEV)
    n = min(256, V // 4)
    high = width * 4.2 + 6.0 * torch.rand((T, 1), generator=g, device=DEV)
    slope = 0.8 + 1.7 * torch.rand((T, 1), generator=g, device=DEV)
    x = torch.randn((T, V), generator=g, device=DEV).mul_(width)
    at = torch.randint(0, V // n, (T, n), generator=g, device=DEV)
    at = at + torch.arange(n, device=DEV) * (V // n)
    rank = torch.rand((T, n), generator=g, device=DEV).argsort(1) + 1
    return x.scatter_(1, at, high - slope * rank.float().log())


def _prepare_verify(case, g):
    B, D, V, dtype = case["B"], case["D"], case["V"], _dtype(case["dtype"])
    n = torch.full((B,), D, device=DEV)
    if case["ragged"]:
        n = (torch.rand(B, generator=g, device=DEV) * (D + 1)).long()
        n[0] = D
    cu = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    cu[1:] = torch.cumsum(n, 0)
    N = int(cu[-1])
    of = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=N)
    row = torch.arange(N, device=DEV) + of  # each draft's row of logits
    z = _rows(N + B, V, g)
    s = {"case": dict(case), "cu": cu, "draft_z": None, "tau_d": None, "mask": None}
    tau = torch.full((B,), case["tau"], device=DEV)
    if case["mixed"]:
        tau = 0.4 + 0.8 * torch.rand(B, generator=g, device=DEV)
        tau[torch.rand(B, generator=g, device=DEV) < 0.2] = 0.0  # greedy requests
        s["mask"] = (torch.rand(B, generator=g, device=DEV) > 0.1).to(torch.uint8)
    s["tau"] = None if case["tau"] == 1.0 and not case["mixed"] else tau
    if case["draft"] == "model":  # a small model's logits, its tokens drawn from them
        zd = (z[row] + 0.8 * torch.randn((N, V), generator=g, device=DEV)).to(dtype)
        e = torch.empty((N, V), device=DEV).exponential_(generator=g)
        pick = zd.float() / tau.clamp(min=0.05)[of].view(-1, 1) - torch.log(e)
        s["draft_z"], s["tau_d"], ids = zd, s["tau"], pick.argmax(1)
    else:  # right two times in three, for all that the target cares
        some = torch.randint(0, V, (N,), generator=g, device=DEV)
        right = torch.rand(N, generator=g, device=DEV) < 0.67
        ids = torch.where(right, z[row].argmax(1), some)
    s["z"], s["ids"] = z.to(dtype), ids.int()
    s["u"] = torch.rand(N, generator=g, device=DEV)
    s["u_final"] = torch.rand(B, generator=g, device=DEV)
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["family"] == "verify":
        return _prepare_verify(case, g)
    T, H, s = case["T"], case["H"], {"case": dict(case)}
    if case["family"] == "logits":
        s["x"], s["xs"] = _e4m3(_hidden(T, H, g, torch.float32))
        V = case["V"]
        s["w"] = torch.empty((V, H), dtype=torch.float8_e4m3fn, device=DEV)
        s["ws"] = torch.empty(V, device=DEV)
        for a in range(0, V, 16384):
            w = torch.randn((min(16384, V - a), H), generator=g, device=DEV) / math.sqrt(H)
            s["w"][a:a + 16384], s["ws"][a:a + 16384] = _e4m3(w)
        return s
    dtype = _dtype(case["dtype"])
    w = 1.0 + 0.2 * torch.randn(H, generator=g, device=DEV)
    s["w"] = w if case["wide"] else w.to(dtype)  # a norm's weights are often kept in fp32
    s["mask"] = _mask(T, case["pad"], g)
    s["x"] = _hidden(T, H, g, dtype)
    s["r"] = s["dy"] = s["dh"] = None
    if case["family"] == "norm" and case["residual"]:
        s["r"] = _hidden(T, H, g, dtype)
    if case["family"] == "back":
        s["dy"] = (torch.randn((T, H), generator=g, device=DEV) * 1e-3).to(dtype)
        if case["residual"]:
            s["dh"] = (torch.randn((T, H), generator=g, device=DEV) * 1e-3).to(dtype)
    return s


# ------------------------------------------------------------------ the library's calls
_binding = None


def _lib():
    global _binding
    if _binding is None:
        from paper_2609_32444_gb300 import binding
        _binding = binding
    return _binding


def _own_norm(s):
    eight = s["case"]["out"] == "e4m3"
    return _lib().cis_rmsnorm_fwd(s["x"], s["w"], residual=s["r"], eps=EPS, mask=s["mask"],
                                  want_y=not eight, want_q=eight)


def _own_back(s):
    return _lib().cis_rmsnorm_bwd(s["dy"], s["x"], s["w"], dh=s["dh"], eps=EPS, mask=s["mask"])


def _own_logits(s):
    return _lib().cis_lmhead_logits(s["x"], s["xs"], s["w"], s["ws"],
                                    logits_dtype=_dtype(s["case"]["out"]))


def _own_verify(s):
    return _lib().cis_verify_tokens(s["z"], s["ids"], s["cu"], s["u"], s["u_final"],
                                    max_drafts=s["case"]["D"], draft_logits=s["draft_z"],
                                    temperature=s["tau"], draft_temperature=s["tau_d"],
                                    mask=s["mask"], want_lp=True, want_lp_sampled=True)


# ------------------------------------------------------------------ the plain forms
def _plain_norm(s):
    x, w, case = s["x"].float(), s["w"].float(), s["case"]
    h = x if s["r"] is None else x + s["r"].float()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * w
    off = None if s["mask"] is None else (s["mask"] == 0).view(-1, 1)
    if off is not None:
        h, y = h.masked_fill(off, 0.0), y.masked_fill(off, 0.0)
    out = {"h": None if s["r"] is None else h.to(s["x"].dtype), "y": None, "q": None,
           "scale": None}
    if case["out"] == "e4m3":
        scale = y.abs().amax(1, keepdim=True).clamp(min=FLOOR) / 448.0
        out["q"] = (y / scale).to(torch.float8_e4m3fn)
        out["scale"] = scale.view(-1) if off is None else scale.masked_fill(off, 0.0).view(-1)
    else:
        out["y"] = y.to(s["x"].dtype)
    return out


def _plain_back(s):
    dy, h, w = s["dy"].float(), s["x"].float(), s["w"].float()
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    g = dy * w
    dx = r * (g - h * (r * r) * (g * h).mean(1, keepdim=True))
    per = dy * h * r
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    if s["mask"] is not None:
        off = (s["mask"] == 0).view(-1, 1)
        dx, per = dx.masked_fill(off, 0.0), per.masked_fill(off, 0.0)
    return {"dx": dx.to(s["dy"].dtype), "dweight": per.sum(0)}


def _plain_logits(s):
    z = (s["x"].float() @ s["w"].float().t()) * s["xs"].view(-1, 1) * s["ws"].view(1, -1)
    return z.to(_dtype(s["case"]["out"]))


def _plain_verify(s):
    case, z, cu = s["case"], s["z"].double(), s["cu"].long()
    B, D, V = case["B"], case["D"], case["V"]
    n, N = cu[1:] - cu[:-1], s["ids"].numel()
    of = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=N)
    row = torch.arange(N, device=DEV) + of
    ids = s["ids"].long()
    one = torch.ones(B, dtype=torch.float64, device=DEV)
    tau = one if s["tau"] is None else s["tau"].double()
    greedy = tau == 0
    rows_of = torch.repeat_interleave(torch.arange(B, device=DEV), n + 1, output_size=N + B)
    tau_row = torch.where(greedy, one, tau)[rows_of].view(-1, 1)
    top = z.amax(1, keepdim=True)
    raw = (z - top) - torch.log(torch.exp(z - top).sum(1, keepdim=True))
    lp = (z - top) / tau_row
    lp = lp - torch.log(torch.exp(lp).sum(1, keepdim=True))
    p = torch.exp(lp)
    first = torch.where(z == top, torch.arange(V, device=DEV), V).amin(1)  # the largest entry
    if s["draft_z"] is not None:
        tau_d = torch.where(greedy, one, one if s["tau_d"] is None else s["tau_d"].double())
        q = torch.softmax(s["draft_z"].double() / tau_d[of].view(-1, 1), 1)
        qx = torch.gather(q, 1, ids.view(-1, 1)).view(-1)
    else:
        q = torch.zeros((N, V), dtype=torch.float64, device=DEV).scatter_(1, ids.view(-1, 1), 1.0)
        qx = torch.ones(N, dtype=torch.float64, device=DEV)
    ok = s["u"].double() * qx < torch.gather(p[row], 1, ids.view(-1, 1)).view(-1)
    ok = torch.where(greedy[of], ids == first[row], ok)
    grid = torch.arange(D + 1, device=DEV).view(1, -1)
    at = (cu[:-1].view(-1, 1) + grid).clamp(max=max(N - 1, 0))
    there = grid < n.view(-1, 1)
    kept = torch.cumprod((there & ok[at]).long(), 1).sum(1)
    last = cu[:-1] + torch.arange(B, device=DEV) + kept  # the row of the token after them
    mass = p[last]
    less = q[(cu[:-1] + kept).clamp(max=max(N - 1, 0))]
    mass = torch.where((kept < n).view(-1, 1), (mass - less).clamp(min=0.0), mass)
    mass = torch.where(mass.sum(1, keepdim=True) > 0, mass, p[last])
    run_ = torch.cumsum(mass, 1)
    j = (run_ <= s["u_final"].double().view(-1, 1) * run_[:, -1:]).sum(1)
    j = torch.where(greedy, first[last], j)
    on = torch.ones(B, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    kept = torch.where(on, kept, -1)
    out = torch.where(grid < kept.view(-1, 1), ids[at], -1)
    out = torch.where(grid == kept.view(-1, 1), j.view(-1, 1), out)
    where = (cu[:-1] + torch.arange(B, device=DEV)).view(-1, 1) + grid
    where = where.clamp(max=N + B - 1)
    idx = out.clamp(min=0)
    lpo = torch.where(out >= 0, raw[where, idx], 0.0)
    lps = torch.where((out >= 0) & ~greedy.view(-1, 1), lp[where, idx], 0.0)
    return out.int(), kept.int(), lpo.float(), lps.float()


def run(state):
    f = state["case"]["family"]
    if own:
        return {"norm": _own_norm, "back": _own_back, "logits": _own_logits,
                "verify": _own_verify}[f](state)
    return {"norm": _plain_norm, "back": _plain_back, "logits": _plain_logits,
            "verify": _plain_verify}[f](state)


# ------------------------------------------------------------------ work and exact values
def work(case):
    if case["family"] == "verify":
        B, D, V = case["B"], case["D"], case["V"]
        e = 2 if case["dtype"] == "bf16" else 4
        n = B * D / 2 if case["ragged"] else B * D
        rows = n + B + (n if case["draft"] == "model" else 0)
        # the target's and the draft's rows; ids, numbers, the tokens with two log-probabilities
        return {"bytes": rows * V * e + 8 * n + B * (12 + 12 * (D + 1)), "flops": 4 * rows * V}
    T, H = case["T"], case["H"]
    if case["family"] == "logits":
        V, o = case["V"], 2 if case["out"] == "bf16" else 4
        return {"bytes": V * H + T * H + 4 * (T + V) + T * V * o, "flops": 2 * T * H * V}
    e, n = 2 if case["dtype"] == "bf16" else 4, T * (1 - case["pad"])
    we = 4 if case["wide"] or case["dtype"] == "f32" else 2
    if case["family"] == "norm":
        b = n * H * e * (2 if case["residual"] else 1) + H * we + T
        b += T * H * e if case["residual"] else 0
        b += T * (H + 4) if case["out"] == "e4m3" else T * H * e
        return {"bytes": b, "flops": 6 * n * H}
    b = n * H * e * (3 if case["residual"] else 2) + T * H * e + H * (we + 4) + T
    return {"bytes": b, "flops": 12 * n * H}


def _exact_verify(s):
    case, cu, D, V = s["case"], s["cu"].tolist(), s["case"]["D"], s["case"]["V"]
    ids, u, last = s["ids"].tolist(), s["u"].tolist(), s["u_final"].tolist()
    out, kept, lp, lps = [], [], [], []
    for b in range(case["B"]):
        rows, a = s["z"][cu[b] + b:cu[b + 1] + b + 1], cu[b]
        n, one, two, toks = cu[b + 1] - cu[b], [], [], []
        if s["mask"] is not None and s["mask"][b].item() == 0:
            out.append([-1] * (D + 1)), kept.append(-1)
            lp.append([0.0] * (D + 1)), lps.append([0.0] * (D + 1))
            continue
        tau = 1.0 if s["tau"] is None else s["tau"][b].item()
        for i in range(n + 1):
            x = rows[i].double()
            p = torch.softmax(x / tau, 0) if tau > 0 else (x == x.max()).double()
            if tau == 0:  # all of it on the first of the largest
                p = torch.zeros_like(p).index_fill_(0, p.argmax() if p.sum() == 1 else
                                                    p.nonzero()[0], 1.0)
            tok = None
            if i < n:
                t = ids[a + i]
                if s["draft_z"] is None or tau == 0:
                    q = torch.zeros_like(p).index_fill_(0, torch.tensor([t], device=DEV), 1.0)
                else:
                    td = 1.0 if s["tau_d"] is None else s["tau_d"][b].item()
                    q = torch.softmax(s["draft_z"][a + i].double() / td, 0)
                if (p[t] > 0 if tau == 0 else u[a + i] * q[t] < p[t]):
                    tok = t
                elif (p > q).any():
                    p = (p - q).clamp(min=0)
            stop = tok is None
            if stop:
                c = torch.cumsum(p, 0)
                tok = int(torch.searchsorted(c, c[-1:] * last[b], right=True)) if tau > 0 \
                    else int(p.argmax())
            toks.append(tok)
            one.append((x[tok] - torch.logsumexp(x, 0)).item())
            two.append((x[tok] / tau - torch.logsumexp(x / tau, 0)).item() if tau > 0 else 0.0)
            if stop:
                break
        fill = D + 1 - len(toks)
        kept.append(len(toks) - 1), out.append(toks + [-1] * fill)
        lp.append(one + [0.0] * fill), lps.append(two + [0.0] * fill)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    f64 = lambda v: torch.tensor(v, dtype=torch.float64)  # noqa: E731
    return i32(out), i32(kept), f64(lp), f64(lps)


def _exact_norm(s, case):
    h = s["x"].double()
    if s["r"] is not None:
        h = h + s["r"].double()
    on = slice(None) if s["mask"] is None else s["mask"].bool()
    y = torch.zeros_like(h)
    y[on] = h[on] * torch.rsqrt(h[on].pow(2).mean(1, keepdim=True) + EPS) * s["w"].double()
    hz = torch.zeros_like(h)
    hz[on] = h[on]
    out = {"h": None if s["r"] is None else hz, "y": y, "q": None, "scale": None}
    if case["out"] == "e4m3":
        amax = torch.linalg.vector_norm(y, math.inf, dim=1)
        scale = amax.clamp(min=FLOOR) / 448
        out["q"], out["y"] = y / scale[:, None], None
        out["scale"] = scale * (1.0 if s["mask"] is None else s["mask"].double())
    return out


def _exact_back(s):
    """The norm's vector-Jacobian product by its Jacobian, (I - n n^T / H) r with n = h r."""
    h, w = s["x"].double(), s["w"].double()
    r = torch.rsqrt(h.pow(2).mean(1, keepdim=True) + EPS)
    unit, g = h * r, s["dy"].double()
    dx = (g * w - unit * torch.einsum("th,th->t", g * w, unit)[:, None] / h.shape[1]) * r
    if s["dh"] is not None:
        dx += s["dh"].double()
    if s["mask"] is not None:
        m = s["mask"].double()[:, None]
        dx, g = dx * m, g * m
    return {"dx": dx, "dweight": torch.einsum("th,th->h", g, unit)}


def exact(case, seed):
    s, f = prepare(case, seed), case["family"]
    if f == "verify":
        return _exact_verify(s)
    if f == "norm":
        return _exact_norm(s, case)
    if f == "back":
        return _exact_back(s)
    z = torch.empty((case["T"], case["V"]), dtype=torch.float64, device=DEV)
    x = s["x"].double() * s["xs"].double()[:, None]
    for a in range(0, case["V"], 16384):
        w = s["w"][a:a + 16384].double() * s["ws"][a:a + 16384].double()[:, None]
        z[:, a:a + 16384] = x @ w.t()
    return z
