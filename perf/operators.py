"""What the performance of the sampling and distillation calls is measured on.

A rollout step samples a token from each row of logits (cis_sample_tokens); a teacher scores
the rollout and keeps its most likely tokens with their log-probabilities (cis_topk_logprobs);
the student is trained towards those lists (cis_distill_fwd_bwd).  Sizes are those of the
synthetic workloads, the tests and the benchmark, with odd ones beside them.

Families (a case's "family"):
  sample   one decoding step's tokens and their log-probabilities, from given uniform numbers.
  topk     the K most likely tokens of each row, their log-probabilities, the row's logsumexp.
  distill  the loss against a teacher's lists and its gradient with respect to the logits.

Where `own` is false, `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False  # set by whoever measures: true takes the library's calls

DEV = "cuda"
TAIL_MIN = 1e-6
KINDS = ("forward", "reverse", "topk")
FILTERS = ("none", "top_k", "top_p", "both", "min_p", "mixed")


def _topk(T, V, K, dtype="bf16", tau=1.0, pad=0.0):
    return {"family": "topk", "T": T, "V": V, "K": K, "dtype": dtype, "tau": tau, "pad": pad}


def _distill(T, V, K, kind="forward", dtype="bf16", grad="bf16", tau=1.0, pad=0.0,
             seq_mean=False, weighted=False, short=0.0):
    return {"family": "distill", "T": T, "V": V, "K": K, "kind": kind, "dtype": dtype,
            "grad": grad, "tau": tau, "pad": pad, "seq_mean": seq_mean, "weighted": weighted,
            "short": short}


def _sample(T, V, filt="none", dtype="bf16", tau=1.0, flat=False):
    return {"family": "sample", "T": T, "V": V, "filter": filt, "dtype": dtype, "tau": tau,
            "flat": flat}


def listed():
    return [
        # one request's decoding step, the usual settings of a chat model
        dict(_sample(1, 151936, "both", tau=0.6), name="sample_one"),
        # a rollout's decoding step: the model's own distribution, nothing cut off
        dict(_sample(256, 151936), name="sample_rollout"),
        # a serving batch whose requests each have settings of their own; a vocabulary that
        # tokens were added to, fp32 logits
        dict(_sample(512, 32003, "mixed", "f32"), name="sample_mixed"),
        # a wide nucleus: flat rows (a young model, a high temperature)
        dict(_sample(64, 151936, "top_p", tau=1.5, flat=True), name="sample_flat"),
        # a large rollout engine's step with a nucleus
        dict(_sample(1024, 151936, "top_p", tau=0.7), name="sample_nucleus"),
        # the teacher's lists for one decoding step of a few dozen requests
        dict(_topk(24, 151936, 20), name="topk_few"),
        # the teacher's pass over a rollout batch
        dict(_topk(8192, 151936, 64), name="topk_batch"),
        # long lists from fp32 logits with rows of no alignment, softened, a quarter padding
        dict(_topk(2048, 32003, 128, "f32", 2.0, 0.25), name="topk_odd"),
        # the smallest step (the smoke test's size), where the call's own cost counts
        dict(_distill(256, 1024, 16, dtype="f32", grad="f32"), name="distill_small"),
        # a rollout batch against the teacher's lists
        dict(_distill(8192, 151936, 64), name="distill_batch"),
        # on-policy distillation (reverse divergence) of padded responses, each weighing the same
        dict(_distill(4096, 32000, 32, "reverse", pad=0.25, seq_mean=True),
             name="distill_reverse"),
        # renormalised lists of different lengths, softened, fp32, rows of no alignment, weights
        dict(_distill(4096, 32003, 128, "topk", "f32", "f32", 2.0, 0.25, False, True, 0.3),
             name="distill_odd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocab(rng, lo=1000, hi=151936):
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.3 else -(-v // 8) * 8  # most vocabularies are padded


def draw(rng):
    kind = rng.random()
    V = _vocab(rng)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0.0, 0.0, 0.25, 0.4])
    tau = rng.choice([1.0, 1.0, round(rng.uniform(0.5, 4.0), 2)])
    if kind < 0.35:
        return _sample(_log_int(rng, 1, min(1024, 150000000 // V)), V, rng.choice(FILTERS), dtype,
                       rng.choice([1.0, round(rng.uniform(0.3, 1.5), 2)]), rng.random() < 0.15)
    K = _log_int(rng, 1, 256)
    T = _log_int(rng, 8, min(16384, 600000000 // V))
    if kind < 0.65:
        return _topk(T, V, K, dtype, tau, pad)
    return _distill(T, V, K, rng.choice(KINDS), dtype, rng.choice([dtype, dtype, "bf16", "f32"]),
                    tau, pad, rng.random() < 0.3, rng.random() < 0.3,
                    rng.choice([0.0, 0.0, 0.3]))


# ------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(T, V, dtype, g, flat=False):
    """Rows of logits: a bell of width 2 to 3, and a head of 256 tokens that fall off with
    the logarithm of their rank, as high above the bell as the row is confident."""
    z = torch.empty((T, V), dtype=dtype, device=DEV)
    width = 2.0 + torch.rand((T, 1), generator=g, device=DEV)
    n = 0 if flat else min(256, V // 4)
    high = width * 4.2 + 6.0 * torch.rand((T, 1), generator=g, device=DEV)
    slope = 0.8 + 1.7 * torch.rand((T, 1), generator=g, device=DEV)
    step = max(1, (1 << 28) // V)
    for a in range(0, T, step):
        x = torch.randn((min(step, T - a), V), generator=g, device=DEV).mul_(width[a:a + step])
        if n:
            m = x.shape[0]  # one token in each of n stretches, their ranks shuffled
            at = torch.randint(0, V // n, (m, n), generator=g, device=DEV)
            at = at + torch.arange(n, device=DEV) * (V // n)
            rank = torch.rand((m, n), generator=g, device=DEV).argsort(1) + 1
            x.scatter_(1, at, high[a:a + step] - slope[a:a + step] * rank.float().log())
        z[a:a + step] = x
    return z


def _slots(T, pad):
    """Responses of up to 256 tokens, right-padded so that round(pad T) tokens are padding,
    unevenly over the responses: (starts, valid lengths)."""
    n = max(1, T // 256)
    start = [i * T // n for i in range(n + 1)]
    left, out = int(round(pad * T)), []
    for i in range(n):
        size, rest = start[i + 1] - start[i], n - i
        cut = left if rest == 1 else int(left / rest * (0.4 + 1.2 * ((i * 7 + 3) % 11) / 10.0))
        cut = max(left - (T - start[i + 1]), min(cut, left, size - 1 if rest > 1 else size))
        left -= cut
        out.append(size - cut)
    return start, out


def _mask(T, pad):
    start, length = _slots(T, pad)
    mask = torch.zeros(T, dtype=torch.uint8)
    for a, n in zip(start, length):
        mask[a:a + n] = 1
    return mask.to(DEV) if pad > 0 else None, torch.tensor(start, dtype=torch.int32, device=DEV)


def _lists(z, K, tau, g):
    """A teacher's lists: its logits are the student's, each moved by N(0, 0.5^2); their K
    largest, with the log-probabilities of its own softmax."""
    T, V = z.shape
    ids = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    lp = torch.full((T, K), -math.inf, device=DEV)
    step = max(1, (1 << 27) // V)
    k = min(K, V)
    for a in range(0, T, step):
        x = z[a:a + step].float()
        x = (x + 0.5 * torch.randn(x.shape, generator=g, device=DEV)) / tau
        v, i = torch.topk(x, k, dim=1)
        ids[a:a + step, :k] = i.int()
        lp[a:a + step, :k] = v - torch.logsumexp(x, 1, keepdim=True)
    return ids, lp


def _settings(case, g):
    """Each row's temperature, top_k, top_p and min_p (None: the call goes without)."""
    T, f = case["T"], case["filter"]
    r = [torch.rand(T, generator=g, device=DEV) for _ in range(5)]
    if f == "mixed":
        tau = 0.4 + 0.8 * r[0]
        tau[r[4] < 0.1] = 0.0  # greedy requests
        k = torch.where(r[1] < 0.5, 0, (1 + 99 * r[2])).int()
        p = torch.where(r[2] < 0.5, 1.0, 0.7 + 0.29 * r[1]).float()
        m = torch.where(r[3] < 0.7, 0.0, 0.2 * r[0]).float()
        return {"temperature": tau, "top_k": k, "top_p": p, "min_p": m}
    tau = None if case["tau"] == 1.0 else torch.full((T,), case["tau"], device=DEV)
    k = (10 + 50 * r[1]).int() if f in ("top_k", "both") else None
    p = (0.8 + 0.18 * r[2]) if f in ("top_p", "both") else None
    m = (0.01 + 0.1 * r[3]) if f == "min_p" else None
    return {"temperature": tau, "top_k": k, "top_p": p, "min_p": m}


def prepare(case, seed):
    g = _gen(seed)
    T, V = case["T"], case["V"]
    s = {"case": dict(case), "z": _rows(T, V, _dtype(case["dtype"]), g, case.get("flat", False))}
    if case["family"] == "sample":
        s["u"] = torch.rand(T, generator=g, device=DEV)
        s["set"] = _settings(case, g)
        return s
    s["mask"], cu = _mask(T, case["pad"])
    if case["family"] == "distill":
        s["ids"], s["lp"] = _lists(s["z"], case["K"], case["tau"], g)
        if case["short"] > 0:  # lists that end early: the slots after their end are empty
            n = (torch.rand((T, 1), generator=g, device=DEV) * case["K"]).long() + 1
            cut = torch.rand((T, 1), generator=g, device=DEV) < case["short"]
            s["ids"][cut & (torch.arange(case["K"], device=DEV).view(1, -1) >= n)] = -1
        s["cu"] = cu if case["seq_mean"] else None
        s["w"] = torch.rand(T, generator=g, device=DEV) * 2 if case["weighted"] else None
    return s


# ------------------------------------------------------------------ the library's calls
_binding = None


def _lib():
    global _binding
    if _binding is None:
        from paper_2609_32444_gb300 import binding
        _binding = binding
    return _binding


def _own_sample(s):
    return _lib().cis_sample_tokens(s["z"], s["u"], **s["set"], want_lp=True,
                                    want_lp_sampled=True)


def _own_topk(s):
    return _lib().cis_topk_logprobs(s["z"], s["case"]["K"], temperature=s["case"]["tau"],
                                    mask=s["mask"], want_lse=True)


def _own_distill(s):
    if "params" not in s:  # set up once, like an optimiser's
        case = s["case"]
        s["params"] = _lib().cis_distill_default_params(
            case["kind"], temperature=case["tau"], tail_min=TAIL_MIN, agg=int(case["seq_mean"]))
    out = _lib().cis_distill_fwd_bwd(s["z"], s["ids"], s["lp"], s["params"], mask=s["mask"],
                                     cu_seqlens=s["cu"], token_weight=s["w"],
                                     dlogits_dtype=_dtype(s["case"]["grad"]))
    return {"dlogits": out["dlogits"], "kl": out["kl"], "loss": out["loss"].float()}


# ------------------------------------------------------------------ the plain forms
def _plain_sample(s):
    z, u, opt = s["z"].float() + 0.0, s["u"].double().view(-1, 1), s["set"]
    T, V = z.shape
    one = torch.ones((T, 1), dtype=torch.float64, device=z.device)
    tau = one if opt["temperature"] is None else opt["temperature"].double().view(-1, 1)
    greedy = tau == 0
    tau = torch.where(greedy, one, tau)
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    x = (zs.double() - zs[:, :1].double()) / tau
    w = torch.exp(x)
    keep = torch.ones_like(w, dtype=torch.bool)
    if opt["top_k"] is not None:
        k = opt["top_k"].long().view(-1, 1)
        keep = torch.arange(V, device=z.device).view(1, -1) < torch.where(k > 0, k, V)
    if opt["top_p"] is not None:
        p = opt["top_p"].double().view(-1, 1)
        mass = torch.cumsum(w * keep, 1)
        before = torch.cat([torch.zeros_like(one), mass[:, :-1]], 1)
        keep = keep & ((before < p * mass[:, -1:]) | (p >= 1))
    if opt["min_p"] is not None:
        keep = keep & (x >= torch.log(opt["min_p"].double().view(-1, 1)))
    kept = torch.zeros_like(w).scatter_(1, order, w * keep)
    mass = torch.cumsum(kept, 1)
    total = mass[:, -1:]
    ids = (mass <= u * total).sum(1, keepdim=True)
    ids = torch.where(greedy, order[:, :1], ids)
    zi = torch.gather(z, 1, ids).double()
    top = zs[:, :1].double()
    lp = zi - top - torch.log(torch.exp(z - zs[:, :1]).sum(1, keepdim=True, dtype=torch.float64))
    lps = torch.where(greedy, torch.zeros_like(one), (zi - top) / tau - torch.log(total))
    return ids.view(-1).int(), lp.view(-1).float(), lps.view(-1).float()


def _plain_topk(s):
    case, z = s["case"], s["z"].float() + 0.0
    T, V = z.shape
    k = min(case["K"], V)
    bits = z.view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)  # in the order of the values
    key = (key << 32) | (0xFFFFFFFF - torch.arange(V, device=z.device))  # ties: the lowest index
    best = torch.topk(key, k, dim=1).values
    del key, bits
    at = 0xFFFFFFFF - (best & 0xFFFFFFFF)
    x = z / case["tau"]
    lse = torch.logsumexp(x, 1)
    lp = torch.gather(x, 1, at) - lse.view(-1, 1)
    ids = at.int()
    if k < case["K"]:
        more = (0, case["K"] - k)
        ids = torch.nn.functional.pad(ids, more, value=-1)
        lp = torch.nn.functional.pad(lp, more, value=-math.inf)
    if s["mask"] is not None:
        off = s["mask"] == 0
        ids, lp = ids.masked_fill(off.view(-1, 1), -1), lp.masked_fill(off.view(-1, 1), -math.inf)
        lse = lse.masked_fill(off, 0.0)
    return ids, lp, lse


def _scale(mask, cu, T):
    """s_t: 1/n over the valid tokens, or 1/(G |y_i|) over responses; 0 where masked."""
    m = torch.ones(T, device=DEV) if mask is None else (mask != 0).float()
    if cu is None:
        return m / m.sum().clamp(min=1)
    of = torch.repeat_interleave(torch.arange(cu.numel() - 1, device=DEV),
                                 (cu[1:] - cu[:-1]).long(), output_size=T)
    n = torch.zeros(cu.numel() - 1, device=DEV).index_add_(0, of, m)
    return m / (n[of].clamp(min=1) * (n > 0).sum())


def _plain_distill(s):
    case, z = s["case"], s["z"]
    T, V = z.shape
    kind, tau = case["kind"], case["tau"]
    on = (s["ids"] >= 0) & (s["lp"] > -math.inf)
    at = torch.where(on, s["ids"], 0).long()
    top = z.float().amax(1, keepdim=True)
    e = torch.exp((z.float() - top) / tau)  # 32 bits an entry; a row's numbers in 64
    S = e.sum(1, keepdim=True, dtype=torch.float64)
    lk = (torch.gather(z, 1, at).double() - top.double()) / tau - torch.log(S)  # log p, listed
    a = s["lp"].double().masked_fill(~on, -math.inf)
    d = e / S.float()  # the softmax
    if kind == "topk":
        most = a.amax(1, keepdim=True)
        loga = a - most - torch.log(torch.exp(a - most).sum(1, keepdim=True))
        q = torch.where(on, torch.exp(loga), 0.0)
        kl = torch.where(on, q * (loga - lk), 0.0).sum(1)
        d.scatter_add_(1, at, -q.float())
    else:
        out = torch.zeros((T, V), device=DEV).scatter_add_(1, at, on.float()) > 0  # the listed
        pr = e.masked_fill_(out, 0.0).sum(1, keepdim=True, dtype=torch.float64) / S
        q = torch.where(on, torch.exp(a), 0.0)
        rest = 1 - q.sum(1, keepdim=True)
        if kind == "forward":
            rest = torch.where(rest < TAIL_MIN, 0.0, rest)
            has, total = rest > 0, q.sum(1, keepdim=True) + rest
            kl = torch.where(on, q * (a - lk), 0.0).sum(1) + torch.where(
                has, rest * (torch.log(rest) - torch.log(pr)), 0.0).sum(1)
            low = total - torch.where(has, rest / pr, 0.0)
            d *= torch.where(out, total.float(), low.float())
            d.scatter_add_(1, at, -q.float())
        else:
            rest = rest.clamp(min=TAIL_MIN)
            pk = torch.where(on, torch.exp(lk), 0.0)
            far, fr = lk - a, torch.log(pr) - torch.log(rest)
            mean = torch.where(pk > 0, pk * far, 0.0).sum(1, keepdim=True) + torch.where(
                pr > 0, pr * fr, 0.0)
            d *= (fr - mean).float()
            d.masked_fill_(out, 0.0)
            d.scatter_add_(1, at, torch.where(pk > 0, pk * (far - mean), 0.0).float())
            kl = mean.view(-1)
    some = on.any(1) if kind == "topk" else torch.ones(T, dtype=torch.bool, device=DEV)
    if s["mask"] is not None:
        some = some & (s["mask"] != 0)
    kl = torch.where(some, kl, 0.0)
    c = _scale(s["mask"], s["cu"], T)
    if s["w"] is not None:
        c = c * s["w"]
    loss = (c.double() * kl).sum().float().view(1)
    d = torch.where(some.view(-1, 1), d * (c / tau).view(-1, 1), 0.0)
    return {"dlogits": d.to(_dtype(case["grad"])), "kl": kl.float(), "loss": loss}


def run(state):
    f = state["case"]["family"]
    if own:
        return {"sample": _own_sample, "topk": _own_topk, "distill": _own_distill}[f](state)
    return {"sample": _plain_sample, "topk": _plain_topk, "distill": _plain_distill}[f](state)


# ------------------------------------------------------------------ work and exact values
def work(case):
    T, V = case["T"], case["V"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["family"] == "sample":
        # logits once; the uniform number and the settings; id and two log-probabilities
        return {"bytes": T * V * e + T * (4 + 12 + 12), "flops": 4 * T * V}
    n = T - int(round(case["pad"] * T))
    if case["family"] == "topk":
        return {"bytes": n * V * e + T * (8 * case["K"] + 4), "flops": 4 * n * V}
    o = 2 if case["grad"] == "bf16" else 4
    return {"bytes": n * V * e + T * V * o + n * 8 * case["K"] + 8 * T, "flops": 7 * n * V}


def _exact_sample(s):
    z, opt = s["z"].double(), s["set"]
    T, V = z.shape
    ids, lp, lps = [], [], []
    col = lambda v, i, off: off if v is None else v[i].item()  # noqa: E731
    for i in range(T):
        x, tau = z[i], col(opt["temperature"], i, 1.0)
        best = x.max()
        raw = torch.logsumexp(x, 0)
        if tau == 0:
            j = int((x == best).nonzero()[0])
            ids.append(j), lp.append((x[j] - raw).item()), lps.append(0.0)
            continue
        p = torch.softmax(x / tau, 0)
        k, top, low = col(opt["top_k"], i, 0), col(opt["top_p"], i, 1.0), col(opt["min_p"], i, 0.0)
        v, at = torch.sort(x, descending=True, stable=True)
        n = V if k <= 0 else min(k, V)
        if top < 1:
            c = torch.cumsum(p[at[:n]], 0)
            n = min(n, int((c < top * c[-1]).sum()) + 1)
        if low > 0:
            n = min(n, int(((v - best) / tau >= math.log(low)).sum()))
        kept = torch.sort(at[:n]).values
        c = torch.cumsum(p[kept], 0)
        j = int(kept[torch.searchsorted(c, s["u"][i].double() * c[-1], right=True)])
        ids.append(j), lp.append((x[j] - raw).item())
        lps.append((x[j] / tau - torch.logsumexp(x[kept] / tau, 0)).item())
    f = lambda v: torch.tensor(v, dtype=torch.float64)  # noqa: E731
    return torch.tensor(ids, dtype=torch.int32), f(lp), f(lps)


def _exact_topk(s, K, tau):
    z = s["z"]
    T, V = z.shape
    ids = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    lp = torch.full((T, K), -math.inf, dtype=torch.float64, device=DEV)
    lse = torch.zeros(T, dtype=torch.float64, device=DEV)
    rows = range(T) if s["mask"] is None else (s["mask"] != 0).nonzero().view(-1).tolist()
    step = max(1, (1 << 27) // V)
    rows = torch.tensor(list(rows), device=DEV)
    for part in rows.split(step):
        v, at = torch.sort(z[part].double(), dim=1, descending=True, stable=True)
        e = torch.exp((v - v[:, :1]) / tau).sum(1).log() + v[:, 0] / tau
        n = min(K, V)
        ids[part, :n] = at[:, :n].int()
        lp[part, :n] = v[:, :n] / tau - e.view(-1, 1)
        lse[part] = e
    return ids, lp, lse


def _exact_distill(s, case):
    z, kind, tau, K = s["z"], case["kind"], case["tau"], case["K"]
    T, V = z.shape
    dz = torch.zeros((T, V), dtype=torch.float64, device=DEV)
    kl = torch.zeros(T, dtype=torch.float64, device=DEV)
    valid = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    c = torch.zeros(T, dtype=torch.float64, device=DEV)
    if s["cu"] is None:
        c[valid] = 1.0 / max(1, int(valid.sum()))
    else:
        cut = s["cu"].tolist()
        n = [int(valid[a:b].sum()) for a, b in zip(cut, cut[1:])]
        for (a, b), m in zip(zip(cut, cut[1:]), n):
            if m:
                c[a:b] = 1.0 / (m * sum(x > 0 for x in n))
        c = c * valid
    if s["w"] is not None:
        c = c * s["w"].double()
    step = max(1, (1 << 26) // V)
    for a in range(0, T, step):
        p = torch.softmax(z[a:a + step].double() / tau, 1)
        ids, lq = s["ids"][a:a + step].long(), s["lp"][a:a + step].double()
        q = torch.zeros((p.shape[0], V + 1), dtype=torch.float64, device=DEV)
        none = (ids < 0) | (lq == -math.inf)
        if kind == "topk":
            lq = torch.log_softmax(lq.masked_fill(none, -math.inf), 1)
        # a column past the vocabulary takes the empty slots
        q.scatter_(1, ids.masked_fill(none, V), lq.exp().masked_fill(none, 0.0))
        q = q[:, :V]
        inside = q > 0
        if kind == "topk":
            kl[a:a + step] = torch.special.xlogy(q, q / p).sum(1)
            dz[a:a + step] = p * q.sum(1, keepdim=True) - q
            continue
        rest = 1 - q.sum(1, keepdim=True)
        pr = p.masked_fill(inside, 0.0).sum(1, keepdim=True)
        if kind == "forward":
            rest = rest * (rest >= TAIL_MIN)
            kl[a:a + step] = (torch.special.xlogy(q, q / p).sum(1, keepdim=True)
                              + torch.special.xlogy(rest, rest / pr)).view(-1)
            total = q.sum(1, keepdim=True) + rest
            dz[a:a + step] = total * p - torch.where(inside, q, p * (rest / pr))
        else:
            rest = rest.clamp(min=TAIL_MIN)
            far = torch.where(inside, torch.log(p / q), torch.log(pr / rest))
            mean = (p * far).sum(1, keepdim=True)
            kl[a:a + step] = mean.view(-1)
            dz[a:a + step] = p * (far - mean)
    kl = kl * valid
    dz *= (c / tau).view(-1, 1)
    return {"dlogits": dz, "kl": kl, "loss": (c * kl).sum().view(1)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["family"] == "sample":
        return _exact_sample(s)
    if case["family"] == "topk":
        return _exact_topk(s, case["K"], case["tau"])
    return _exact_distill(s, case)
