"""The operators on the record of a row's top logits, as measurable cases.

A record is the short form of a row of V logits: its k largest logits with
their token ids and, where the reader needs it, the logarithm of the mass of
all the others relative to the largest one's.  Three operators make and read it:

  topk     the record of each row, and a token drawn from it (what a draft
           model proposes from, what a replay buffer keeps of the teacher);
  distill  loss and gradient of a student's rows against a teacher's record;
  verify   acceptance, first rejection and extra token of proposals that were
           drawn from the draft's record.

`run` computes them in plain torch operations where `own` is false, and calls
the library where it is true.  Logits follow the recipe of the other measured
workloads (target ~ N(0, std^2), draft = target + N(0, noise^2)), made on the
GPU with torch's seeded generator.  (Temperatures are float32 in the library:
the ones here are exact in it.)
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
MAX_V = {"bf16": 131072, "f32": 65536}
MAX_K = 256  # slots of a record


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------

def listed():
    return [
        # One user's stream: the draft model's next token, drawn from its 64
        # largest logits.  The smallest call; latency and host time count.
        dict(name="topk_token_single", op="topk", N=1, V=32000, k=64, dtype="bf16", T=1.0, std=3.0, rest=False,
             draw=True),
        # The same step of a serving batch whose head answers in float32 for a
        # vocabulary with a few added tokens (rows on no 16-byte boundary).
        dict(name="topk_token_batch", op="topk", N=64, V=32003, k=50, dtype="f32", T=0.75, std=2.5, rest=False,
             draw=True),
        # What a verification step leaves in the replay buffer: the records of
        # its 64 x 9 target rows.
        dict(name="topk_record_step", op="topk", N=576, V=32128, k=64, dtype="bf16", T=0.75, std=2.5, rest=True,
             draw=False),
        # Records of a large vocabulary, the pass that fills a buffer.
        dict(name="topk_record_large_vocab", op="topk", N=2048, V=128256, k=128, dtype="bf16", T=1.0, std=3.0,
             rest=True, draw=False),
        # One sequence's online update, a large vocabulary and the longest
        # record: few and long rows.
        dict(name="distill_single", op="distill", B=1, K=4, V=128256, k=256, dtype="bf16", T=1.0, std=3.0, noise=1.0,
             kind="fkl", beta=0.5, masked=1.0, rest=True, grad=True),
        # Every position of a verification step, from the step's own records.
        dict(name="distill_step", op="distill", B=64, K=8, V=32128, k=64, dtype="bf16", T=0.75, std=2.5, noise=1.5,
             kind="jsd", beta=0.5, masked=1.0, rest=True, grad=True),
        # Float32 logits of an odd vocabulary against short records: the loss
        # alone, as an evaluation between updates takes it.
        dict(name="distill_eval_f32", op="distill", B=32, K=6, V=50257, k=20, dtype="f32", T=1.0, std=3.0, noise=1.0,
             kind="rkl", beta=0.5, masked=1.0, rest=True, grad=False),
        # A training pass over the buffer of stored positions, 40 % of them
        # selected, the teacher truncated to its record.
        dict(name="distill_buffer", op="distill", B=16384, K=1, V=32000, k=64, dtype="bf16", T=1.0, std=3.0,
             noise=1.0, kind="fkl", beta=0.5, masked=0.4, rest=False, grad=True),
        # One user's stream, four proposals.
        dict(name="verify_single", op="verify", B=1, K=4, V=32000, k=64, dtype="bf16", T=1.0, std=3.0, noise=1.0,
             ragged=False),
        # A full serving batch.
        dict(name="verify_batch", op="verify", B=64, K=8, V=32128, k=64, dtype="bf16", T=0.75, std=2.5, noise=1.5,
             ragged=False),
        # Float32 target rows of a vocabulary with a few added tokens,
        # proposals of ragged lengths from short records.
        dict(name="verify_f32_added_tokens", op="verify", B=32, K=6, V=32003, k=20, dtype="f32", T=1.0, std=3.0,
             noise=1.0, ragged=True),
        # A large batch of a large-vocabulary model.
        dict(name="verify_large_vocab", op="verify", B=256, K=8, V=128256, k=128, dtype="bf16", T=0.875, std=3.0,
             noise=1.0, ragged=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# A drawn case moves at most this many bytes (below the largest listed case of
# its operator).
_DRAW_BYTES = {"topk": 5.0e8, "distill": 1.2e9, "verify": 5.0e8}


def draw(rng):
    while True:
        op = rng.choice(["topk", "distill", "verify"])
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        V = _log_uniform(rng, 8000, MAX_V[dtype])
        if rng.random() < 0.5:  # vocabularies are often padded
            V = V // 64 * 64
        case = dict(op=op, V=V, k=_log_uniform(rng, 1, MAX_K), dtype=dtype, T=rng.choice([0.75, 0.875, 1.0]),
                    std=rng.choice([2.0, 2.5, 3.0]))
        if op == "topk":
            sampled = rng.random() < 0.5
            case.update(N=_log_uniform(rng, 1, 8192), rest=not sampled or rng.random() < 0.3, draw=sampled)
        elif op == "distill":
            kind = rng.choice(["fkl", "rkl", "jsd"])
            case.update(B=_log_uniform(rng, 1, 8192), K=rng.choice([1, 4, 8]), noise=rng.choice([0.25, 1.0, 2.0]),
                        kind=kind, beta=rng.choice([0.25, 0.5, 0.75]), masked=rng.choice([0.4, 1.0]),
                        rest=kind == "rkl" or rng.random() < 0.6, grad=rng.random() < 0.8)
        else:
            case.update(B=_log_uniform(rng, 1, 512), K=rng.randint(1, 16), noise=rng.choice([0.25, 1.0, 2.0]),
                        ragged=rng.random() < 0.4)
        if work(case)["bytes"] <= _DRAW_BYTES[op]:
            return case


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _normal(shape, scale, g):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale)


def _record(x, k, T, rest):
    """Record of float32 rows that hold values of the logits' dtype (its k
    largest logits in descending order)."""
    top, ids = x.topk(k, -1)
    if not rest:
        return ids.to(torch.int32), top, None
    left = x.scatter(-1, ids, -math.inf)
    return ids.to(torch.int32), top, torch.logsumexp((left - top[..., :1]) / T, -1)


def _teacher_record(case, rows, g):
    """Student rows, and the record of their teacher's rows, some at a time."""
    dt, V, k = DTYPES[case["dtype"]], case["V"], case["k"]
    s = torch.empty(rows, V, dtype=dt, device=DEV)
    ids = torch.empty(rows, k, dtype=torch.int32, device=DEV)
    top = torch.empty(rows, k, dtype=dt, device=DEV)
    rest = torch.empty(rows, dtype=torch.float32, device=DEV) if case["rest"] else None
    step = max(1, (64 << 20) // V)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        t = _normal((n, V), case["std"], g).to(dt).float()
        s[r:r + n] = t + _normal((n, V), case["noise"], g)
        i, v, m = _record(t, k, case["T"], case["rest"])
        ids[r:r + n], top[r:r + n] = i, v
        if rest is not None:
            rest[r:r + n] = m
    return s, ids, top, rest


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op, V, k, T = case["op"], case["V"], case["k"], case["T"]
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if op == "topk":
        s["x"] = _normal((case["N"], V), case["std"], g).to(dt)
        s["u"] = torch.rand(case["N"], generator=g, device=DEV) if case["draw"] else None
        return s
    B, K = case["B"], case["K"]
    if op == "distill":
        x, ids, top, rest = _teacher_record(case, B * K, g)
        s["x"] = x.view(B, K, V)
        s["ids"], s["top"] = ids.view(B, K, k), top.view(B, K, k)
        s["rest"] = None if rest is None else rest.view(B, K)
        s["mask"] = None
        if case["masked"] < 1.0:
            s["mask"] = (torch.rand(B, K, generator=g, device=DEV) < case["masked"]).to(torch.uint8)
        return s
    t = _normal((B, K + 1, V), case["std"], g)
    d = (t[:, :K] + _normal((B, K, V), case["noise"], g)).to(dt)
    s["x"] = t.to(dt)
    ids, top, _ = _record(d.float(), k, T, False)
    s["ids"], s["top"] = ids, top.to(dt)
    # One proposal per row, drawn from the record (largest logit + Gumbel noise).
    noise = torch.empty(B, K, k, device=DEV).exponential_(generator=g).log_()
    s["tokens"] = ids.gather(-1, (top / T - noise).argmax(-1, keepdim=True)).squeeze(-1)
    s["ua"] = torch.rand(B, K, generator=g, device=DEV)
    s["ur"] = torch.rand(B, generator=g, device=DEV)
    s["len"] = torch.randint(1, K + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if case["ragged"] else None
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        import paper_2310_07177_amd as osd
        if case["op"] == "topk":
            out = osd.osd_topk(s["x"], case["k"], case["T"], u=s["u"], rest=case["rest"])
        elif case["op"] == "distill":
            out = osd.osd_distill_topk_loss_grad(s["ids"], s["top"], s["rest"], s["x"], case["kind"], case["beta"],
                                                 case["T"], mask=s["mask"], grad=case["grad"])
        else:
            out = osd.osd_verify_topk(s["x"], s["ids"], s["top"], s["tokens"], s["ua"], s["ur"], case["T"],
                                      draft_len=s["len"])
        return [o for o in out if o is not None]
    return {"topk": _topk, "distill": _distill, "verify": _verify}[case["op"]](s, case)


def _topk(s, case):
    """The k largest logits, the lowest id first among equal ones."""
    x = s["x"].float()
    top, ids = torch.sort(x, dim=-1, descending=True, stable=True)
    top, ids = top[:, :case["k"]], ids[:, :case["k"]]
    out = [ids.to(torch.int32), top.to(s["x"].dtype)]
    if case["rest"]:  # the mass of the others, relative to the row's maximum
        e = torch.exp((x - top[:, :1]) / case["T"]).scatter(-1, ids, 0.0)
        out.append(torch.log(e.sum(-1)))
    if case["draw"]:  # in 64 bits: a uniform may lie next to an edge
        c = torch.exp((top.double() - top[:, :1].double()) / case["T"]).cumsum(-1)
        r = (c <= s["u"].double().unsqueeze(-1) * c[:, -1:]).sum(-1, keepdim=True).clamp_max(case["k"] - 1)
        out.append(ids.gather(-1, r).squeeze(-1).to(torch.int32))
    return out


def _distill(s, case):
    tau, beta, kind = case["T"], case["beta"], case["kind"]
    x, ids = s["x"].float() / tau, s["ids"].long()
    # Teacher and student over k + 1 buckets: the record's tokens, the others.
    t = (s["top"].float() - s["top"][..., :1].float()) / tau
    last = torch.full_like(t[..., :1], -math.inf) if s["rest"] is None else s["rest"].unsqueeze(-1)
    t = torch.cat([t, last], -1)
    p = torch.exp(t - t.amax(-1, keepdim=True))
    Sp = p.sum(-1, keepdim=True)
    lp, p = t - t.amax(-1, keepdim=True) - torch.log(Sp), p / Sp
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    left = e.scatter(-1, ids, 0.0).sum(-1, keepdim=True)
    S = left + e.gather(-1, ids).sum(-1, keepdim=True)
    lq = torch.cat([x.gather(-1, ids) - m, torch.log(left)], -1) - torch.log(S)
    q = torch.exp(lq)
    if kind == "fkl":
        D = torch.where(p > 0, p * (lp - lq), 0.0).sum(-1)
        f = 1.0 - p / q
    elif kind == "rkl":
        D = (q * (lq - lp)).sum(-1)
        f = lq - lp - D.unsqueeze(-1)
    else:
        lm = torch.log(beta * p + (1.0 - beta) * q)
        Dq = (q * (lq - lm)).sum(-1)
        D = beta * torch.where(p > 0, p * (lp - lm), 0.0).sum(-1) + (1.0 - beta) * Dq
        f = (1.0 - beta) * (lq - lm - Dq.unsqueeze(-1))
    on = torch.ones_like(D) if s["mask"] is None else s["mask"].float()
    D = torch.where(on > 0, D, 0.0)
    total = D.double().sum()
    out = [torch.stack([total / on.double().sum().clamp_min(1.0), total]).float(), D]
    if case["grad"]:
        # Every token's gradient is its probability times its bucket's factor.
        g = (e / S) * f[..., -1:]
        kept = torch.exp(x.gather(-1, ids) - m) / S * f[..., :-1]
        if kind == "fkl":
            kept = q[..., :-1] - p[..., :-1]
        g = g.scatter(-1, ids, kept) * (on / tau).unsqueeze(-1)
        out.append(g.to(s["x"].dtype))
    return out


def _verify(s, case):
    """All in 64 bits: a uniform may lie next to a border."""
    T, K = case["T"], case["K"]
    B = s["x"].shape[0]
    ids, y = s["ids"].long(), s["tokens"].long()
    length = torch.full((B,), K, device=DEV) if s["len"] is None else s["len"].long()
    x = s["x"].double() / T
    e = torch.exp(x - x.amax(-1, keepdim=True))
    S = e.sum(-1)
    d = s["top"].double() / T
    q = torch.exp(d - d.amax(-1, keepdim=True))
    q = q / q.sum(-1, keepdim=True)
    py = e[:, :K].gather(-1, y.unsqueeze(-1)).squeeze(-1) / S[:, :K]
    qy = torch.where(ids == y.unsqueeze(-1), q, 0.0).sum(-1)
    i = torch.arange(K, device=DEV)
    stops = (i >= length.unsqueeze(-1)) | ~(s["ua"].double() * qy < py)
    a = torch.cumprod((~stops).long(), -1).sum(-1)
    rejected = a < length
    rows = torch.arange(B, device=DEV)
    pa = e[rows, a] / S[rows, a].unsqueeze(-1)
    ja = a.clamp_max(K - 1)
    r = pa.scatter_add(-1, ids[rows, ja], torch.where(rejected.unsqueeze(-1), -q[rows, ja], 0.0)).clamp_min(0.0)
    c = r.cumsum(-1)
    extra = (c <= s["ur"].double().unsqueeze(-1) * c[:, -1:]).sum(-1).clamp_max(case["V"] - 1)
    place = torch.arange(K + 1, device=DEV)
    padded = torch.cat([y, y[:, :1]], -1)
    toks = torch.where(place < a.unsqueeze(-1), padded, torch.where(place == a.unsqueeze(-1), extra.unsqueeze(-1), -1))
    rmask = (i == a.unsqueeze(-1)) & rejected.unsqueeze(-1)
    return [a.to(torch.int32), toks.to(torch.int32), rmask.to(torch.uint8)]


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    """Every row that the operator needs read once, every output written once.
    (Ragged lengths count with their mean (K + 1) / 2, a verification reads the
    target rows of every proposal and one bonus row per sequence.)"""
    op, V, k, es = case["op"], case["V"], case["k"], SIZE[case["dtype"]]
    slot = k * (4 + es)
    if op == "topk":
        N = case["N"]
        more = (4 if case["rest"] else 0) + (8 if case["draw"] else 0)
        return dict(bytes=N * (V * es + slot + more), flops=N * V * (4 if case["rest"] else 1))
    B, K = case["B"], case["K"]
    if op == "distill":
        n = B * K
        on = n * case["masked"]
        more = 4 + (1 if case["masked"] < 1.0 else 0)
        read = on * (V * es + slot + (4 if case["rest"] else 0))
        return dict(bytes=int(read + n * ((V * es if case["grad"] else 0) + more) + 8),
                    flops=int(on * V * (8 if case["grad"] else 4)))
    m = (K + 1) / 2 if case["ragged"] else K
    return dict(bytes=int(B * ((m + 1) * V * es + m * (slot + 9) + 4 * (K + 3))), flops=int(B * (m + 1) * V * 4))


# --------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"topk": _exact_topk, "distill": _exact_distill, "verify": _exact_verify}[case["op"]](s, case)


def _exact_topk(s, case):
    k, T, x = case["k"], case["T"], s["x"]
    N, V = x.shape
    ids = torch.empty(N, k, dtype=torch.int32, device=DEV)
    top = torch.empty(N, k, dtype=torch.float64, device=DEV)
    rest = torch.empty(N, dtype=torch.float64, device=DEV)
    place = torch.arange(V, device=DEV)
    step = max(1, (16 << 20) // V)
    for r in range(0, N, step):
        z = x[r:r + step]
        # One whole number per element: the float's order, then the lower id.
        bits = z.float().view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        at = ((order << 20) | (V - 1 - place)).topk(k, -1).values & 0xFFFFF
        at = V - 1 - at
        ids[r:r + step] = at.to(torch.int32)
        top[r:r + step] = z.double().gather(-1, at)
        if case["rest"]:
            others = z.double().scatter(-1, at, -math.inf) - top[r:r + step, :1]
            rest[r:r + step] = torch.logsumexp(others / T, -1)
    out = [ids, top]
    if case["rest"]:
        out.append(rest)
    if case["draw"]:
        edge = torch.softmax(top / T, -1).cumsum(-1)
        rank = torch.searchsorted(edge, s["u"].double().unsqueeze(-1) * edge[:, -1:], right=True).clamp_max(k - 1)
        out.append(ids.gather(-1, rank).squeeze(-1))
    return out


def _exact_distill(s, case):
    """The divergence by its definition; the gradient by differentiating it."""
    tau, beta, kind, k = case["T"], case["beta"], case["kind"], case["k"]
    n = case["B"] * case["K"]
    x, ids, top = s["x"].view(n, -1), s["ids"].view(n, k).long(), s["top"].view(n, k)
    V = x.shape[1]
    on = torch.ones(n, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].view(n) != 0
    D = torch.zeros(n, dtype=torch.float64, device=DEV)
    grad = torch.zeros(n, V, dtype=torch.float64, device=DEV) if case["grad"] else None
    rows = on.nonzero().squeeze(-1)
    step = max(1, (16 << 20) // V)
    for r in range(0, rows.numel(), step):
        at = rows[r:r + step]
        z = x[at].double().requires_grad_(case["grad"])
        t = (top[at] - top[at, :1].double()) / tau
        if s["rest"] is not None:
            t = torch.cat([t, s["rest"].view(n)[at].double().unsqueeze(-1)], -1)
        lp = torch.log_softmax(t, -1)
        lq = torch.log_softmax(z / tau, -1)
        others = torch.logsumexp(lq.scatter(-1, ids[at], -math.inf), -1, keepdim=True)
        lq = torch.cat([lq.gather(-1, ids[at]), others], -1)
        if s["rest"] is None:
            if kind == "jsd":  # the bucket of the others: no teacher mass there
                extra = -(1.0 - beta) * torch.exp(others.squeeze(-1)) * math.log(1.0 - beta)
            else:
                extra = 0.0
            lq = lq[:, :-1]
        else:
            extra = 0.0
        if kind == "fkl":
            d = (lp.exp() * (lp - lq)).sum(-1)
        elif kind == "rkl":
            d = (lq.exp() * (lq - lp)).sum(-1)
        else:
            lm = torch.log(beta * lp.exp() + (1.0 - beta) * lq.exp())
            d = beta * (lp.exp() * (lp - lm)).sum(-1) + (1.0 - beta) * (lq.exp() * (lq - lm)).sum(-1) + extra
        if case["grad"]:
            grad[at] = torch.autograd.grad(d.sum(), z)[0]
        D[at] = d.detach()
    loss = torch.stack([D.sum() / max(1, int(on.sum())), D.sum()])
    shape = (case["B"], case["K"])
    return [loss, D.view(shape)] + ([grad.view(*shape, V)] if case["grad"] else [])


def _exact_verify(s, case):
    T, K, V = case["T"], case["K"], case["V"]
    B = s["x"].shape[0]
    accepted, tokens, mask = [], [], []
    length = [K] * B if s["len"] is None else s["len"].tolist()
    y, ua, ur = s["tokens"].tolist(), s["ua"].double().tolist(), s["ur"].double().tolist()
    for b in range(B):
        P = torch.softmax(s["x"][b, :length[b] + 1].double() / T, -1)
        Q = torch.zeros(length[b], V, dtype=torch.float64, device=DEV)
        Q.scatter_(-1, s["ids"][b, :length[b]].long(), torch.softmax(s["top"][b, :length[b]].double() / T, -1))
        at = torch.tensor(y[b][:length[b]], device=DEV).unsqueeze(-1)
        p, q = P[:-1].gather(-1, at).squeeze(-1).tolist(), Q.gather(-1, at).squeeze(-1).tolist()
        a = 0
        while a < length[b] and ua[b][a] < (p[a] / q[a] if q[a] > 0 else math.inf):
            a += 1
        mass = (P[a] - Q[a]).clamp_min(0.0) if a < length[b] else P[a]
        edge = mass.cumsum(-1)
        extra = int(torch.searchsorted(edge, edge[-1:] * ur[b], right=True).clamp_max(V - 1))
        accepted.append(a)
        tokens.append(y[b][:a] + [extra] + [-1] * (K - a))
        mask.append([int(i == a and a < length[b]) for i in range(K)])
    return [torch.tensor(accepted, dtype=torch.int32, device=DEV), torch.tensor(tokens, dtype=torch.int32, device=DEV),
            torch.tensor(mask, dtype=torch.uint8, device=DEV)]
