"""The operators on rows of logits, as cases that can be timed and compared.

A verification leaves a row of logits per tree node.  To answer, a program draws a token from a row
(dream_sample) or cuts the rows of a tree to their likely tokens before the acceptance draws from them
(dream_truncate_logits).  To train a draft it holds the draft's rows against the target's top logits
(dream_distill_loss, with the gradient in the same pass or by dream_distill_grad).

Five kinds of case:

  sample    a token per row: temperature, top-k, top-p and min-p by row, one uniform number a row
  truncate  the rows with everything outside the kept tokens at -inf
  loss      the forward pass of the distillation
  grad      its backward pass from the saved log-sum-exp
  step      both in one call

Logits are N(0, 2) with some forty tokens per row raised by up to 14, a shape between a model that is sure of
its next word and one that has hundreds to choose from.  The student's logits are the teacher's, scaled and with noise.
Everything is made on the GPU from the seed.

`run` with `own` false is the plain form.  Masses of the sampling are taken in 64 bits, because a token changes when a
running sum passes a border; the distillation is in 32 bits, with the few numbers per row in 64.
"""
import torch

own = False

DEVICE = "cuda:0"
NEG = float("-inf")


def _sampling(name, op, rows, vocab, dtype="f32", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, pad=0):
    return dict(name=name, op=op, rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k, top_p=top_p,
                min_p=min_p, mixed=mixed, pad=pad)


def _distill(name, op, rows, vocab, dtype="bf16", top=16, tail=False, temperature=1.0, masked=False, pad=0):
    return dict(name=name, op=op, rows=rows, vocab=vocab, dtype=dtype, top=top, tail=tail, temperature=temperature, masked=masked,
                pad=pad)


def listed():
    return [
        # one request's next token with the usual settings: latency counts
        _sampling("sample one row", "sample", 1, 32000, temperature=0.7, top_k=50, top_p=0.9),
        # eight requests, the widest vocabulary, nucleus only: the mass of the whole row decides
        _sampling("sample wide nucleus", "sample", 8, 262144, top_p=0.95),
        # a batch whose requests each bring their own settings, odd vocabulary, bf16 rows
        _sampling("sample mixed bf16", "sample", 61, 32003, dtype="bf16", mixed=True),
        # a large batch at a temperature and nothing else
        _sampling("sample temperature", "sample", 256, 131072, temperature=0.8),
        # the rows of one tree before the acceptance draws from them
        _sampling("truncate tree", "truncate", 61, 32000, temperature=0.8, top_k=40, top_p=0.95),
        # four trees over a wide vocabulary, rows padded to another stride
        _sampling("truncate four trees", "truncate", 244, 131072, temperature=1.0, top_p=0.9, min_p=0.002, pad=64),
        # distillation: a short answer's rows
        _distill("loss short", "loss", 256, 32000, top=8),
        # evaluation over fp32 rows, the rest of the vocabulary as a bucket
        _distill("loss wide tail", "loss", 1000, 131072, dtype="f32", top=64, tail=True, temperature=2.0),
        # the backward pass alone, some rows being padding
        _distill("grad", "grad", 2048, 32000, top=16, masked=True),
        # odd vocabulary in fp32: no row but the first starts on a 16-byte boundary
        _distill("grad odd tail", "grad", 777, 49155, dtype="f32", top=100, tail=True),
        # a training step's rows, loss and gradient together
        _distill("step", "step", 4096, 32000, top=16, tail=True, masked=True),
        # the same over the widest vocabulary
        _distill("step wide", "step", 1024, 262144, top=64, temperature=2.0),
    ]


def draw(rng):
    import math
    op = rng.choice(["sample", "sample", "truncate", "loss", "grad", "step"])
    vocab = int(round(math.exp(rng.uniform(math.log(500), math.log(262144)))))
    if rng.random() < 0.5:
        vocab = max(504, vocab // 8 * 8)
    most = min(4096 if op in ("loss", "grad", "step") else 256, (1 << 27) // vocab)
    rows = int(round(math.exp(rng.uniform(0.0, math.log(most)))))
    dtype, pad = rng.choice(["f32", "bf16"]), rng.choice([0, 0, 8, rng.randrange(1, 64)])
    if op in ("sample", "truncate"):
        return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, temperature=round(rng.uniform(0.3, 1.5), 3),
                    top_k=rng.choice([0, 0, rng.randrange(1, 100), rng.randrange(100, vocab)]), top_p=rng.choice([1.0, 0.9, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 4)]), mixed=rng.random() < 0.3, pad=pad)
    return dict(op=op, rows=rows, vocab=vocab, dtype=dtype, top=rng.randrange(1, 129), tail=rng.random() < 0.5,
                temperature=rng.choice([1.0, 2.0, round(rng.uniform(0.7, 4.0), 3)]), masked=rng.random() < 0.4, pad=pad)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _room(case):
    """[rows, vocab] with rows `pad` elements further apart than they are long."""
    full = torch.empty(case["rows"], case["vocab"] + case["pad"], dtype=_type(case), device=DEVICE)
    return full[:, :case["vocab"]]


def _model_rows(n, vocab, g):
    x = torch.randn(n, vocab, generator=g, device=DEVICE) * 2.0
    part = vocab // 40                                      # one raised token in each fortieth: none is raised twice
    at = torch.randint(0, part, (n, 40), generator=g, device=DEVICE) + torch.arange(40, device=DEVICE) * part
    return x.scatter_add_(1, at, torch.rand(n, 40, generator=g, device=DEVICE) * 14.0)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    R, V = case["rows"], case["vocab"]
    st = dict(case=case, logits=_room(case))
    step = max(1, (1 << 26) // V)
    if case["op"] in ("sample", "truncate"):
        for r in range(0, R, step):
            st["logits"][r:r + step] = _model_rows(min(step, R - r), V, g)
        if case["mixed"]:
            pick = lambda vals, kind: torch.tensor(vals, dtype=kind, device=DEVICE)[torch.randint(0, len(vals), (R,), generator=g, device=DEVICE)]  # noqa: E731
            st["temperature"] = pick([0.0, 0.5, 0.7, 1.0, 1.3], torch.float32)
            st["top_k"] = pick([0, 1, 20, 50, min(V, 1000)], torch.int32)
            st["top_p"] = pick([1.0, 0.8, 0.95], torch.float32)
            st["min_p"] = pick([0.0, 0.02, 0.1], torch.float32)
        else:                                               # what a batch does not use it does not pass
            full = lambda v, kind: torch.full((R,), v, dtype=kind, device=DEVICE)  # noqa: E731
            st["temperature"] = full(case["temperature"], torch.float32) if case["temperature"] != 1.0 else None
            st["top_k"] = full(case["top_k"], torch.int32) if case["top_k"] else None
            st["top_p"] = full(case["top_p"], torch.float32) if case["top_p"] < 1.0 else None
            st["min_p"] = full(case["min_p"], torch.float32) if case["min_p"] > 0.0 else None
        st["kept"] = torch.zeros(R, dtype=torch.int32, device=DEVICE)
        if case["op"] == "sample":
            st["uniforms"] = torch.rand(R, generator=g, device=DEVICE)
            st["tokens"], st["logprob"] = torch.zeros(R, dtype=torch.int32, device=DEVICE), torch.zeros(R, device=DEVICE)
        else:
            st["out"] = _room(case)
        return st
    K, tau = min(case["top"], V), case["temperature"]
    st["ids"] = torch.empty(R, K, dtype=torch.int32, device=DEVICE)
    st["top"] = torch.empty(R, K, device=DEVICE)
    st["teacher_lse"] = torch.empty(R, device=DEVICE) if case["tail"] else None
    for r in range(0, R, step):
        x = _model_rows(min(step, R - r), V, g)
        t, i = torch.topk(x, K, dim=1)
        st["top"][r:r + step], st["ids"][r:r + step] = t, i.int()
        if case["tail"]:
            st["teacher_lse"][r:r + step] = torch.logsumexp(x.double() / tau, 1).float()
        st["logits"][r:r + step] = x * 0.9 + torch.randn(x.shape, generator=g, device=DEVICE) * 0.7
    # what reaches a row from the batch's mean loss; rows of padding get nothing
    st["row_scale"] = torch.rand(R, generator=g, device=DEVICE) + 0.5
    if case["masked"]:
        st["row_scale"] *= (torch.rand(R, generator=g, device=DEVICE) < 0.8).float()
    st["loss"], st["lse"] = torch.zeros(R, device=DEVICE), torch.zeros(R, device=DEVICE)
    st["log_rest"] = torch.zeros(R, device=DEVICE) if case["tail"] else None
    if case["op"] == "grad":
        for r in range(0, R, step):
            z = st["logits"][r:r + step].double() / tau
            st["lse"][r:r + step] = torch.logsumexp(z, 1).float()
            if case["tail"]:
                z = z.scatter(1, st["ids"][r:r + step].long(), NEG)
                st["log_rest"][r:r + step] = (torch.logsumexp(z, 1) - st["lse"][r:r + step].double()).float()
    if case["op"] != "loss":
        st["grad"] = _room(case)
    return st


# ---------------------------------------------------------------------------------- the framework's calls

def _run_own(st):
    from paper_2505_19201_b200 import api
    case = st["case"]
    if case["op"] == "sample":
        api.dream_sample(st["logits"], st["uniforms"], st["tokens"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                         min_p=st["min_p"], logprob=st["logprob"], kept=st["kept"])
        return st["tokens"], st["logprob"], st["kept"]
    if case["op"] == "truncate":
        api.dream_truncate_logits(st["logits"], st["out"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                                  min_p=st["min_p"], kept=st["kept"])
        return st["out"], st["kept"]
    if case["op"] == "grad":
        api.dream_distill_grad(st["logits"], st["ids"], st["top"], st["lse"], st["grad"], teacher_lse=st["teacher_lse"],
                               log_rest=st["log_rest"], temperature=case["temperature"], row_scale=st["row_scale"])
        return st["grad"]
    grad = dict(grad=st["grad"], row_scale=st["row_scale"]) if case["op"] == "step" else {}
    api.dream_distill_loss(st["logits"], st["ids"], st["top"], st["loss"], st["lse"], teacher_lse=st["teacher_lse"],
                           log_rest=st["log_rest"], temperature=case["temperature"], **grad)
    return [st[k] for k in ("loss", "lse", "log_rest", "grad") if st.get(k) is not None]


# ---------------------------------------------------------------------------------- the plain forms

def _masses(st):
    """Weights relative to the best token [R][V] and which tokens stay, in 64 bits."""
    x = st["logits"].float()
    R, V = x.shape
    greedy = torch.zeros(R, 1, dtype=torch.bool, device=x.device)
    d = x.double() - x.amax(1, keepdim=True).double()
    if st["temperature"] is not None:
        t = st["temperature"].double()[:, None]
        greedy = ~(t > 0)
        d = d / torch.where(greedy, torch.ones_like(t), t)
    w = torch.exp(d)
    if st["temperature"] is None and st["top_k"] is None and st["top_p"] is None and st["min_p"] is None:
        return w, x > NEG
    if st["top_k"] is None and st["top_p"] is None and st["min_p"] is None and not st["case"]["mixed"]:
        return w, x > NEG                                   # cases without mixed rows have temperatures above zero
    order = torch.sort(x, dim=1, descending=True, stable=True).indices     # ties: the lower id first
    ws = torch.gather(w, 1, order)
    rank = torch.arange(V, device=x.device)[None, :]
    k = torch.full((R, 1), V, device=x.device) if st["top_k"] is None else st["top_k"].long()[:, None]
    k = torch.where(greedy, torch.ones_like(k), torch.where(k > 0, k, torch.full_like(k, V)))
    keep = rank < k
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        run = torch.cumsum(ws, 1)
        total = torch.gather(run, 1, k.clamp(max=V) - 1)
        keep = keep & ((run - ws < p * total) | (p >= 1))
    if st["min_p"] is not None:
        keep = keep & (ws >= st["min_p"].double()[:, None])
    keep = keep | (rank == 0)
    stay = torch.zeros_like(keep).scatter(1, order, keep)
    return w, stay & (x > NEG)


def _run_sample(st):
    w, stay = _masses(st)
    mass = torch.where(stay, w, torch.zeros_like(w))
    run = torch.cumsum(mass, 1)
    total = run[:, -1:]
    token = (run <= st["uniforms"].double()[:, None] * total).sum(1, keepdim=True)
    token = token.clamp(max=w.shape[1] - 1)
    logprob = torch.log(torch.gather(mass, 1, token) / total)
    return token[:, 0].int(), logprob[:, 0].float(), stay.sum(1).int()


def _run_truncate(st):
    _, stay = _masses(st)
    x = st["logits"]
    return torch.where(stay, x, torch.full_like(x, NEG)), stay.sum(1).int()


def _teacher(st):
    """The teacher's probabilities of its top tokens [R][K] and of the rest [R], in 64 bits."""
    t = st["top"].double() / st["case"]["temperature"]
    if st["teacher_lse"] is None:
        e = torch.exp(t - t.amax(1, keepdim=True))
        return e / e.sum(1, keepdim=True), torch.zeros(t.shape[0], dtype=torch.float64, device=t.device)
    q = torch.exp(t - st["teacher_lse"].double()[:, None])
    return q, (1.0 - q.sum(1)).clamp(min=0.0)


def _run_loss(st):
    tail, ids = st["teacher_lse"] is not None, st["ids"].long()
    z = st["logits"].float() / st["case"]["temperature"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    lse = torch.log(e.sum(1, dtype=torch.float64)) + m[:, 0].double()
    q, qr = _teacher(st)
    loss = (q * (torch.log(q.clamp(min=1e-300)) - torch.gather(z, 1, ids).double() + lse[:, None])).sum(1)
    out = [loss, lse]
    if tail:
        log_rest = torch.log(e.scatter(1, ids, 0.0).sum(1, dtype=torch.float64)) + m[:, 0].double() - lse
        out[0] = loss + qr * (torch.log(qr.clamp(min=1e-300)) - log_rest)
        out.append(log_rest)
    out = [v.float() for v in out]
    if st["case"]["op"] == "step":
        out.append(_gradient(st, z, lse, out[2].double() if tail else None, q, qr))
    return out


def _gradient(st, z, lse, log_rest, q, qr):
    ids, total = st["ids"].long(), q.sum(1) + qr
    scale = (st["row_scale"].double() / st["case"]["temperature"])[:, None]
    rest = total if log_rest is None else total - qr * torch.exp(-log_rest)
    p = torch.exp(z - lse.float()[:, None])
    top = scale * (total[:, None] * torch.exp(torch.gather(z, 1, ids).double() - lse[:, None]) - q)
    g = p * (scale * rest[:, None]).float()
    return g.scatter(1, ids, top.float()).to(st["logits"].dtype)


def _run_grad(st):
    z = st["logits"].float() / st["case"]["temperature"]
    q, qr = _teacher(st)
    return _gradient(st, z, st["lse"].double(), None if st["log_rest"] is None else st["log_rest"].double(), q, qr)


def run(st):
    if own:
        return _run_own(st)
    return {"sample": _run_sample, "truncate": _run_truncate, "loss": _run_loss, "step": _run_loss, "grad": _run_grad}[st["case"]["op"]](st)


def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    n = case["rows"] * case["vocab"]
    passes = 2 if case["op"] in ("truncate", "grad", "step") else 1
    side = case["rows"] * (28 if case["op"] in ("sample", "truncate") else 8 * case["top"] + 20)
    # a subtraction, a scaling, an exponential and an addition per token, and a product and a rounding where there is a gradient
    return {"bytes": passes * n * esz + side, "flops": n * (6 if case["op"] in ("grad", "step") else 4)}


# ---------------------------------------------------------------------------------- from the definitions, in 64 bits

def _exact_row(x, t, k, p, mp):
    """Ids of the tokens that stay, and every token's probability at temperature t (x, float64)."""
    if not t > 0:
        t, k = 1.0, 1
    prob = torch.softmax(x / t, 0)
    ranked = sorted_ids = torch.sort(x, descending=True, stable=True).indices
    if 0 < k < x.numel():
        ranked = sorted_ids[:k]
    n = ranked.numel()
    if p < 1:
        share = torch.cumsum(prob[ranked], 0) / prob[ranked].sum()          # token r stays while those before it hold less than p
        n = min(n, 1 + int((share[:-1] < p).sum()))
    if mp > 0:
        n = min(n, max(1, int((prob[ranked] >= mp * prob[sorted_ids[0]]).sum())))
    return ranked[:n], prob


def _exact_sampling(case, st):
    at = lambda name, r, off: off if st[name] is None else st[name][r].item()  # noqa: E731
    tokens, logprob, kept = [], [], []
    out = torch.full((case["rows"], case["vocab"]), NEG, dtype=torch.float64, device=DEVICE) if case["op"] == "truncate" else None
    for r in range(case["rows"]):
        x = st["logits"][r].double()
        ids, prob = _exact_row(x, at("temperature", r, 1.0), at("top_k", r, 0), at("top_p", r, 1.0), at("min_p", r, 0.0))
        kept.append(ids.numel())
        if out is not None:
            out[r, ids] = x[ids]
            continue
        ids = torch.sort(ids).values
        share = prob[ids] / prob[ids].sum()
        n = int((torch.cumsum(share, 0) <= st["uniforms"][r].double()).sum())
        n = min(n, ids.numel() - 1)
        tokens.append(int(ids[n]))
        logprob.append(float(torch.log(share[n])))
    kept = torch.tensor(kept, dtype=torch.int32)
    if out is not None:
        return out, kept
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprob, dtype=torch.float64), kept


def _exact_distill(case, st):
    tau, step = case["temperature"], max(1, (1 << 25) // case["vocab"])
    got = {k: [] for k in ("loss", "lse", "log_rest", "grad")}
    for r in range(0, case["rows"], step):
        s = slice(r, r + step)
        ids = st["ids"][s].long()
        logp = torch.log_softmax(st["logits"][s].double() / tau, 1)
        lse = torch.logsumexp(st["logits"][s].double() / tau, 1)
        if case["op"] == "grad":                            # the saved values are inputs
            logp, lse = st["logits"][s].double() / tau - st["lse"][s].double()[:, None], st["lse"][s].double()
        t = st["top"][s].double() / tau
        q = torch.softmax(t, 1) if not case["tail"] else torch.exp(t - st["teacher_lse"][s].double()[:, None])
        log_top = torch.gather(logp, 1, ids)
        loss = torch.special.xlogy(q, q).sum(1) - (q * log_top).sum(1)
        target = torch.zeros_like(logp).scatter_(1, ids, q)
        prob, total = torch.exp(logp), q.sum(1, keepdim=True)
        if case["tail"]:
            qr = (1.0 - q.sum(1)).clamp(min=0.0)
            others = logp.scatter(1, ids, NEG)
            log_rest = torch.logsumexp(others, 1) if case["op"] != "grad" else st["log_rest"][s].double()
            loss = loss + torch.special.xlogy(qr, qr) - qr * log_rest
            got["log_rest"].append(log_rest)
            target += torch.exp(others - log_rest[:, None]) * qr[:, None]
            total = total + qr[:, None]
        got["loss"].append(loss)
        got["lse"].append(lse)
        if case["op"] != "loss":
            got["grad"].append(((total * prob - target) * (st["row_scale"][s].double() / tau)[:, None]).float())
    got = {k: torch.cat(v) for k, v in got.items() if v}
    if case["op"] == "grad":
        return got["grad"]
    return [got[k] for k in ("loss", "lse", "log_rest", "grad") if k in got]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("sample", "truncate"):
        return _exact_sampling(case, st)
    return _exact_distill(case, st)
