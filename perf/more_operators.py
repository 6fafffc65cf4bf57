"""The operators on a paged KV cache that a program holds itself, as cases that can be timed and compared.

A serving program keeps the keys and values of its sequences in pages.  Every step it appends the step's rows, rotated to
their positions (dream_cache_append), and attends: densely, where the sequences of the batch begin with the same pages, an
image's, say, on which each asks its own question (dream_cache_attn); or, behind a long context, only to the pages that a
bound on their scores selects for each query (dream_cache_select, dream_cache_attn_pages).

Five kinds of case:

  append   rows rotated and written to their pages, with the bounds of pages that become full
  attn     attention of a ragged batch over its sequences, of which the first pages are shared
  select   the pages a query attends to, from the bounds
  pages    attention over given pages
  sparse   select and pages, as a decode step calls them

Keys are N(0, 1) with a drift from page to page, so that pages differ in their scores as they do in a text; queries lean towards one of
them.  Everything is made on the GPU from the seed.

`run` with `own` false is the plain form, in 32 bits; the scores of pages are taken in 64 bits and rounded to 32, because a page's
place in the order changes with the last bit.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
NEG = float("-inf")
THETA = 10000.0
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _model(heads, kv_heads, dim, dtype="bf16", page=64):
    return dict(heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page)


def listed():
    return [
        # one request's next token: latency counts
        dict(name="append one token", op="append", seqs=1, tokens=1, ragged=False, far=2000, rot=128, interleaved=False, bounds=False, **_model(32, 32, 128)),
        # a decode step of a batch far into long contexts, pages filling up
        dict(name="append batch far", op="append", seqs=64, tokens=1, ragged=False, far=120000, rot=128, interleaved=False, bounds=True, **_model(32, 8, 128)),
        # prompts of several requests at once, odd lengths, a part of the head rotated in neighbouring pairs
        dict(name="append prompts", op="append", seqs=5, tokens=1700, ragged=True, far=300, rot=128, interleaved=True, bounds=True, **_model(16, 8, 256)),
        # one sequence, one token, nothing shared: the shortest step
        dict(name="attn one token", op="attn", seqs=1, tokens=1, ragged=False, shared=0, tail=833, tree=False, **_model(32, 32, 128)),
        # questions on one image, answered together
        dict(name="attn questions", op="attn", seqs=32, tokens=1, ragged=True, shared=4352, tail=300, tree=False, **_model(32, 8, 128)),
        # four trees on one image, verified together
        dict(name="attn trees", op="attn", seqs=4, tokens=61, ragged=False, shared=576, tail=400, tree=True, **_model(32, 32, 128)),
        # the questions themselves, of odd lengths, run through behind the prefix
        dict(name="attn prompts", op="attn", seqs=7, tokens=500, ragged=True, shared=4096, tail=700, tree=False, **_model(16, 8, 256)),
        # a large batch behind a long document
        dict(name="attn long", op="attn", seqs=128, tokens=1, ragged=True, shared=32768, tail=1000, tree=False, **_model(32, 32, 64)),
        # pages for a batch of long contexts
        dict(name="select batch", op="select", seqs=8, tokens=1, context=65536, budget=64, **_model(32, 8, 128)),
        # small pages in an odd context, a few tokens of each sequence
        dict(name="select small pages", op="select", seqs=3, tokens=3, context=30011, budget=100, **_model(16, 8, 256, page=16)),
        # attention over given pages alone
        dict(name="pages batch", op="pages", seqs=24, tokens=1, context=32768, budget=48, **_model(32, 8, 128, dtype="f16")),
        # a decode step of one long request: selection and attention
        dict(name="sparse one token", op="sparse", seqs=1, tokens=1, context=131072, budget=64, **_model(32, 8, 128)),
    ]


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:                                                  # no case larger than the largest of the list
        case = _some_case(rng)
        if all(work(case)[k] <= most[k] for k in most):
            return case


def _some_case(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    heads, kv_heads, dim = rng.choice([(32, 32, 64), (32, 32, 128), (32, 8, 128), (16, 8, 256), (40, 40, 128), (24, 8, 64), (28, 4, 128)])
    m = _model(heads, kv_heads, dim, rng.choice(["bf16", "bf16", "f16"]), rng.choice([16, 32, 64, 64, 128, 256]))
    op = rng.choice(["append", "attn", "attn", "select", "pages", "sparse"])
    if op == "append":
        seqs = spread(1, 64)
        return dict(op=op, seqs=seqs, tokens=spread(1, max(1, 8192 // seqs)), ragged=rng.random() < 0.5, far=spread(1, 120000),
                    rot=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.3, bounds=rng.random() < 0.6, **m)
    if op == "attn":
        seqs, tree = spread(1, 96), rng.random() < 0.25
        tokens = rng.choice([1, 1, spread(1, 61)]) if tree or seqs > 8 else spread(1, 500)
        return dict(op=op, seqs=seqs, tokens=min(tokens, max(1, 3000 // seqs)), ragged=rng.random() < 0.6, shared=rng.choice([0, spread(16, 16384)]),
                    tail=spread(1, 1000), tree=tree, **m)
    seqs = spread(1, 16)
    context = spread(16 * m["page"], min(131072, (1 << 28) // (seqs * kv_heads * dim)))
    return dict(op=op, seqs=seqs, tokens=rng.choice([1, 1, spread(1, 4)]), context=context,
                budget=spread(4, min(256, 16384 // m["page"], context // m["page"] // 2)), **m)


# ---------------------------------------------------------------------------------- what a program has in hand

def _lengths(case):
    """Query tokens of each sequence, as a list: the same for every seed."""
    n, t = case["seqs"], case["tokens"]
    if not case.get("ragged") or t == 1:
        return [t] * n
    r = random.Random(n * 10007 + t)
    return [r.randint(1, t) for _ in range(n)]


def _pools(case, n_pages):
    dt = TYPES[case["dtype"]]
    shape = (n_pages, case["kv_heads"], case["page"], case["dim"])
    return torch.zeros(shape, dtype=dt, device=DEVICE), torch.zeros(shape, dtype=dt, device=DEVICE)


def _fill(case, pool, g, drift):
    step = max(1, (1 << 26) // pool[0].numel())
    for p in range(0, pool.shape[0], step):
        part = pool[p:p + step]
        x = torch.randn(part.shape, generator=g, device=DEVICE)
        if drift:
            x += 0.7 * torch.randn(part.shape[0], part.shape[1], 1, part.shape[3], generator=g, device=DEVICE)
        part.copy_(x)


def _rope_table(n_pos, rot):
    pos = torch.arange(n_pos, dtype=torch.float64, device=DEVICE)[:, None]
    angle = pos * THETA ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=DEVICE) / rot)
    return torch.stack((torch.cos(angle), torch.sin(angle)), 2).float()


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    H, hkv, d, pt, B = case["heads"], case["kv_heads"], case["dim"], case["page"], case["seqs"]
    dt = TYPES[case["dtype"]]
    st = dict(case=case)
    T = _lengths(case)
    rows = sum(T)
    starts = [sum(T[:b]) for b in range(B + 1)]
    seq_of = [b for b in range(B) for _ in range(T[b])]
    if case["op"] == "append":
        # the rows of a fused projection: queries, keys and values side by side
        qkv = torch.randn(rows, H + 2 * hkv, d, generator=g, device=DEVICE).to(dt)
        st["q"], st["k_new"], st["v_new"] = qkv[:, :H], qkv[:, H:H + hkv], qkv[:, H + hkv:]
        first = torch.randint(0, case["far"], (B,), generator=g, device=DEVICE).tolist()
        if T == [1] * B and case["bounds"]:                      # a part of the batch fills a page in this step
            first = [f - f % pt + pt - 1 if b % 4 == 0 else f for b, f in enumerate(first)]
        slots = [first[b] + i for b in range(B) for i in range(T[b])]
        lo = [f // pt for f in first]                            # pages in front of these are not touched and have no memory here
        need = [(first[b] + T[b] - 1) // pt - lo[b] + 1 for b in range(B)]
        n_pages = sum((t + pt - 2) // pt + 1 for t in T)         # the most that these many tokens can lie in
        order = torch.randperm(n_pages, generator=g, device=DEVICE).tolist()
        table = torch.full((B, max(lo[b] + need[b] for b in range(B))), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            table[b, lo[b]:lo[b] + need[b]] = torch.tensor(order[at:at + need[b]], dtype=torch.int32)
            at += need[b]
        st["table"] = table.to(DEVICE)
        st["k"], st["v"] = _pools(case, n_pages)
        _fill(case, st["k"], g, False)
        _fill(case, st["v"], g, False)
        st["bounds"] = torch.zeros(n_pages, hkv, 2, d, dtype=dt, device=DEVICE) if case["bounds"] else None
        st["seq"], st["slots"] = _int(seq_of), _int(slots)
        st["rope"] = _rope_table(max(slots) + 1, case["rot"])
        st["q_out"] = torch.zeros(rows, H, d, dtype=dt, device=DEVICE)
    else:
        if case["op"] == "attn":
            shared = case["shared"] // pt
            tail = torch.randint(1, case["tail"] + 1, (B,), generator=g, device=DEVICE).tolist() if case["ragged"] else [case["tail"]] * B
            length = [shared * pt + max(tail[b], T[b]) for b in range(B)]
        else:
            shared = 0
            length = [max(T[b], case["context"] - b * 7 % max(1, case["context"] // 2)) for b in range(B)]
        need = [(n + pt - 1) // pt - shared for n in length]
        n_pages = shared + sum(need)
        order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
        table = torch.zeros(B, shared + max(need), dtype=torch.int32, device=DEVICE)
        at = shared
        for b in range(B):
            table[b, :shared] = order[:shared]
            table[b, shared:shared + need[b]] = order[at:at + need[b]]
            at += need[b]
        st.update(table=table, shared=shared)
        st["k"], st["v"] = _pools(case, n_pages)
        _fill(case, st["k"], g, True)
        if case["op"] != "select":
            _fill(case, st["v"], g, False)
        # a query leans towards a key of its sequence
        q = torch.randn(rows, H, d, generator=g, device=DEVICE)
        lean = torch.randint(0, n_pages, (rows,), generator=g, device=DEVICE)
        q += 0.5 * st["k"][lean, :, 0].float().repeat_interleave(H // hkv, 1)
        st["q"], st["out"] = q.to(dt), torch.zeros(rows, H, d, dtype=dt, device=DEVICE)
        st["q_start"], st["length"] = _int(starts), _int(length)
        st["seq"], st["at"] = _int(seq_of), _int([length[b] - T[b] + i for b in range(B) for i in range(T[b])])
        st["most"], st["longest"] = max(T), max(length)
        st["tree"] = None
        if case.get("tree"):
            parent = [[-1] + [int(x) for x in (torch.rand(max(0, n - 1), generator=g, device=DEVICE) * torch.arange(1, max(1, n), device=DEVICE)).tolist()] for n in T]
            words = []
            for p in parent:
                sets = []
                for i, up in enumerate(p):
                    sets.append((sets[up] if up >= 0 else 0) | 1 << i)
                words += [[(s >> 32 * w & 0xffffffff) - (1 << 32 if s >> 32 * w + 31 & 1 else 0) for w in range(4)] for s in sets]
            st["tree"] = torch.tensor(words, dtype=torch.int32, device=DEVICE)
        if case["op"] in ("select", "sparse"):
            st["bounds"] = torch.stack((st["k"].amin(2), st["k"].amax(2)), 2)
        if case["op"] != "attn":
            st["ids"] = torch.zeros(rows, hkv, case["budget"], dtype=torch.int32, device=DEVICE)
        if case["op"] == "pages":
            n = torch.div(st["at"], pt, rounding_mode="floor") + 1          # pages of the row's context
            pick = torch.rand(rows, hkv, int(n.max()), generator=g, device=DEVICE)
            page = torch.arange(pick.shape[2], device=DEVICE)
            pick = torch.where(page == n[:, None, None] - 1, 2.0, pick).masked_fill(page >= n[:, None, None], -1.0)
            val, ids = torch.topk(pick, min(case["budget"], pick.shape[2]), 2)
            ids = torch.sort(torch.where(val >= 0, ids, 1 << 30), 2).values
            st["ids"][:, :, :ids.shape[2]] = torch.where(ids < 1 << 30, ids, -1).int()
            st["ids"][:, :, ids.shape[2]:] = -1
    st["scale"] = 1.0 / math.sqrt(d)
    if own:
        from paper_2505_19201_b200 import api
        st["cache"] = api.Cache(st["k"], st["v"], st["table"], st.get("bounds"))
        if case["op"] != "append":
            need = [api.dream_cache_attn_bytes(st["cache"], rows, H)]
            if st.get("bounds") is not None:
                need.append(api.dream_cache_select_bytes(st["cache"], rows))
            st["workspace"] = torch.empty(max(need), dtype=torch.uint8, device=DEVICE)
    return st


# ---------------------------------------------------------------------------------- the framework's calls

def _run_own(st):
    from paper_2505_19201_b200 import api
    op = st["case"]["op"]
    if op == "append":
        api.dream_cache_append(st["cache"], st["q"], st["k_new"], st["v_new"], st["seq"], st["slots"], st["q_out"], rope=st["rope"],
                               interleaved=st["case"]["interleaved"])
        return [st[k] for k in ("q_out", "k", "v", "bounds") if st[k] is not None]
    if op == "attn":
        api.dream_cache_attn(st["cache"], st["q"], st["q_start"], st["length"], st["out"], st["workspace"], shared_pages=st["shared"],
                             tree_mask=st["tree"], scale=st["scale"])
        return st["out"]
    if op in ("select", "sparse"):
        api.dream_cache_select(st["cache"], st["q"], st["seq"], st["at"], st["ids"], st["workspace"])
    if op == "select":
        return st["ids"]
    api.dream_cache_attn_pages(st["cache"], st["q"], st["seq"], st["at"], st["ids"], st["out"], st["workspace"], scale=st["scale"])
    return (st["ids"], st["out"]) if op == "sparse" else st["out"]


# ---------------------------------------------------------------------------------- the plain forms

def _turned(x, rope, interleaved):
    """x [rows, heads, dim] rotated in its first channels; rope [rows, rot / 2, 2]."""
    x, rot = x.float(), 2 * rope.shape[1]
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * s, b * c + a * s
    head = torch.stack((ra, rb), 3).flatten(2) if interleaved else torch.cat((ra, rb), 2)
    return torch.cat((head, x[..., rot:]), 2)


def _run_append(st):
    case, pt, dt = st["case"], st["case"]["page"], st["q"].dtype
    seq, slot = st["seq"].long(), st["slots"].long()
    rope = st["rope"][slot]
    st["q_out"].copy_(_turned(st["q"], rope, case["interleaved"]))
    page, off = st["table"][seq, slot // pt].long(), slot % pt
    st["k"][page, :, off] = _turned(st["k_new"], rope, case["interleaved"]).to(dt)
    st["v"][page, :, off] = st["v_new"]
    if case["bounds"]:
        full = page[off == pt - 1]
        st["bounds"][full] = torch.stack((st["k"][full].amin(2), st["k"][full].amax(2)), 2)
    return [st[k] for k in ("q_out", "k", "v", "bounds") if st[k] is not None]


def _run_attn(st):
    """Rows laid out by sequence; scores against the shared pages, once, beside those against each sequence's own."""
    case, pt, H, hkv, d = st["case"], st["case"]["page"], st["case"]["heads"], st["case"]["kv_heads"], st["case"]["dim"]
    start, length, most, P = st["q_start"].long(), st["length"].long(), st["most"], st["shared"] * pt
    B, S = length.shape[0], st["longest"] - P
    T = start[1:] - start[:-1]
    node = torch.arange(most, device=DEVICE)
    row = (start[:-1, None] + node).clamp(max=st["q"].shape[0] - 1)         # [B, most]
    q = st["q"][row].float().view(B, most, hkv, H // hkv, d) * st["scale"]
    own_pages = st["table"][:, st["shared"]:].long()
    key = torch.arange(S, device=DEVICE)
    k = st["k"][own_pages].float().transpose(2, 3).reshape(B, -1, hkv, d)[:, :S]
    v = st["v"][own_pages].float().transpose(2, 3).reshape(B, -1, hkv, d)[:, :S]
    s = torch.einsum("btkgd,bskd->bkgts", q, k)
    base = length - T
    seen = P + key[None, None] <= (base[:, None] + node)[:, :, None]
    if st["tree"] is not None:
        i = (P + key[None] - base[:, None]).clamp(0, 127)                   # place of a key among the tree's nodes
        bits = torch.gather(st["tree"][row].long(), 2, (i // 32)[:, None].expand(B, most, S)) >> (i % 32)[:, None] & 1
        seen = seen & ((P + key[None] < base[:, None])[:, None] | (bits == 1))
    s = s.masked_fill(~seen[:, None, None], NEG)
    if P:
        pre = st["table"][0, :st["shared"]].long()
        kp = st["k"][pre].float().transpose(0, 1).reshape(hkv, P, d)
        vp = st["v"][pre].float().transpose(0, 1).reshape(hkv, P, d)
        s = torch.cat((torch.einsum("btkgd,kpd->bkgtp", q, kp), s), 4)
    s = torch.exp(s - s.amax(4, keepdim=True))
    s = s / s.sum(4, keepdim=True)
    o = torch.einsum("bkgts,bskd->btkgd", s[..., P:], v)
    if P:
        o = o + torch.einsum("bkgtp,kpd->btkgd", s[..., :P], vp)
    st["out"][row[node[None] < T[:, None]]] = o[node[None] < T[:, None]].flatten(1, 2).to(st["out"].dtype)
    return st["out"]


def _run_select(st):
    case, pt, H, hkv, d = st["case"], st["case"]["page"], st["case"]["heads"], st["case"]["kv_heads"], st["case"]["dim"]
    R, budget = st["q"].shape[0], case["budget"]
    seq = st["seq"].long()
    last = torch.div(st["at"].long(), pt, rounding_mode="floor")             # the query's own page
    n = st["table"].shape[1]
    page = torch.arange(n, device=DEVICE)
    score = torch.empty(R, hkv, n, device=DEVICE)
    step = max(1, (1 << 27) // (n * hkv * d))
    for r in range(0, R, step):                                              # a few rows at a time: the bounds in 64 bits are large
        q = st["q"][r:r + step].double().view(-1, hkv, H // hkv, d)
        lo, hi = st["bounds"][st["table"][seq[r:r + step]].long()].double().unbind(3)
        s = torch.einsum("rkgd,rpkd->rkgp", q.clamp(min=0), hi) + torch.einsum("rkgd,rpkd->rkgp", q.clamp(max=0), lo)
        score[r:r + step] = s.amax(2).float()
    kept = (page[None] < 1) | (page[None] == last[:, None])
    score = score.masked_fill(kept[:, None], float("inf")).masked_fill((page[None] > last[:, None])[:, None], NEG)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :budget]
    ids = torch.where(order <= last[:, None, None], order, n)
    ids = torch.sort(ids, 2).values
    st["ids"].fill_(-1)
    st["ids"][:, :, :ids.shape[2]] = torch.where(ids < n, ids, -1).int()
    return st["ids"]


def _run_pages(st):
    case, pt, H, hkv, d = st["case"], st["case"]["page"], st["case"]["heads"], st["case"]["kv_heads"], st["case"]["dim"]
    R = st["q"].shape[0]
    ids = st["ids"].long()
    page = st["table"].long()[st["seq"].long()[:, None, None], ids.clamp(min=0)]             # [R, hkv, budget]
    head = torch.arange(hkv, device=DEVICE)[None, :, None]
    k, v = st["k"][page, head].float(), st["v"][page, head].float()                           # [R, hkv, budget, pt, d]
    q = st["q"].float().view(R, hkv, H // hkv, d) * st["scale"]
    at = ids[..., None] * pt + torch.arange(pt, device=DEVICE)
    seen = (ids[..., None] >= 0) & (at <= st["at"].long()[:, None, None, None])
    s = torch.einsum("rkgd,rkbpd->rkgbp", q, k).masked_fill(~seen[:, :, None], NEG).flatten(3)
    s = torch.exp(s - s.amax(3, keepdim=True))
    s = s / s.sum(3, keepdim=True)
    st["out"].copy_(torch.einsum("rkgs,rksd->rkgd", s, v.flatten(2, 3)).flatten(1, 2))
    return st["out"]


def run(st):
    if own:
        return _run_own(st)
    if st["case"]["op"] == "sparse":
        ids = _run_select(st)
        return ids, _run_pages(st)
    return {"append": _run_append, "attn": _run_attn, "select": _run_select, "pages": _run_pages}[st["case"]["op"]](st)


def work(case):
    H, hkv, d, pt, B = case["heads"], case["kv_heads"], case["dim"], case["page"], case["seqs"]
    rows = sum(_lengths(case))
    T = rows / B
    kv = 4 * hkv * d                                              # bytes of a token's key and value
    if case["op"] == "append":
        pairs = rows * (H + hkv) * case["rot"] / 2
        return {"bytes": rows * (4 * H * d + 2 * kv + 4 * case["rot"] + 8), "flops": 6 * pairs}
    if case["op"] == "attn":
        P = case["shared"] // pt * pt
        tail = max(T, (case["tail"] + 1) / 2 if case["ragged"] else case["tail"])
        return {"bytes": (P + B * tail) * kv + 4 * rows * H * d, "flops": 4 * d * H * rows * (P + tail - T / 2)}
    n = (case["context"] + pt - 1) // pt
    some = min(case["budget"], n)
    select = {"bytes": B * n * hkv * 4 * d + rows * (2 * H * d + 4 * hkv * some), "flops": 2 * d * H * rows * n}
    pages = {"bytes": rows * (hkv * some * (pt * 4 * d + 4) + 4 * H * d), "flops": 4 * d * H * rows * some * pt}
    if case["op"] == "sparse":
        return {k: select[k] + pages[k] for k in select}
    return select if case["op"] == "select" else pages


# ---------------------------------------------------------------------------------- from the definitions, in 64 bits

def _exact_append(case, st):
    pt, dt, out = case["page"], TYPES[case["dtype"]], []
    slot = st["slots"].double()
    angle = slot[:, None] * torch.exp(-math.log(THETA) * 2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEVICE) / case["rot"])
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    rot = case["rot"]

    def turned(x):
        x = x.double().clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x
    out.append(turned(st["q"]))
    k, v = st["k"].double(), st["v"].double()
    keys = turned(st["k_new"])
    page = st["table"][st["seq"].long(), st["slots"].long() // pt].long()
    k[page, :, st["slots"].long() % pt] = keys
    v[page, :, st["slots"].long() % pt] = st["v_new"].double()
    out += [k, v]
    if case["bounds"]:
        bounds = st["bounds"].double()
        for r in range(len(page)):
            if int(st["slots"][r]) % pt == pt - 1:
                bounds[page[r]] = torch.stack((k[page[r]].amin(1), k[page[r]].amax(1)), 1)
        out.append(bounds)
    return out


def _context(st, b, n, pt):
    """Keys and values of the first n tokens of sequence b, [kv heads, n, dim] in 64 bits."""
    pages = st["table"][b, :(n + pt - 1) // pt].long()
    return [torch.cat(list(st[x][pages].double()), 1)[:, :n] for x in ("k", "v")]


def _exact_attn(case, st):
    G, pt = case["heads"] // case["kv_heads"], case["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    starts, lengths = st["q_start"].tolist(), st["length"].tolist()
    for b, n in enumerate(lengths):
        k, v = _context(st, b, n, pt)
        T = starts[b + 1] - starts[b]
        step = max(1, (1 << 26) // (n * case["heads"]))
        for i0 in range(0, T, step):
            nodes = range(i0, min(T, i0 + step))
            seen = torch.zeros(len(nodes), n, dtype=torch.bool, device=DEVICE)
            for i in nodes:
                if st["tree"] is None:
                    seen[i - i0, :n - T + i + 1] = True
                else:
                    seen[i - i0, :n - T] = True
                    words = [w & 0xffffffff for w in st["tree"][starts[b] + i].tolist()]
                    for j in range(T):
                        if words[j // 32] >> j % 32 & 1:
                            seen[i - i0, n - T + j] = True
            q = st["q"][starts[b] + i0:starts[b] + i0 + len(nodes)].double()
            kk, vv = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
            s = torch.matmul(q.transpose(0, 1), kk.transpose(1, 2)) / math.sqrt(case["dim"])
            p = torch.softmax(torch.where(seen, s, torch.full_like(s, NEG)), 2)
            out[starts[b] + i0:starts[b] + i0 + len(nodes)] = torch.matmul(p, vv).transpose(0, 1)
    return out


def _exact_pages(case, st, ids):
    G, pt, d = case["heads"] // case["kv_heads"], case["page"], case["dim"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEVICE)
    seqs, at = st["seq"].tolist(), st["at"].tolist()
    for r in range(len(seqs)):
        for h in range(case["kv_heads"]):
            some = ids[r, h][ids[r, h] >= 0].long()
            where = (some[:, None] * pt + torch.arange(pt, device=DEVICE)).flatten()
            pages = st["table"][seqs[r]][some].long()
            k, v = st["k"][pages, h].double().reshape(-1, d), st["v"][pages, h].double().reshape(-1, d)
            q = st["q"][r, h * G:(h + 1) * G].double()
            s = torch.where(where <= at[r], q @ k.T / math.sqrt(d), torch.tensor(NEG, dtype=torch.float64, device=DEVICE))
            out[r, h * G:(h + 1) * G] = torch.softmax(s, 1) @ v
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, st)
    if case["op"] == "attn":
        return _exact_attn(case, st)
    if case["op"] == "select":
        return None
    if case["op"] == "pages":
        return _exact_pages(case, st, st["ids"])
    return None, _exact_pages(case, st, _run_select(st))
