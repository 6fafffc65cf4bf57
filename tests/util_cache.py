"""A small paged cache for tests, and what the calls on it mean, in 64 bits and token by token of the definition."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}                 # half a step, relative
NAN = float("nan")


def pools(n_pages, hkv, pt, d, dtype, layout="hnd", dev="cuda"):
    """K and V full of NaN: [page, head, token, d], or views of that shape into another order or with room between pages."""
    def one():
        if layout == "nhd":
            return torch.full((n_pages, pt, hkv, d), NAN, dtype=TYPES[dtype], device=dev).permute(0, 2, 1, 3)
        if layout == "room":
            return torch.full((n_pages, hkv + 1, pt, d + 8), NAN, dtype=TYPES[dtype], device=dev)[:, :hkv, :, :d]
        if layout == "heads":                                  # head after head
            return torch.full((hkv, n_pages, pt, d), NAN, dtype=TYPES[dtype], device=dev).permute(1, 0, 2, 3)
        return torch.full((n_pages, hkv, pt, d), NAN, dtype=TYPES[dtype], device=dev)
    return one(), one()


class Pages:
    """Sequences of the given lengths, the first `shared` pages common to all, in shuffled pages; everything else in the pools is NaN."""

    def __init__(self, lengths, hkv, d, pt, dtype="bf16", shared=0, layout="hnd", seed=0, spare=2, extra_entries=1, gain=1.0):
        from paper_2505_19201_b200 import api
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        need = [max(0, (n + pt - 1) // pt - shared) for n in lengths]
        n_pages = shared + sum(need) + spare
        order = torch.randperm(n_pages, generator=g, device="cuda").int()
        self.k, self.v = pools(n_pages, hkv, pt, d, dtype, layout)
        width = shared + max(need + [0]) + extra_entries
        self.table = torch.full((len(lengths), width), -7, dtype=torch.int32, device="cuda")      # entries behind the end are not looked at
        at = shared
        for b, n in enumerate(lengths):
            self.table[b, :shared] = order[:shared]
            self.table[b, shared:shared + need[b]] = order[at:at + need[b]]
            at += need[b]
        for b, n in enumerate(lengths):
            for j in range((n + pt - 1) // pt):
                m = min(pt, n - j * pt)
                page = int(self.table[b, j])
                if j < shared and b > 0 and not torch.isnan(self.k[page, 0, m - 1, 0]):
                    continue
                self.k[page, :, :m] = (gain * torch.randn(hkv, m, d, generator=g, device="cuda") + torch.randn(hkv, 1, d, generator=g, device="cuda") * 0.5).to(self.k.dtype)
                self.v[page, :, :m] = torch.randn(hkv, m, d, generator=g, device="cuda").to(self.k.dtype)
        self.lengths, self.hkv, self.d, self.pt, self.shared, self.dtype = lengths, hkv, d, pt, shared, dtype
        self.cache = api.Cache(self.k, self.v, self.table)

    def context(self, b, tokens):
        """K and V of these tokens (a list or tensor of numbers) of sequence b: [hkv, n, d] in 64 bits."""
        t = torch.as_tensor(tokens, device="cuda").long()
        page = self.table[b].long()[t // self.pt]
        return self.k[page, :, t % self.pt].transpose(0, 1).double(), self.v[page, :, t % self.pt].transpose(0, 1).double()

    def queries(self, rows, heads, gain=1.0):
        return (gain * torch.randn(rows, heads, self.d, generator=self.g, device="cuda")).to(self.k.dtype)


def attend(q, k, v, seen, scale):
    """q [n, H, d], k and v [hkv, m, d], seen [n, m] or [hkv, n, m] -> out [n, H, d], lse [n, H], sum of weights times |v| [n, H, d]."""
    n, H, d = q.shape
    hkv = k.shape[0]
    G = H // hkv
    out = torch.zeros(n, H, d, dtype=torch.float64, device=q.device)
    size, lse = out.clone(), torch.full((n, H), -math.inf, dtype=torch.float64, device=q.device)
    if k.shape[1] == 0:
        return out, lse, size
    for h in range(hkv):
        s = torch.einsum("ngd,md->ngm", q[:, h * G:(h + 1) * G].double(), k[h]) * scale
        m = seen if seen.dim() == 2 else seen[h]
        s = s.masked_fill(~m[:, None], -math.inf)
        lse[:, h * G:(h + 1) * G] = torch.logsumexp(s, 2)
        p = torch.where(m.any(1)[:, None, None], torch.softmax(s, 2), torch.zeros_like(s)).nan_to_num(0.0)
        out[:, h * G:(h + 1) * G] = p @ v[h]
        size[:, h * G:(h + 1) * G] = p @ v[h].abs()
    return out, lse, size


def dense_reference(pg, q, q_start, tree=None, scale=None):
    scale = pg.d ** -0.5 if scale is None else scale
    outs, lses, sizes = [], [], []
    for b, n in enumerate(pg.lengths):
        T = q_start[b + 1] - q_start[b]
        k, v = pg.context(b, range(n))
        at = torch.arange(n, device="cuda")[None]
        i = torch.arange(T, device="cuda")[:, None]
        if tree is None:
            seen = at <= n - T + i
        else:
            words = tree[q_start[b]:q_start[b + 1]].long() & 0xffffffff
            j = (at - (n - T)).clamp(0, 127).expand(T, n)
            bit = (torch.gather(words, 1, j // 32) >> (j % 32)) & 1
            seen = (at < n - T) | ((at >= n - T) & (bit == 1))
        o, l, s = attend(q[q_start[b]:q_start[b + 1]], k, v, seen, scale)
        outs.append(o), lses.append(l), sizes.append(s)
    return torch.cat(outs), torch.cat(lses), torch.cat(sizes)


def pages_reference(pg, q, row_seq, row_pos, ids, scale=None):
    scale = pg.d ** -0.5 if scale is None else scale
    R, H, d = q.shape
    G = H // pg.hkv
    out = torch.zeros(R, H, d, dtype=torch.float64, device="cuda")
    lse, size = torch.full((R, H), -math.inf, dtype=torch.float64, device="cuda"), out.clone()
    for r in range(R):
        for h in range(pg.hkv):
            tokens, before = [], -1
            for e, i in enumerate(ids[r, h].tolist()):
                if i >= 0 and i * pg.pt <= row_pos[r] and (e == 0 or i > before):
                    tokens += [t for t in range(i * pg.pt, (i + 1) * pg.pt) if t <= row_pos[r]]
                before = i
            if row_seq[r] < 0 or not tokens:
                continue
            k, v = pg.context(row_seq[r], tokens)
            o, l, s = attend(q[r:r + 1, h * G:(h + 1) * G], k[h:h + 1], v[h:h + 1], torch.ones(1, len(tokens), dtype=torch.bool, device="cuda"), scale)
            out[r, h * G:(h + 1) * G], lse[r, h * G:(h + 1) * G], size[r, h * G:(h + 1) * G] = o[0], l[0], s[0]
    return out, lse, size


def close(out, want, size, dtype, spread=0.0):
    """Every element within its bound.  A weight is rounded to the type once, relative error h (half a step), and the sum that divides is that of the rounded ones:
    the result moves by at most h * sum w |v - out| <= h (size + |out|), and is itself rounded, h |out|.  Scores are sums of up to 256 products in 32
    bits, where every addition may lose 2^-23 of the largest partial sum: below 2^-15 of a score's magnitude, which is a few units here; `spread` is the
    largest such magnitude where it is more.  Results below the smallest normal number of the type have its absolute step."""
    h = HALF[dtype]
    bound = 1.02 * (h * (size + 2 * want.abs()) + 2.0 ** -15 * (8.0 + spread) * (size + want.abs())) + torch.finfo(TYPES[dtype]).tiny
    err = (out.double() - want).abs()
    assert torch.isfinite(out).all()
    assert (err <= bound).all(), f"{(err / bound).max().item()} times the bound"


def close_lse(lse, want, spread=0.0):
    """Weights are off by 2^-15 of the scores' magnitude at most (see close), and so is the logarithm of their sum; its own rounding is 2^-24 of it."""
    dead = torch.isinf(want)
    assert torch.equal(torch.isinf(lse) & (lse < 0), dead)
    err = (lse.double() - want).abs()[~dead]
    assert err.numel() == 0 or (err <= 2.0 ** -15 * (8.0 + spread) + 2.0 ** -22 * want[~dead].abs()).all()


def tree_words(parents):
    """[n][4] int32 ancestor-or-self words of a parent array."""
    sets, words = [], []
    for i, p in enumerate(parents):
        sets.append((sets[p] if p >= 0 else 0) | 1 << i)
        words.append([(sets[i] >> 32 * w & 0xffffffff) - (1 << 32 if sets[i] >> 32 * w + 31 & 1 else 0) for w in range(4)])
    return words
