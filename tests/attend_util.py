"""Attention over a paged cache by its definition in 64 bits, and how far a kernel's fp32 sums and roundings may be from it."""
import math

import torch

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


class Batch:
    """Sequences with random tokens in a paged cache whose other slots hold NaN, tables whose entries past a length name no page.

    own: tokens of each row; prompts: tokens of each prompt (row r has that of r // per), or None."""

    def __init__(self, own, dim, kv_heads, page, dtype, prompts=None, per=1, seed=0, spare=2, room=None, value=1.0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dim, self.kv_heads, self.page, self.dtype, self.per = dim, kv_heads, page, DTYPES[dtype.split()[0]], per
        self.shape = {"16": 1, "128": 2}.get(dtype.split()[-1], 0)
        self.own, self.prompts = list(own), prompts
        both = self.own + (prompts or [])
        need = [-(-n // page) for n in both]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed + 1)).tolist()
        self.lists = []
        for n in need:
            self.lists.append(order[:n])
            order = order[n:]
        shape = (pages, kv_heads, page, dim)
        self.k = torch.full(shape, NAN, dtype=self.dtype, device="cuda")
        self.v = torch.full(shape, NAN, dtype=self.dtype, device="cuda")
        for n, of in zip(both, self.lists):
            for i, p in enumerate(of):
                m = min(page, n - i * page)
                self.k[p, :, :m] = self.random(kv_heads, m, dim)
                self.v[p, :, :m] = value * self.random(kv_heads, m, dim)
        width = max([1] + need[:len(own)]) if room is None else room
        self.table = self._table(self.lists[:len(own)], width)
        self.lens = torch.tensor(self.own, dtype=torch.int32, device="cuda")
        self.prompt_table = self.prompt_lens = None
        if prompts is not None:
            self.prompt_table = self._table(self.lists[len(own):], max([1] + need[len(own):]))
            self.prompt_lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")

    def random(self, *shape):
        return torch.randn(*shape, device="cuda", generator=self.g).to(self.dtype)

    @staticmethod
    def _table(lists, width):
        bad = [-7, 1 << 30, -(1 << 31), 2000000000]
        return torch.tensor([of + [bad[(i + j) % 4] for j in range(width - len(of))] for i, of in enumerate(lists)], dtype=torch.int32, device="cuda")

    def _of(self, cache, i, n):
        of = self.lists[i]
        if not n:
            return torch.zeros(self.kv_heads, 0, self.dim, dtype=torch.float64, device="cuda")
        return cache[of].double().transpose(0, 1).reshape(self.kv_heads, -1, self.dim)[:, :n]

    def tokens(self, r):
        """Keys and values [kv_heads, tokens, dim] of row r, its prompt's and its own."""
        out = []
        for cache in (self.k, self.v):
            own = self._of(cache, r, self.own[r])
            if self.prompts is not None:
                own = torch.cat([self._of(cache, len(self.own) + r // self.per, self.prompts[r // self.per]), own], dim=1)
            out.append(own)
        return out

    def place(self, r, t):
        """(page, slot) of token t of row r."""
        before = 0 if self.prompts is None else self.prompts[r // self.per]
        i, t = (len(self.own) + r // self.per, t) if t < before else (r, t - before)
        return self.lists[i][t // self.page], t % self.page


def seen_by(at, total, window, sinks):
    j = torch.arange(total, device="cuda")
    see = j <= at
    if window > 0:
        see &= (j > at - window) | (j < sinks)
    return see


def attention(q, k, v, see, scale):
    """One query [heads, dim] against keys and values [kv_heads, n, dim], of which `see` are seen: the result [heads, dim], and how
    far a kernel may be from it (u: half a step of the type).

    Scores are sums of dim products in fp32: off by at most (dim + 4) 2^-24 of the sum of their magnitudes; a weight by that twice (in
    the weight and in what it is divided by), by the exponential's argument and result (|s| 2^-23 + 2^-22), and the sums over n tokens, taken in
    parts, by (n + 64) 2^-24.  bf16 weights add 2 u each: a weight is rounded by at most u of it, and so is their
    sum, by what they are rounded by on average.  All of it relative to sum_j p_j |v_j|; then the result is rounded, by u."""
    heads, dim = q.shape
    kv_heads = k.shape[0]
    g = heads // kv_heads
    u = torch.finfo(q.dtype).eps / 2
    qd = q.double().view(kv_heads, g, dim)
    k, v = k[:, see], v[:, see]
    n = k.shape[1]
    if n == 0:
        return torch.zeros_like(q, dtype=torch.float64), torch.zeros_like(q, dtype=torch.float64)
    s = (qd.unsqueeze(2) * k.unsqueeze(1)).sum(-1) * scale
    size = (qd.unsqueeze(2) * k.unsqueeze(1)).abs().sum(-1).amax() * abs(scale)
    p = torch.softmax(s, dim=-1)
    out = (p.unsqueeze(-1) * v.unsqueeze(1)).sum(2)
    spread = (p.unsqueeze(-1) * v.abs().unsqueeze(1)).sum(2)
    off = 2 * ((dim + 4) * 2.0 ** -24 * size + 1.5 * s.abs().amax() * 2.0 ** -23 + 2.0 ** -22) + (n + 64) * 2.0 ** -24
    if q.dtype == torch.bfloat16:
        off = off + 2 * u
    far = off * spread * 1.01 + u * out.abs() * 1.02 + 1e-30
    return out.reshape(heads, dim), far.reshape(heads, dim)


def check(out, q, batch, scale=None, window=0, sinks=0, rows=None, offsets=None):
    """out, q: [tokens, heads * dim].  offsets: row r has the queries offsets[r] .. offsets[r + 1] of its last tokens."""
    dim = batch.dim
    scale = dim ** -0.5 if scale is None else scale
    worst = 0.0
    for r in range(len(batch.own)) if rows is None else rows:
        k, v = batch.tokens(r)
        total = k.shape[1]
        first, last = (r, r + 1) if offsets is None else (offsets[r], offsets[r + 1])
        for i in range(first, last):
            at = total - (last - i)
            want, far = attention(q[i].view(-1, dim), k, v, seen_by(at, total, window, sinks), scale)
            got = out[i].view(-1, dim).double()
            d = (got - want).abs()
            assert bool((d <= far).all()), (r, i, at, total, float((d / far).nan_to_num(nan=math.inf).max()))
            if d.numel() and float(far.max()) > 1e-20:
                worst = max(worst, float((d / far.clamp_min(1e-30)).max()))
    return worst
