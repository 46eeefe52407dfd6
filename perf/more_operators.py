"""The operators of a model that attends to its context: a paged cache of keys and values, and the attention that reads it.

Three kinds of case:
  add      keys and values of new tokens into the cache: one a row, or ragged prompts (as_cache_add)
  attend   one new token a row over the cache; rows of one prompt share its pages (as_attend)
  prompts  ragged prompts, or the next chunks of them, over the cache (as_attend_prompts)

A query at position i sees the keys j <= i; with a window those with j > i - window, and the first `sinks` tokens.
listed() are the calls of a serving loop over N lattice codes a prompt; draw() gives more of the same ranges.
prepare() makes inputs on the GPU from the seed alone; run() is one pass, in plain torch or, where `own` is true,
through the library; exact() is the same from the definitions in 64 bits; work() what a pass cannot do without.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def _case(name, kind, heads, kv_heads, dim, dtype="bf16", page=16, **more):
    case = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page, **more}
    return dict(case, name=name) if name else case


def _add(name, heads, kv_heads, dim, rows, room, new, **more):
    """`new` 0: one token a row, of sequences of up to `room` tokens; else chunks of up to `new`."""
    return _case(name, "add", heads, kv_heads, dim, rows=rows, room=room, new=new, **more)


def _attend(name, heads, kv_heads, dim, prompts, codes, prompt, tokens, window=0, sinks=0, empty=False, **more):
    """Prompts of up to `prompt` tokens (0: none), each row up to `tokens` of its own; `empty`: some rows have none at all."""
    return _case(name, "attend", heads, kv_heads, dim, prompts=prompts, codes=codes, prompt=prompt, tokens=tokens, window=window, sinks=sinks,
                 empty=empty, **more)


def _prompts(name, heads, kv_heads, dim, rows, before, new, window=0, sinks=0, **more):
    """Chunks of up to `new` tokens behind up to `before` that are in the cache already."""
    return _case(name, "prompts", heads, kv_heads, dim, rows=rows, before=before, new=new, window=window, sinks=sinks, **more)


def listed():
    return [
        # the benchmark's batch, 16 prompts of 64 codes: each row's token of one step
        _add("add_batch", 32, 8, 128, 1024, 128, 0),
        # a batch of documents taken up, 16 of up to 4096 tokens
        _add("add_prompts", 32, 8, 128, 16, 4096, 4096),
        # one sequence, one token, a model of rank 512: nothing but latency
        _attend("attend_one_row", 8, 8, 64, 1, 1, 0, 200),
        # the benchmark's batch with a model of rank 512: prompts of up to 512 tokens, up to 64 of each code's own
        _attend("attend_batch", 8, 2, 64, 16, 64, 512, 64),
        # wide lattices over long documents: the largest of the prompts' shared part
        _attend("attend_wide", 32, 8, 128, 4, 256, 8192, 256),
        # a few long conversations, nothing shared: the cache is read at the memory's rate
        _attend("attend_long", 32, 8, 128, 8, 1, 0, 65536),
        # a model with a sliding window that keeps its first tokens, many users
        _attend("attend_window", 16, 4, 128, 256, 1, 0, 8192, window=1024, sinks=4, page=64),
        # a small fp32 model of odd sizes, small pages
        _attend("attend_f32_odd", 9, 3, 72, 5, 7, 130, 333, dtype="f32", page=8),
        # the benchmark's prompts taken up by the model of rank 512
        _prompts("prompts_batch", 8, 2, 64, 16, 0, 512),
        # one long document
        _prompts("prompts_long", 32, 8, 128, 1, 0, 8192),
        # the next chunks of documents, with a window and first tokens
        _prompts("prompts_window", 16, 4, 128, 6, 3000, 2048, window=1024, sinks=4, page=64),
        # a small fp32 model's prompts
        _prompts("prompts_f32_odd", 6, 2, 72, 9, 77, 301, dtype="f32", page=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["add", "attend", "attend", "attend", "attend", "prompts", "prompts", "prompts"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([64, 64, 128, 128, 128, 80, 96, 256, 8 * rng.randint(1, 32)])
    kv_heads = _log_int(rng, 1, 16)
    group = rng.choice([1, 1, 2, 3, 4, 4, 5, 8, 8, 16])
    while kv_heads * group * dim > 8192:
        kv_heads = max(1, kv_heads // 2)
        group = max(1, group // 2)
    heads, kv = kv_heads * group, kv_heads * dim
    mask = dict(window=0, sinks=0)
    if rng.random() < 0.4:
        mask = dict(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, rng.randint(1, 64)]))
    common = dict(dtype=dtype, page=rng.choice([1, 8, 16, 16, 16, 32, 64, 128, 256]))
    if kind == "add":
        rows = _log_int(rng, 1, 2048)
        most = max(1, min(4096, 60_000_000 // (rows * kv)))
        room = _log_int(rng, 1, most)
        return _add(None, heads, kv_heads, dim, rows, room, 0 if rng.random() < 0.5 else _log_int(rng, 1, room), **common)
    if kind == "attend":
        values = 800_000_000 // SIZE[dtype]
        if rng.random() < 0.5:
            rows = _log_int(rng, 1, 512)
            most = max(1, min(65536, values // (rows * kv), 250_000_000 // (rows * heads)))
            return _attend(None, heads, kv_heads, dim, rows, 1, 0, _log_int(rng, 1, most), empty=rng.random() < 0.3, **mask, **common)
        prompts, codes = _log_int(rng, 1, 32), _log_int(rng, 2, 256)
        rows = prompts * codes
        tokens = _log_int(rng, 1, max(1, min(512, values // 2 // (rows * kv))))
        most = 8192 if dtype == "bf16" else 1024
        prompt = _log_int(rng, 1, max(1, min(most, values // 2 // (prompts * kv), 250_000_000 // (rows * heads))))
        return _attend(None, heads, kv_heads, dim, prompts, codes, prompt, tokens, empty=rng.random() < 0.2, **mask, **common)
    rows = _log_int(rng, 1, 32)
    new = _log_int(rng, 1, 8192)
    before = rng.choice([0, 0, _log_int(rng, 1, 8192)])
    flops = 4e11 if dtype == "bf16" else 2.5e10
    while (4.0 * rows * heads * dim * new * (new / 2 + before) > flops or rows * heads * new * (new + before) > 2e9
           or rows * (new + before) * kv > 200_000_000):
        if rows > 1 and rng.random() < 0.5:
            rows = max(1, rows // 2)
        elif before > new:
            before = before // 2
        else:
            new = max(1, new * 2 // 3)
            before = before * 2 // 3
    return _prompts(None, heads, kv_heads, dim, rows, before, new, **mask, **common)


# ------------------------------------------------------------------------------------------------------ inputs

def _lens(g, rows, most, least=None):
    """Lengths from half of the longest to all of it, the first the longest."""
    lens = torch.randint(most // 2 if least is None else least, most + 1, (rows,), device="cuda", generator=g, dtype=torch.int32)
    lens[0] = most
    return lens


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt, page, dim = case["kind"], DTYPES[case["dtype"]], case["page"], case["dim"]
    heads, kv_heads = case["heads"], case["kv_heads"]
    s = {"table": None, "prompt_table": None, "prompt_lens": None, "offsets": None}
    pages_of = lambda n: -(-n // page)  # noqa: E731
    if kind == "attend":
        prompts, rows = case["prompts"], case["prompts"] * case["codes"]
        width, prompt_width = pages_of(case["tokens"]), pages_of(case["prompt"])
        s["lens"] = _lens(g, rows, case["tokens"], 0 if case["empty"] else None)
        if case["prompt"]:
            s["prompt_lens"] = _lens(g, prompts, case["prompt"], 0 if case["empty"] else None)
        if case["empty"]:
            s["lens"] *= torch.rand(rows, device="cuda", generator=g) < 0.8
        queries = rows
    else:
        rows, prompts, prompt_width = case["rows"], 0, 0
        room = case["room"] if kind == "add" else case["before"] + case["new"]
        width = pages_of(room)
        if case["new"] == 0:
            s["lens"] = _lens(g, rows, room).clamp_min_(1)
            queries = rows
        else:
            # (chunks as ragged, but of the same lengths in another order for another seed: as many tokens in all)
            new = torch.linspace(case["new"], case["new"] - case["new"] // 2, rows, device="cuda").round_().int()
            new = new[torch.randperm(rows, device="cuda", generator=g)]
            before = _lens(g, rows, room - case["new"])
            s["lens"] = before + new
            s["offsets"] = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
            s["offsets"][1:] = new.cumsum(0)
            queries = int(s["offsets"][-1])
    # the pages lie anywhere in the cache, which holds some more
    pages = rows * width + prompts * prompt_width + 3
    order = torch.randperm(pages, device="cuda", generator=g).int()
    s["table"] = order[:rows * width].view(rows, width)
    if prompt_width:
        s["prompt_table"] = order[rows * width:rows * width + prompts * prompt_width].view(prompts, prompt_width)
    s["k"] = torch.randn(pages, kv_heads, page, dim, device="cuda", generator=g, dtype=dt)
    s["v"] = torch.randn(pages, kv_heads, page, dim, device="cuda", generator=g, dtype=dt)
    # query, key and value as one product leaves them; queries lean towards a direction, and so do the first tokens' keys
    qkv = torch.randn(queries, (heads + 2 * kv_heads) * dim, device="cuda", generator=g)
    lean = torch.randn(kv_heads, 1, dim, device="cuda", generator=g)
    qkv[:, :heads * dim] = (1.5 * qkv[:, :heads * dim].view(queries, kv_heads, -1, dim) + lean).view(queries, -1)
    first = (s["table"] if s["prompt_table"] is None else s["prompt_table"])[:, 0].long()
    if kind != "add":
        s["k"][first, :, 0] = (s["k"][first, :, 0].float() + 0.4 * lean[:, 0]).to(dt)
    s["qkv"] = qkv.to(dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2210_15458_amd import binding as B
    rows, heads, kv_heads, dim = s["table"].shape[0], case["heads"], case["kv_heads"], case["dim"]
    s["ctx"] = B.Ctx(max(rows, s["qkv"].shape[0]), 32128, DTYPES[case["dtype"]])
    s["cache"] = B.Cache(s["k"], s["v"])
    s["seqs"] = B.Sequences(rows, s["table"], s["lens"], s["prompt_table"], s["prompt_lens"], case.get("codes", 1))
    s["q"], s["k_new"], s["v_new"] = s["qkv"].split([heads * dim, kv_heads * dim, kv_heads * dim], dim=1)
    s["out"] = torch.empty(s["qkv"].shape[0], heads * dim, dtype=DTYPES[case["dtype"]], device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ a pass

def _gathered(cache, table, n):
    """Tokens 0 .. n-1 of each sequence of the table: [sequences, kv_heads, n, dim]."""
    t = torch.arange(n, device="cuda")
    page = cache.shape[2]
    return cache[table[:, t // page].long(), :, t % page].float().transpose(1, 2).contiguous()


def _visible(c, at, key):
    see = key <= at
    if c["window"] > 0:
        see &= (key > at - c["window"]) | (key < c["sinks"])
    return see


def _weights(score, see):
    """exp(score - max) where seen, and its sum over the last dimension (1 where nothing is seen)."""
    score = torch.where(see, score, torch.full_like(score, -math.inf))
    top = score.amax(dim=-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(dim=-1, keepdim=True)
    return e, torch.where(total > 0, total, torch.ones_like(total))


def _plain_attend(s):
    c = s["case"]
    B, N, H, K, D = c["prompts"], c["codes"], c["heads"], c["kv_heads"], c["dim"]
    rows, G, P, T = B * N, H // K, c["prompt"], c["tokens"]
    q = s["qkv"][:, :H * D].float() / math.sqrt(D)
    k, v = _gathered(s["k"], s["table"], T), _gathered(s["v"], s["table"], T)
    score = (q.view(rows, K, G, D) @ k.transpose(2, 3).contiguous()).view(rows, H, T)
    start = torch.zeros(rows, dtype=torch.long, device="cuda")
    key = torch.arange(T, device="cuda")
    if P:
        start = s["prompt_lens"].long().repeat_interleave(N)
    at = (start + s["lens"] - 1).view(rows, 1, 1)
    see = _visible(c, at, start.view(rows, 1, 1) + key)
    if P:
        pk, pv = _gathered(s["k"], s["prompt_table"], P), _gathered(s["v"], s["prompt_table"], P)
        by_prompt = q.view(B, N, K, G, D).transpose(1, 2).reshape(B, K, N * G, D)
        shared = (by_prompt @ pk.transpose(2, 3).contiguous()).view(B, K, N, G, P).transpose(1, 2).reshape(rows, H, P)
        place = torch.arange(P, device="cuda")
        score = torch.cat([shared, score], dim=2)
        see = torch.cat([_visible(c, at, place) & (place < start.view(rows, 1, 1)), see], dim=2)
    e, total = _weights(score, see)
    o = (e[:, :, P:].reshape(rows, K, G, T) @ v).view(rows, H, D)
    if P:
        by_prompt = e[:, :, :P].reshape(B, N, K, G, P).transpose(1, 2).reshape(B, K, N * G, P)
        o = o + (by_prompt @ pv).view(B, K, N, G, D).transpose(1, 2).reshape(rows, H, D)
    return (o / total).view(rows, H * D).to(s["qkv"].dtype)


def _plain_prompts(s):
    c = s["case"]
    R, H, K, D, n = c["rows"], c["heads"], c["kv_heads"], c["dim"], c["new"]
    G, T = H // K, c["before"] + c["new"]
    offsets, queries = s["offsets"], s["qkv"].shape[0]
    token = torch.arange(queries, device="cuda")
    whose = torch.bucketize(token, offsets, right=True) - 1
    # a block of n queries a sequence, the last rows of short ones unused
    block = (offsets[:-1, None] + torch.arange(n, device="cuda")).clamp_max(queries - 1)
    q = (s["qkv"][:, :H * D].float() / math.sqrt(D))[block].view(R, n, K, G, D).permute(0, 2, 3, 1, 4).reshape(R, K, G * n, D)
    k, v = _gathered(s["k"], s["table"], T), _gathered(s["v"], s["table"], T)
    score = (q @ k.transpose(2, 3).contiguous()).view(R, H, n, T)
    at = (s["lens"] - (offsets[1:] - offsets[:-1])).view(R, 1, 1, 1) + torch.arange(n, device="cuda").view(1, 1, n, 1)
    e, total = _weights(score, _visible(c, at, torch.arange(T, device="cuda")))
    o = ((e.view(R, K, G * n, T) @ v).view(R, H, n, D) / total).transpose(1, 2)
    return o[whose, token - offsets[whose]].reshape(queries, H * D).to(s["qkv"].dtype)


def _plain_add(s):
    c = s["case"]
    H, K, D, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    queries = s["qkv"].shape[0]
    if c["new"] == 0:
        whose, at = torch.arange(queries, device="cuda"), s["lens"].long() - 1
    else:
        token = torch.arange(queries, device="cuda")
        whose = torch.bucketize(token, s["offsets"], right=True) - 1
        at = s["lens"][whose] - s["offsets"][whose + 1] + token
    place = s["table"][whose, at // page].long()
    new = s["qkv"][:, H * D:].view(queries, 2, K, D)
    s["k"][place, :, at % page] = new[:, 0]
    s["v"][place, :, at % page] = new[:, 1]
    return s["k"], s["v"]


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2210_15458_amd import binding as B
        if kind == "add":
            B.as_cache_add(s["ctx"], s["cache"], s["seqs"], s["k_new"], s["v_new"], s["offsets"])
            return s["k"], s["v"]
        if kind == "attend":
            B.as_attend(s["ctx"], s["cache"], s["seqs"], s["q"], s["out"], window=c["window"], sinks=c["sinks"])
        else:
            B.as_attend_prompts(s["ctx"], s["cache"], s["seqs"], s["q"], s["offsets"], s["out"], window=c["window"], sinks=c["sinks"])
        return s["out"]
    return {"add": _plain_add, "attend": _plain_attend, "prompts": _plain_prompts}[kind](s)


# ----------------------------------------------------------------------------------------- the definitions in 64 bits

def _tokens_of(cache, table_row, n):
    """[kv_heads, n, dim] in 64 bits, page by page."""
    page = cache.shape[2]
    return cache[table_row[:-(-n // page)].long()].double().transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def _attention(q, k, v, first, window, sinks):
    """Queries [n, dim] at positions first .. first + n - 1 against all keys [T, dim], by the definition."""
    n, T = q.shape[0], k.shape[0]
    behind = torch.arange(first, first + n, device="cuda").unsqueeze(1) - torch.arange(T, device="cuda").unsqueeze(0)
    hidden = behind < 0
    if window > 0:
        hidden |= (behind >= window) & (torch.arange(T, device="cuda") >= sinks)
    a = torch.matmul(q, k.t().contiguous()) / math.sqrt(q.shape[1])
    a.masked_fill_(hidden, -math.inf)
    return torch.softmax(a, dim=1) @ v


def exact(case, seed):
    s = _inputs(case, seed)
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    G, window, sinks = H // K, case.get("window", 0), case.get("sinks", 0)
    lens = s["lens"].tolist()
    if case["kind"] == "add":
        k, v, table, page = s["k"].double(), s["v"].double(), s["table"].tolist(), case["page"]
        offsets = list(range(len(lens) + 1)) if s["offsets"] is None else s["offsets"].tolist()
        new = s["qkv"][:, H * D:].double()
        for r, n in enumerate(lens):
            at, end = n - (offsets[r + 1] - offsets[r]), n
            while at < end:                     # a page, or what of it is new
                upto = min(end, (at // page + 1) * page)
                from_ = offsets[r + 1] - (end - at)
                piece = new[from_:from_ + upto - at].view(-1, 2, K, D)
                where = (table[r][at // page], slice(None), slice(at % page, at % page + upto - at))
                k[where], v[where] = piece[:, 0].transpose(0, 1), piece[:, 1].transpose(0, 1)
                at = upto
        return k, v
    q = s["qkv"][:, :H * D].double()
    out = torch.zeros_like(q)
    if case["kind"] == "attend":
        prompt_lens = s["prompt_lens"].tolist() if case["prompt"] else [0] * case["prompts"]
        for b in range(case["prompts"]):
            pk = pv = None
            if prompt_lens[b]:
                pk, pv = (_tokens_of(s[x], s["prompt_table"][b], prompt_lens[b]) for x in "kv")
            for r in range(b * case["codes"], (b + 1) * case["codes"]):
                total = prompt_lens[b] + lens[r]
                if not total:
                    continue
                k, v = (_tokens_of(s[x], s["table"][r], lens[r]) for x in "kv")
                if pk is not None:
                    k, v = torch.cat([pk, k], dim=1), torch.cat([pv, v], dim=1)
                if window > 0 and total > window:      # (what is not seen is left out: at most the first tokens and the window)
                    keep = torch.cat([torch.arange(min(sinks, total - window)), torch.arange(total - window, total)]).cuda()
                    k, v = k[:, keep], v[:, keep]
                a = torch.bmm(q[r].view(K, G, D), k.transpose(1, 2).contiguous()) / math.sqrt(D)
                out[r] = torch.bmm(torch.softmax(a, dim=2), v.contiguous()).view(-1)
        return out
    offsets = s["offsets"].tolist()
    for r, total in enumerate(lens):
        a, b = offsets[r], offsets[r + 1]
        k, v = (_tokens_of(s[x], s["table"][r], total) for x in "kv")
        for h in range(H):
            out[a:b, h * D:(h + 1) * D] = _attention(q[a:b, h * D:(h + 1) * D], k[h // G], v[h // G], total - (b - a), window, sinks)
    return out


# ------------------------------------------------------------------------------------------------- what it takes

def _mean(most, rows, empty=False):
    """Of such lengths."""
    return most * (0.75 + 0.25 / rows) if not empty else most * 0.4 if rows > 1 else float(most)


def work(case):
    kind, esz, D, H, K = case["kind"], SIZE[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]
    kv = 2.0 * K * D * esz                             # key and value of a token
    if kind == "add":
        tokens = case["rows"] * (_mean(case["new"], case["rows"]) if case["new"] else 1.0)
        return {"bytes": 2.0 * kv * tokens + 8.0 * case["rows"], "flops": 0.0}
    window, sinks = case["window"], case["sinks"]
    seen = lambda n: min(n, window + sinks) if window > 0 else n  # noqa: E731
    if kind == "attend":
        B, rows = case["prompts"], case["prompts"] * case["codes"]
        prompt, tokens = _mean(case["prompt"], B, case["empty"]), _mean(case["tokens"], rows, case["empty"])
        mine = seen(prompt + tokens)                   # of a row
        shared = mine if window <= 0 else min(prompt, max(mine - tokens, 0.0) + min(sinks, tokens))
        shared = min(shared, prompt)
        return {"bytes": kv * (B * shared + rows * max(mine - shared, 0.0)) + 2.0 * rows * H * D * esz + 8.0 * rows, "flops": 4.0 * rows * H * D * mine}
    rows = case["rows"]
    new, before = _mean(case["new"], rows), _mean(case["before"], rows)
    pairs = new * before + new * new / 2
    if window > 0:
        w = window + sinks
        # before the window is full a query sees all there is
        ramp = max(0.0, min(new, w - before))
        pairs = min(pairs, ramp * before + ramp * ramp / 2 + (new - ramp) * w)
    tokens = new + (min(before, window + sinks) if window > 0 else before)
    return {"bytes": rows * (kv * tokens + 2.0 * new * H * D * esz), "flops": 4.0 * rows * pairs * H * D}
