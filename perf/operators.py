"""The paged KV cache of a serving step: operators whose time is tracked.

A step of R requests takes three calls. kv_slots turns request lengths into pages, a block table,
slots and positions; kv_write stores the new K and V rows in their slots; paged_attention lets the new
tokens attend over the cache, one token per request (decode), a chunk of a prompt, or a mixture.

The cache is two tensors [pages, page size, heads, head size] ("slot" layout) or the same with each
head's slots side by side in a page ("head" layout). `own` selects the framework's kernels; without it
`run` is the plain form in torch operations.
"""
import functools
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decode step's bookkeeping of a small batch: pure latency
        dict(name="slots decode 8", **_slots(8, 1, 2048, 0, 16, 1)),
        # a step that admits prompts beside running requests: ragged chunks, padded rows at the end
        dict(name="slots ragged 300", **_slots(300, 130, 4000, 200, 16, 2, pad=77)),
        # K and V of one decode step (8 requests, 8 heads of 128)
        dict(name="write decode 8", **_write("bf16", 8, 8, 128, 16, "slot", 0)),
        # K and V of a long prompt's chunk, the head layout
        dict(name="write chunk 8192", **_write("bf16", 8192, 8, 128, 16, "head", 0)),
        # float32, heads of 80, pages of 24 slots, padded rows
        dict(name="write f32 odd", **_write("f32", 777, 5, 80, 24, "slot", 23)),
        # the smallest call: one request of a 7B model, a short conversation, every head its own K and V
        dict(name="attend decode 1x500", **_attend("bf16", 1, 1, 499, 0, 32, 32, 128, 16, 3)),
        # a running batch: 64 requests of ragged lengths, four query heads to a K head
        dict(name="attend decode 64x8k", **_attend("bf16", 64, 1, 8191, 64, 32, 8, 128, 16, 4, ragged=True)),
        # one request at the end of a 131072-token context: few rows, a long axis
        dict(name="attend decode 1x131072", **_attend("bf16", 1, 1, 131071, 0, 32, 8, 128, 64, 5)),
        # a 2048-token chunk of a prompt behind 6144 tokens: the matrix cores' case
        dict(name="attend chunk 2048", **_attend("bf16", 1, 2048, 6144, 0, 32, 8, 128, 16, 6)),
        # chunks and single tokens in one batch, a window, pages of 24 slots, padded rows, the head layout
        dict(name="attend mixed window", **_attend("bf16", 24, 700, 3000, 18, 16, 2, 128, 24, 7, ragged=True,
                                                   window=1024, pad=13, layout="head")),
        # the wide heads of a 6B model, four prompts from their first token
        dict(name="attend prompts hd256", **_attend("bf16", 4, 1024, 0, 0, 16, 16, 256, 32, 8, ragged=True)),
        # float32, small heads, ragged chunks
        dict(name="attend f32 ragged", **_attend("f32", 6, 200, 1500, 2, 8, 4, 64, 16, 9, ragged=True)),
    ]


def _slots(R, new, ctx, singles, page, lens, pad=0):
    """R requests holding up to ctx tokens; `singles` of them (all where new is 1) take one more, the others 1..new."""
    return dict(op="slots", R=R, new=new, ctx=ctx, singles=singles, page=page, lens=lens, pad=pad, ragged=True)


def _write(dtype, T, nk, hd, page, layout, pad):
    """T rows, the last `pad` of them without a slot."""
    return dict(op="write", dtype=dtype, T=T, nk=nk, hd=hd, page=page, layout=layout, pad=pad)


def _attend(dtype, R, new, ctx, singles, nq, nk, hd, page, lens, ragged=False, window=0, pad=0, layout="slot"):
    """R requests behind ctx tokens (ragged: 0..ctx) with chunks of `new` (ragged: 1..new), `singles` of them of one token."""
    return dict(op="attend", dtype=dtype, R=R, new=new, ctx=ctx, singles=singles, nq=nq, nk=nk, hd=hd, page=page,
                lens=lens, ragged=ragged, window=window, pad=pad, layout=layout)


def _spread(rng, lo, hi):
    """An integer of lo..hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["slots", "write", "attend", "attend", "attend"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    layout = rng.choice(["slot", "head"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    lens = rng.randrange(1 << 20)
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    if op == "slots":
        R = _spread(rng, 1, 1000)
        new = _spread(rng, 1, max(2, 20000 // R))
        return _slots(R, new, _spread(rng, 1, 8192), rng.randint(0, R), page, lens, pad)
    if op == "write":
        T = _spread(rng, 1, 8000)
        return _write(dtype, T, rng.choice([1, 2, 4, 5, 8]), rng.choice([40, 64, 80, 96, 128, 256]), page, layout,
                      min(pad, T - 1))
    nk = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 5, 8])
    hd = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    window = rng.choice([0, 0, 0, _spread(rng, 16, 4096)])
    if rng.random() < 0.5:                 # decode: R requests, a token each
        R = _spread(rng, 1, 128)
        ctx = _spread(rng, 1, min(100000, 2000000 // (R * nk)))
        return _attend(dtype, R, 1, ctx, R, nk * g, nk, hd, page, lens, ragged=R > 1, window=window, pad=pad,
                       layout=layout)
    R = _spread(rng, 1, 16)                # chunks, some single tokens among them
    ctx = _spread(rng, 1, 6000 // R + 8)
    most = min((2000 if dtype == "bf16" else 500) // R + 8, 200_000_000_000 // (4 * R * (ctx + 2000) * nk * g * hd))
    new = _spread(rng, 2, max(2, most))
    return _attend(dtype, R, new, ctx, rng.randint(0, R - 1), nk * g, nk, hd, page, lens, ragged=True, window=window,
                   pad=pad, layout=layout)


def _lengths(case):
    """(tokens held, tokens new) of each request, from the case alone."""
    rng = random.Random(case["lens"])
    R, new, ctx = case["R"], case["new"], case["ctx"]
    held = [rng.randint(0, ctx) if case["ragged"] else ctx for _ in range(R)]
    more = [rng.randint(1, new) if case["ragged"] else new for _ in range(R)]
    for r in rng.sample(range(R), min(case["singles"], R)):
        more[r] = 1
    return held, more


def _pages(n, page):
    return -(-n // page)


def _cache(gen, pages, page, nk, hd, dtype, layout):
    """One cache tensor [pages, page, nk, hd] of the layout, filled with normal values."""
    shape = (pages, page, nk, hd) if layout == "slot" else (pages, nk, page, hd)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
    return x if layout == "slot" else x.transpose(1, 2)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "write":
        dt, T, nk, hd, page = _DT[case["dtype"]], case["T"], case["nk"], case["hd"], case["page"]
        pages = _pages(2 * T, page) + 1
        s["k"] = torch.randn((T, nk, hd), generator=gen, device="cuda", dtype=dt)
        s["v"] = torch.randn((T, nk, hd), generator=gen, device="cuda", dtype=dt)
        s["kc"] = _cache(gen, pages, page, nk, hd, dt, case["layout"])
        s["vc"] = _cache(gen, pages, page, nk, hd, dt, case["layout"])
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:T]
        slots[T - case["pad"]:] = -1
        s["slots"] = slots
        return s
    held, more = _lengths(case)
    R, page = case["R"], case["page"]
    T = sum(more) + case["pad"]
    total = [_pages(a + b, page) for a, b in zip(held, more)]
    width = max(total) + 2
    pool = sum(total) + 8
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(width, device="cuda")
    if case["op"] == "slots":
        # the pages held so far come off the pool's front, the rest are the stack of free ones
        have = _ints([_pages(a, page) for a in held])
        first = have.cumsum(0) - have
        s["table"] = torch.where(col[None] < have[:, None],
                                 order[(first[:, None] + col[None]).clamp(max=pool - 1)], -1).to(torch.int32)
        left = pool - sum(_pages(a, page) for a in held)
        s["free"] = order.flip(0)[:left].contiguous()
        s["count"] = _ints([left, 0])
        s["kv_len"], s["new"], s["T"] = _ints(held), _ints(more), T
        return s
    dt = _DT[case["dtype"]]
    want = _ints(total)
    first = want.cumsum(0) - want
    s["table"] = torch.where(col[None] < want[:, None],
                             order[(first[:, None] + col[None]).clamp(max=pool - 1)], -1).to(torch.int32)
    s["kv_len"] = _ints([a + b for a, b in zip(held, more)])
    starts = [0]
    for b in more:
        starts.append(starts[-1] + b)
    s["q_start"] = _ints(starts)
    s["q"] = 2 * torch.randn((T, case["nq"], case["hd"]), generator=gen, device="cuda", dtype=dt)
    s["kc"] = _cache(gen, pool, page, case["nk"], case["hd"], dt, case["layout"])
    s["vc"] = _cache(gen, pool, page, case["nk"], case["hd"], dt, case["layout"])
    s["out"] = torch.zeros_like(s["q"])
    s["scale"] = case["hd"] ** -0.5
    s["max_kv"] = max(a + b for a, b in zip(held, more))   # the host's own bookkeeping knows these
    s["max_new"] = max(more)
    return s


@functools.lru_cache(maxsize=None)
def _handle():
    """The specialization cache that a program creates once and keeps."""
    import paper_2609_37241_amd as tri
    return tri.SpecCache(auto_install=True)


def run(s):
    op = s["case"]["op"]
    if own:
        c = _handle()
        if op == "slots":
            return [s["table"]] + list(c.kv_slots(s["kv_len"], s["new"], s["table"], s["free"], s["count"],
                                                  s["case"]["page"], s["T"]))
        if op == "write":
            c.kv_write(s["k"], s["v"], s["slots"], s["kc"], s["vc"])
            return [s["kc"], s["vc"]]
        c.paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["kv_len"], s["q_start"], s["scale"],
                          window=s["case"]["window"], max_kv=s["max_kv"], out=s["out"])
        return s["out"]
    return {"slots": _plain_slots, "write": _plain_write, "attend": _plain_attend}[op](s)


def _plain_slots(s):
    page, T = s["case"]["page"], s["T"]
    old, new, table, free, count = s["kv_len"].long(), s["new"].long(), s["table"], s["free"], s["count"].long()
    q_start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    have, total = (old + page - 1) // page, (old + new + page - 1) // page
    want = total - have
    first = want.cumsum(0) - want
    col = torch.arange(table.shape[1], device=table.device)[None]
    at = count[0] - 1 - (first[:, None] + col - have[:, None])
    page_of = torch.where(at >= 0, free[at.clamp(0, free.shape[0] - 1)], -1)
    table.copy_(torch.where((col >= have[:, None]) & (col < total[:, None]), page_of, table))
    t = torch.arange(T, device=table.device)
    r = (t[:, None] >= q_start[None, 1:]).sum(1)
    inside = r < new.shape[0]
    r = r.clamp(max=new.shape[0] - 1)
    pos = torch.where(inside, old[r] + t - q_start[r], 0)
    p = table[r, pos // page].long()
    slots = torch.where(inside & (p >= 0), p * page + pos % page, -1)
    used = want.sum()
    left = torch.stack([(count[0] - used).clamp(min=0), (used - count[0]).clamp(min=0)])
    return [table, slots, pos.int(), q_start.int(), (old + new).int(), left.int()]


def _plain_write(s):
    kc, vc, slots = s["kc"], s["vc"], s["slots"]
    page = kc.shape[1]
    there = slots >= 0
    at = slots[there]
    kc[at // page, at % page] = s["k"][there]
    vc[at // page, at % page] = s["v"][there]
    return [kc, vc]


def _plain_attend(s):
    """All requests at once: K and V gathered to [R, nk, keys, hd] and the chunks to [R, nk, g new, hd], in 32 bits."""
    q, kc, vc, table = s["q"], s["kc"], s["vc"], s["table"].long()
    kv_len, q_start = s["kv_len"].long(), s["q_start"].long()
    (T, nq, hd), (pages, page, nk, _) = q.shape, kc.shape
    R, g, most, new = table.shape[0], nq // nk, s["max_kv"], s["max_new"]
    j = torch.arange(most, device=q.device)
    at = table[:, j // page]
    seen = (at >= 0) & (at < pages) & (j[None] < kv_len[:, None])
    at = at.clamp(0, pages - 1)
    there = seen[:, :, None, None]
    K = torch.where(there, kc[at, j % page], 0).float().permute(0, 2, 3, 1).contiguous()
    V = torch.where(there, vc[at, j % page], 0).float().transpose(1, 2).contiguous()
    n = q_start[1:] - q_start[:-1]
    i = torch.arange(new, device=q.device)
    row = q_start[:-1, None] + i[None]
    real = i[None] < n[:, None]
    Q = q[row.clamp(max=T - 1)].float().view(R, new, nk, g, hd).permute(0, 2, 3, 1, 4).reshape(R, nk, g * new, hd)
    S = (Q @ K).view(R, nk, g, new, most) * s["scale"]
    p = kv_len[:, None] - n[:, None] + i[None]
    mask = (j <= p[..., None]) & seen[:, None]
    if s["case"]["window"]:
        mask &= j > p[..., None] - s["case"]["window"]
    S = torch.where(mask[:, None, None], S, -math.inf)
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    total = P.sum(-1, keepdim=True)
    O = (P.view(R, nk, g * new, most) @ V).view(R, nk, g, new, hd) / torch.where(total == 0, 1.0, total)
    out = s["out"]
    out[row[real]] = O.permute(0, 3, 1, 2, 4).reshape(R, new, nq, hd)[real].to(out.dtype)
    return out


def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "write":
        T = case["T"]
        return {"bytes": 4 * (T - case["pad"]) * case["nk"] * case["hd"] * es + 8 * T, "flops": 0}
    held, more = _lengths(case)
    page = case["page"]
    T = sum(more) + case["pad"]
    pages = sum(_pages(a + b, page) for a, b in zip(held, more))
    if case["op"] == "slots":
        fresh = pages - sum(_pages(a, page) for a in held)
        # lengths, the pages that hold the first new tokens, the new pages; slots, positions, table, lengths
        return {"bytes": 8 * case["R"] + 4 * case["R"] + 8 * fresh + 12 * T + 8 * case["R"] + 12, "flops": 0}
    w = case["window"]
    pairs = keys = 0
    for a, b in zip(held, more):
        lo = max(0, a + 1 - w) if w else 0
        keys += a + b - lo
        # token i sees min(a + i + 1, w) keys
        full = b if not w else max(0, min(b, w - a - 1))
        pairs += full * a + full * (full + 1) // 2 + (b - full) * w
    row = case["hd"] * es
    return {"bytes": 2 * sum(more) * case["nq"] * row + 2 * keys * case["nk"] * row + 4 * _pages(keys, page)
            + 8 * case["R"], "flops": 4 * pairs * case["nq"] * case["hd"]}


def exact(case, seed):
    """By the definition, request by request and token by token, in 64 bits (whole numbers in Python's own)."""
    s = prepare(case, seed)
    if case["op"] == "slots":
        page = case["page"]
        table, free, count = s["table"].tolist(), s["free"].tolist(), s["count"].tolist()[0]
        slots, pos, starts, lens, need = [], [], [0], [], 0
        for r, (a, b) in enumerate(zip(s["kv_len"].tolist(), s["new"].tolist())):
            for x in range(a, a + b):
                if x % page == 0:
                    table[r][x // page] = free[count - 1 - need] if need < count else -1
                    need += 1
                p = table[r][x // page]
                slots.append(p * page + x % page if p >= 0 else -1)
                pos.append(x)
            starts.append(starts[-1] + b)
            lens.append(a + b)
        rest = s["T"] - len(slots)
        return [_ints(table), torch.tensor(slots + [-1] * rest, device="cuda"), _ints(pos + [0] * rest), _ints(starts),
                _ints(lens), _ints([max(count - need, 0), max(need - count, 0)])]
    if case["op"] == "write":
        out = []
        for x, c in (("k", "kc"), ("v", "vc")):
            rows, to = s[x].double().cpu(), s[c].double().cpu()
            for t, slot in enumerate(s["slots"].tolist()):
                if slot >= 0:
                    to[slot // case["page"], slot % case["page"]] = rows[t]
            out.append(to.cuda())
        return out
    out = s["out"].double()
    g = case["nq"] // case["nk"]
    starts = s["q_start"].tolist()
    for r, n in enumerate(s["kv_len"].tolist()):
        used = s["table"][r, :_pages(n, case["page"])].long()
        K = s["kc"][used].flatten(0, 1)[:n].double().repeat_interleave(g, 1).permute(1, 2, 0).contiguous()
        V = s["vc"][used].flatten(0, 1)[:n].double().repeat_interleave(g, 1).transpose(0, 1).contiguous()
        for t0 in range(starts[r], starts[r + 1], 256):
            t1 = min(t0 + 256, starts[r + 1])
            z = torch.matmul(s["q"][t0:t1].double().transpose(0, 1), K) * s["scale"]
            here = torch.arange(n - starts[r + 1] + t0, n - starts[r + 1] + t1, device=z.device)[:, None]
            key = torch.arange(n, device=z.device)[None]
            hide = key > here
            if case["window"]:
                hide |= here - key >= case["window"]
            z.masked_fill_(hide, -math.inf)
            out[t0:t1] = torch.matmul(torch.softmax(z, -1), V).transpose(0, 1)
    return out
