"""The paged KV cache in 8 bits: operators whose time is tracked.

K and V are codes of 8 bits (signed integers, or floats of 4 exponent and 3 mantissa bits) with one float32
scale for each block of tokens and head: what a code stands for is code * scale. Three calls: kv_write_q8 quantises
the new K and V rows into their slots (a block that holds tokens already keeps its scale, or takes a larger one
and has its codes rounded again), kv_read_q8 gives the values back as rows, paged_attention_q8 lets the new
tokens attend over the codes, one token per request (decode), a chunk of a prompt, or a mixture.

The codes are two tensors [pages, page size, heads, head size] ("slot" layout) or the same with each head's slots side
by side in a page ("head" layout), the scales two tensors [pages, blocks of a page, heads]. A case of a write reads
the blocks it touched back, since their values are its result. `own` selects the framework's kernels; without it
`run` is the plain form in torch operations.
"""
import functools
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_MOST = {"int8": 127.0, "e4m3": 448.0}
_LEAST = 2.0 ** -100                      # the smallest scale


def listed():
    return [
        # one decode step of a small batch: a token to each of 8 requests, inside a block or beginning one
        dict(name="write decode 8", **_rows("write", "bf16", "int8", 8, 1, 2047, 8, 8, 128, 16, 16, 1)),
        # a long prompt's chunk, behind tokens that end inside a block
        dict(name="write chunk 8192", **_rows("write", "bf16", "e4m3", 1, 8192, 1000, 0, 8, 128, 16, 16, 2, layout="head")),
        # float32, heads of 80, pages of 24 slots in blocks of 8, ragged chunks among single tokens, padded rows
        dict(name="write f32 odd", **_rows("write", "f32", "int8", 12, 130, 500, 5, 5, 80, 24, 8, 3, pad=23)),
        # a shared prefix given back as rows, for a kernel that knows no pages
        dict(name="read prefix 2048", **_rows("read", "bf16", "int8", 1, 2048, 0, 0, 8, 128, 16, 16, 4)),
        # a batch's whole caches, ragged, on the way to another layout
        dict(name="read ragged 32", **_rows("read", "bf16", "e4m3", 32, 4000, 0, 0, 8, 128, 16, 8, 5, pad=40)),
        # the smallest attention: one request of a 7B model, a short conversation, every head its own K and V
        dict(name="attend decode 1x500", **_attend("bf16", "int8", 1, 1, 499, 0, 32, 32, 128, 16, 16, 6)),
        # a running batch: 64 requests of ragged lengths, four query heads to a K head
        dict(name="attend decode 64x8k", **_attend("bf16", "e4m3", 64, 1, 8191, 64, 32, 8, 128, 16, 16, 7, ragged=True)),
        # one request at the end of a 131072-token context: few rows, a long axis
        dict(name="attend decode 1x131072", **_attend("bf16", "int8", 1, 1, 131071, 0, 32, 8, 128, 64, 64, 8)),
        # a 2048-token chunk of a prompt behind 6144 tokens: the matrix cores' case
        dict(name="attend chunk 2048", **_attend("bf16", "e4m3", 1, 2048, 6144, 0, 32, 8, 128, 16, 16, 9)),
        # chunks and single tokens in one batch, a window, pages of 24 slots in blocks of 12, padded rows, the head layout
        dict(name="attend mixed window", **_attend("bf16", "int8", 24, 700, 3000, 18, 16, 2, 128, 24, 12, 10, ragged=True,
                                                   window=1024, pad=13, layout="head")),
        # the wide heads of a 6B model, four prompts from their first token
        dict(name="attend prompts hd256", **_attend("bf16", "e4m3", 4, 1024, 0, 0, 16, 16, 256, 32, 32, 11, ragged=True)),
        # float32 queries, small heads, ragged chunks, a scale for each token
        dict(name="attend f32 ragged", **_attend("f32", "int8", 6, 200, 1500, 2, 8, 4, 64, 16, 1, 12, ragged=True)),
    ]


def _rows(op, dtype, code, R, new, ctx, singles, nk, hd, page, block, lens, layout="slot", pad=0):
    """R requests behind ctx tokens (more than one: 0..ctx) with `new` rows (more than one: 1..new), `singles` of one."""
    return dict(op=op, dtype=dtype, code=code, R=R, new=new, ctx=ctx, singles=singles, nk=nk, hd=hd, page=page,
                block=block, lens=lens, layout=layout, pad=pad, ragged=R > 1)


def _attend(dtype, code, R, new, ctx, singles, nq, nk, hd, page, block, lens, ragged=False, window=0, pad=0,
            layout="slot"):
    """R requests behind ctx tokens (ragged: 0..ctx) with chunks of `new` (ragged: 1..new), `singles` of them of one token."""
    return dict(op="attend", dtype=dtype, code=code, R=R, new=new, ctx=ctx, singles=singles, nq=nq, nk=nk, hd=hd,
                page=page, block=block, lens=lens, ragged=ragged, window=window, pad=pad, layout=layout)


def _spread(rng, lo, hi):
    """An integer of lo..hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "attend", "attend", "attend"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    block = rng.choice([b for b in (1, 4, 8, 12, 16, 32, 64) if page % b == 0] + [page, page])
    layout = rng.choice(["slot", "head"])
    dtype, code = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["int8", "e4m3"])
    lens = rng.randrange(1 << 20)
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    if op != "attend":
        R = _spread(rng, 1, 200)
        new = _spread(rng, 1, max(2, (8000 if op == "write" else 40000) // R))
        return _rows(op, dtype, code, R, new, 0 if op == "read" else _spread(rng, 1, max(2, 40000 // R)),
                     rng.randint(0, R), rng.choice([1, 2, 4, 5, 8]), rng.choice([40, 64, 80, 96, 128, 256]), page, block,
                     lens, layout, pad)
    nk = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 5, 8])
    hd = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    window = rng.choice([0, 0, 0, _spread(rng, 16, 4096)])
    if rng.random() < 0.5:                 # decode: R requests, a token each
        R = _spread(rng, 1, 128)
        ctx = _spread(rng, 1, min(100000, 2000000 // (R * nk)))
        return _attend(dtype, code, R, 1, ctx, R, nk * g, nk, hd, page, block, lens, ragged=R > 1, window=window,
                       pad=pad, layout=layout)
    R = _spread(rng, 1, 16)                # chunks, some single tokens among them
    ctx = _spread(rng, 1, 6000 // R + 8)
    most = min((2000 if dtype == "bf16" else 500) // R + 8, 200_000_000_000 // (4 * R * (ctx + 2000) * nk * g * hd))
    new = _spread(rng, 2, max(2, most))
    return _attend(dtype, code, R, new, ctx, rng.randint(0, R - 1), nk * g, nk, hd, page, block, lens, ragged=True,
                   window=window, pad=pad, layout=layout)


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


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(gen, pages, case, gain):
    """(codes [pages, page, nk, hd] of the layout, scales) of normal values, the last dimension times `gain`."""
    page, nk, hd, block = case["page"], case["nk"], case["hd"], case["block"]
    codes = torch.empty((pages, page, nk, hd) if case["layout"] == "slot" else (pages, nk, page, hd), device="cuda",
                        dtype=_CODE[case["code"]])
    codes = codes if case["layout"] == "slot" else codes.transpose(1, 2)
    scales = torch.empty((pages, page // block, nk), device="cuda")
    some = max(1, (1 << 26) // (page * nk * hd))
    for p in range(0, pages, some):
        n = min(some, pages - p)
        x = torch.randn((n, page // block, block, nk, hd), generator=gen, device="cuda") * gain
        s = (x.abs().amax((2, 4)) / _MOST[case["code"]]).clamp(min=_LEAST)
        if case["code"] == "e4m3":
            s = torch.exp2(torch.ceil(torch.log2(s)))
        x = (x / s[:, :, None, :, None]).reshape(n, page, nk, hd)
        codes[p:p + n] = x.round().to(torch.int8) if case["code"] == "int8" else x.clamp(-448, 448).to(codes.dtype)
        scales[p:p + n] = s
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    held, more = _lengths(case)
    R, page, block, nk, hd, dt = case["R"], case["page"], case["block"], case["nk"], case["hd"], _DT[case["dtype"]]
    T = sum(more) + case["pad"]
    total = [_pages(a + b, page) for a, b in zip(held, more)]
    width, pool = max(total) + 2, sum(total) + 8
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    col, want = torch.arange(width, device="cuda"), _ints(total)
    first = want.cumsum(0) - want
    s["table"] = torch.where(col[None] < want[:, None],
                             order[(first[:, None] + col[None]).clamp(max=pool - 1)], -1).to(torch.int32)
    s["kv_len"] = _ints([a + b for a, b in zip(held, more)])
    starts = [0]
    for b in more:
        starts.append(starts[-1] + b)
    s["q_start"] = _ints(starts)
    # a few channels of K are larger than the others, the same ones in all tokens
    gain = torch.where(torch.rand((nk, hd), generator=gen, device="cuda") < 1 / 32, 6.0, 1.0)
    s["kc"], s["ks"] = _cache(gen, pool, case, gain)
    s["vc"], s["vs"] = _cache(gen, pool, case, 1.0)
    s["T"], s["max_new"] = T, max(more)
    if case["op"] == "write":
        s["k"] = (torch.randn((T, nk, hd), generator=gen, device="cuda") * gain).to(dt)
        s["v"] = torch.randn((T, nk, hd), generator=gen, device="cuda").to(dt)
        # what the touched blocks hold in the end, and how many they are (the host's own bookkeeping knows)
        back = [0]
        for a, b in zip(held, more):
            back.append(back[-1] + a + b - a // block * block)
        s["back_start"], s["back"] = _ints(back), back[-1]
        s["blocks"] = sum(_pages(a + b, block) - a // block for a, b in zip(held, more))
    elif case["op"] == "read":
        s["k"] = torch.zeros((T, nk, hd), device="cuda", dtype=dt)
        s["v"] = torch.zeros((T, nk, hd), device="cuda", dtype=dt)
    else:
        s["q"] = 2 * torch.randn((T, case["nq"], hd), generator=gen, device="cuda", dtype=dt)
        s["out"] = torch.zeros_like(s["q"])
        s["scale"] = hd ** -0.5
        s["max_kv"] = max(a + b for a, b in zip(held, more))
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
        cache = (s["kc"], s["vc"], s["ks"], s["vs"], s["table"], s["kv_len"])
        if op == "write":
            c.kv_write_q8(s["k"], s["v"], *cache, s["q_start"])
            return [*c.kv_read_q8(*cache, s["back_start"], s["back"], s["k"].dtype), s["ks"], s["vs"]]
        if op == "read":
            return list(c.kv_read_q8(*cache, s["q_start"], s["T"], s["k"].dtype, k=s["k"], v=s["v"]))
        c.paged_attention_q8(s["q"], *cache, s["q_start"], s["scale"], window=s["case"]["window"], max_kv=s["max_kv"],
                             out=s["out"])
        return s["out"]
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[op](s)


def _request_of(starts, T):
    """(request, whether there is one) of rows 0..T."""
    t = torch.arange(T, device=starts.device)
    r = (t[:, None] >= starts[None, 1:]).sum(1)
    return r.clamp(max=starts.shape[0] - 2), r < starts.shape[0] - 1


def _plain_rows(s, starts, T):
    """(K, V) in 32 bits of the rows' tokens, and which rows are a request's."""
    kv_len, page, block = s["kv_len"].long(), s["case"]["page"], s["case"]["block"]
    r, there = _request_of(starts, T)
    pos = torch.where(there, kv_len[r] - starts[r + 1] + torch.arange(T, device=r.device), 0)
    at, slot = s["table"][r, pos // page].long(), pos % page
    return [c[at, slot].float() * x[at, slot // block][..., None]
            for c, x in ((s["kc"], s["ks"]), (s["vc"], s["vs"]))] + [there]


def _plain_read(s):
    k, v, there = _plain_rows(s, s["q_start"].long(), s["T"])
    for out, x in ((s["k"], k), (s["v"], v)):
        out.copy_(torch.where(there[:, None, None], x.to(out.dtype), out))
    return [s["k"], s["v"]]


def _plain_write(s):
    """Block by block of those touched: [blocks, tokens of a block, nk, hd] of old and new values."""
    case, kv_len, starts = s["case"], s["kv_len"].long(), s["q_start"].long()
    page, block, code, most = case["page"], case["block"], case["code"], _MOST[case["code"]]
    n = starts[1:] - starts[:-1]
    held = kv_len - n
    count = (kv_len + block - 1) // block - held // block
    first = torch.cat([count.new_zeros(1), count.cumsum(0)])
    r, _ = _request_of(first, s["blocks"])
    u = torch.arange(s["blocks"], device=r.device)
    begin = (held[r] // block + u - first[r]) * block
    pos = begin[:, None] + torch.arange(block, device=r.device)[None]
    new = (pos >= held[r, None]) & (pos < kv_len[r, None])
    old = pos < held[r, None]
    row = (starts[r + 1, None] - kv_len[r, None] + pos).clamp(0, s["T"] - 1)
    at, b = s["table"][r, begin // page].long(), begin % page // block
    slot = begin[:, None] % page + torch.arange(block, device=r.device)[None]
    for x, codes, scales in ((s["k"], s["kc"], s["ks"]), (s["v"], s["vc"], s["vs"])):
        x = torch.where(new[..., None, None], x[row].float(), 0.0)
        need = x.abs().amax((1, 3)) / most
        if code == "e4m3":               # the power of two at or above it
            m, e = torch.frexp(need)
            need = torch.ldexp(torch.ones_like(need), torch.where(m == 0.5, e - 1, e))
        need = need.clamp(min=_LEAST)
        was = scales[at, b]
        now = torch.where(old.any(1)[:, None], torch.maximum(was, need), need)
        c = codes[at[:, None], slot].double()
        y = torch.where(new[..., None, None], x.double(), c * was.double()[:, None, :, None])
        y = y / now.double()[:, None, :, None]
        y = torch.where((new | old)[..., None, None], y, c)
        codes[at[:, None], slot] = y.round().to(torch.int8) if code == "int8" else y.float().to(codes.dtype)
        scales[at, b] = now
    k, v, _ = _plain_rows(s, s["back_start"].long(), s["back"])
    return [k.to(s["k"].dtype), v.to(s["v"].dtype), s["ks"], s["vs"]]


def _plain_attend(s):
    """All requests at once: K and V gathered to [R, nk, keys, hd] and the chunks to [R, nk, g new, hd], in 32 bits."""
    q, kc, vc, table, block = s["q"], s["kc"], s["vc"], s["table"].long(), s["case"]["block"]
    kv_len, q_start = s["kv_len"].long(), s["q_start"].long()
    (T, nq, hd), (pages, page, nk, _) = q.shape, kc.shape
    R, g, most, new = table.shape[0], nq // nk, s["max_kv"], s["max_new"]
    j = torch.arange(most, device=q.device)
    at = table[:, j // page]
    seen = (at >= 0) & (at < pages) & (j[None] < kv_len[:, None])
    at = at.clamp(0, pages - 1)
    there, slot = seen[:, :, None, None], j % page
    K = torch.where(there, kc[at, slot].float() * s["ks"][at, slot // block][..., None], 0)
    V = torch.where(there, vc[at, slot].float() * s["vs"][at, slot // block][..., None], 0)
    K, V = K.permute(0, 2, 3, 1).contiguous(), V.transpose(1, 2).contiguous()
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
    es = 2 if case["dtype"] == "bf16" else 4
    held, more = _lengths(case)
    page, block, nk, hd = case["page"], case["block"], case["nk"], case["hd"]
    if case["op"] != "attend":
        scales = sum(_pages(a + b, block) - a // block for a, b in zip(held, more))
        if case["op"] == "read":
            return {"bytes": 2 * nk * (sum(more) * hd * (1 + es) + 4 * scales), "flops": 0}
        # the new rows, their codes and scales (a block's that goes on is read first); then the read of the blocks
        back = sum(a + b - a // block * block for a, b in zip(held, more))
        old = sum(a % block > 0 for a in held)
        return {"bytes": 2 * nk * (sum(more) * hd * (es + 1) + 4 * (scales + old) + back * hd * (1 + es) + 4 * scales),
                "flops": 0}
    w = case["window"]
    pairs = keys = 0
    for a, b in zip(held, more):
        lo = max(0, a + 1 - w) if w else 0
        keys += a + b - lo
        # token i sees min(a + i + 1, w) keys
        full = b if not w else max(0, min(b, w - a - 1))
        pairs += full * a + full * (full + 1) // 2 + (b - full) * w
    return {"bytes": 2 * sum(more) * case["nq"] * hd * es + 2 * keys * nk * hd + 8 * _pages(keys, block) * nk
            + 4 * _pages(keys, page) + 8 * case["R"], "flops": 4 * pairs * case["nq"] * hd}


def _nearest(y, code):
    """The codes' values nearest to y (float64), ties to the even one."""
    if code == "int8":
        return y.round()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (y / step).round() * step


def exact(case, seed):
    """By the definition, request by request, in 64 bits."""
    s = prepare(case, seed)
    page, block, code, nk, hd = case["page"], case["block"], case["code"], case["nk"], case["hd"]
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()

    def values(codes, scales, r, n):
        """The first n tokens of request r."""
        used = s["table"][r, :_pages(n, page)].long()
        x = codes[used].double() * scales[used].double().repeat_interleave(block, 1)[..., None]
        return x.flatten(0, 1)[:n]

    if case["op"] == "read":
        out = [s["k"].double(), s["v"].double()]
        for r, n in enumerate(lens):
            for o, (c, x) in zip(out, (("kc", "ks"), ("vc", "vs"))):
                o[starts[r]:starts[r + 1]] = values(s[c], s[x], r, n)[n - (starts[r + 1] - starts[r]):]
        return out
    if case["op"] == "write":
        back, scales = [], []
        for new, c, x in (("k", "kc", "ks"), ("v", "vc", "vs")):
            after, got = s[x].double(), []
            for r, n in enumerate(lens):
                t = n - (starts[r + 1] - starts[r])             # tokens before
                b0, b1 = t // block, _pages(n, block)           # the blocks touched
                rows = torch.zeros((b1 * block, nk, hd), dtype=torch.float64, device="cuda")
                rows[t:n] = s[new][starts[r]:starts[r + 1]].double()
                need = rows[b0 * block:].view(b1 - b0, block, nk, hd).abs().amax((1, 3)) / _MOST[code]
                # (scales are float32: rounded once, or the power of two at or above)
                need = (torch.exp2(torch.ceil(torch.log2(need.clamp(min=1e-300)))) if code == "e4m3" else
                        need.float().double()).clamp(min=_LEAST)
                at = s["table"][r].long()[torch.arange(b0, b1, device="cuda") * block // page]
                b = torch.arange(b0, b1, device="cuda") % (page // block)
                if t % block:
                    need[0] = torch.maximum(need[0], s[x][at[0], b[0]].double())
                    rows[b0 * block:t] = values(s[c], s[x], r, t)[b0 * block:]
                after[at, b] = need
                each = need.repeat_interleave(block, 0)[..., None]
                got.append((_nearest(rows[b0 * block:] / each, code) * each)[:n - b0 * block])
            back.append(torch.cat(got))
            scales.append(after)
        return back + scales
    out = s["out"].double()
    g = case["nq"] // nk
    for r, n in enumerate(lens):
        K = values(s["kc"], s["ks"], r, n).repeat_interleave(g, 1).permute(1, 2, 0).contiguous()
        V = values(s["vc"], s["vs"], r, n).repeat_interleave(g, 1).transpose(0, 1).contiguous()
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
