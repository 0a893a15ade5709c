"""GPU: attention over 8-bit codes, its error against 64 bits beside that of the plain computation
in 32 bits (root mean squares over all outputs of a call), and beside that of the same in
64 bits with one part fewer of what the kernels take apart: queries (float32) and weights.

bfloat16, tiles of few rows: weights in two parts are off by 2^-16, a 256th of the rounding of the
result (at most 2^-8, in both): the same error but for results that a rounding of float32
moves over a border, far less than a hundredth of them.
Tiles of many rows: a weight, times its key's V scale, is rounded once. What it leaves is even over
half a step of 2^-7 to both sides, so at most 2^-8 / sqrt(3) of the number as a root mean square (for
1; 1.66e-3 over all numbers, the error of the result's rounding). Which numbers meet it the scales
decide, here those of a range: 0.8 to 2.4 times a power of two. Over keys whose V is independent
squares add up in the sum as in its error, so the result has that part of itself, beside its own rounding.
float32: three products a number instead of one make at most three times as many roundings
of a score, which add up as a square root: less than twice the plain form's error. What a part less
leaves is larger, and to be missed by a tenth of it at least.
"""
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged_precision import CHUNKS, SHORT, error, plain
from tests.test_gpu_paged_q8 import CODES, DT, attend, cache, problem, tile_problem  # noqa: F401

pytestmark = pytest.mark.gpu
MANY = [(1 + i % 60, 1) for i in range(300)]


def held(p):
    """The problem with the values of its cache in 64 bits."""
    values = {}
    for c, s in (("kc", "ks"), ("vc", "vs")):
        x = p[c].float().double()
        values[c] = x * p[s].double().repeat_interleave(x.shape[1] // p[s].shape[1], 1)[..., None]
    return dict(p, **values)


def cut(x, parts):
    """x less what `parts` parts of 8 bits, cut off, leave of it."""
    rest = x.float()
    for _ in range(parts):
        rest = rest - (rest.view(torch.int32) & -65536).view(torch.float32)
    return x - rest.double()


def rounded(x, parts):
    """x as `parts` bfloat16 numbers, each the nearest to what the ones before leave."""
    total = torch.zeros_like(x)
    for _ in range(parts):
        total = total + (x - total).float().to(torch.bfloat16).double()
    return total


def coarse(p, dtype, queries, weights):
    """In 64 bits with queries(q) and weights(w s), s the key's V scale; the result rounded once."""
    out = torch.empty(p["q"].shape, dtype=torch.float64, device=p["q"].device)
    page, nk = p["kc"].shape[1:3]
    g, starts = p["q"].shape[1] // nk, p["q_start"].tolist()
    for r, kv in enumerate(p["kv_len"].tolist()):
        a, b = starts[r], starts[r + 1]
        used = p["table"][r, :-(-kv // page)].long()
        hidden = torch.arange(kv, device=out.device) > torch.arange(kv - (b - a), kv, device=out.device)[:, None]
        for h in range(nk if b > a else 0):
            k, v = (p[x][used, :, h].flatten(0, 1)[:kv].float().double() for x in ("kc", "vc"))
            ks, vs = (p[x][used, :, h].double().repeat_interleave(page // p[x].shape[1], 1).flatten()[:kv]
                      for x in ("ks", "vs"))
            q = queries(p["q"][a:b, h * g:(h + 1) * g].double()).transpose(0, 1).reshape(-1, k.shape[1])
            s = (q @ k.t().contiguous()).view(g, b - a, kv) * ks * p["scale"]
            s = s.masked_fill(hidden, -float("inf"))
            w = torch.exp(s - s.amax(-1, keepdim=True))
            o = weights(w * vs).view(-1, kv) @ v / w.sum(-1).view(-1, 1)
            out[a:b, h * g:(h + 1) * g] = o.view(g, b - a, -1).transpose(0, 1)
    return out.to(DT[dtype])


def errors(cache, p, dtype, variant, heads=None):  # noqa: F811
    """Of the kernels and of the plain form; exact."""
    got = attend(cache, p)
    s = cache.last_selection()
    assert s.variant in variant and (heads is None or s.key[3] >> 25 & 3 == heads)
    h = held(p)
    exact = plain(h, dtype, torch.float64)
    return error(got, exact), error(plain(h, dtype, torch.float32), exact), exact


as_is = lambda x: x  # noqa: E731
# a request's tokens, heads, log2 of the K heads of a tile
ROWS = [(SHORT, 16, 4, 64, 0), (SHORT, 20, 4, 128, 0), (MANY, 32, 4, 128, 1), (MANY, 16, 4, 64, 2),
        (MANY, 8, 4, 256, 2), ([(9000, 1)], 8, 2, 64, 1), ([(5000, 1), (700, 2), (40, 1)], 8, 2, 128, 1),
        ([(3000, 1)] * 3, 4, 4, 80, 2), ([(700, 1)] * 5, 8, 1, 256, 0)]


@pytest.mark.parametrize("lens,nq,nk,hd,heads", ROWS)
@pytest.mark.parametrize("code", CODES)
def test_bfloat16_few_rows(cache, code, lens, nq, nk, hd, heads):  # noqa: F811
    p = problem("bf16", code, lens, nq, nk, hd, 16, 8, seed=nq + hd)
    own, ref, exact = errors(cache, p, "bf16", (P.PA8_ROWS,), heads)
    one = error(coarse(p, "bf16", as_is, lambda w: rounded(w, 1)), exact)
    assert abs(own / ref - 1) <= 0.01 < one / ref - 1, (own, ref, one)


@pytest.mark.parametrize("lens,nq,nk,hd", [(CHUNKS, 8, 2, 64), (CHUNKS, 8, 2, 128), (CHUNKS, 4, 1, 256),
                                           ([(900, 900)], 4, 2, 128)])
@pytest.mark.parametrize("code", CODES)
def test_bfloat16_many_rows(cache, code, lens, nq, nk, hd):  # noqa: F811
    p = tile_problem("bf16", code, lens, nq, nk, hd, seed=nq + hd)
    own, ref, _ = errors(cache, p, "bf16", (P.PA8_TILE, P.PA8_PAIR))
    assert own ** 2 <= ref ** 2 + 2.0 ** -16 / 3, (own, ref)


@pytest.mark.parametrize("form,lens,nq,nk,hd,heads", [("rows", *x) for x in ROWS] + [
    ("tile", CHUNKS, 8, 2, 64, 0), ("tile", CHUNKS, 8, 2, 128, 0), ("tile", CHUNKS, 4, 1, 256, 0)])
@pytest.mark.parametrize("code", CODES)
def test_float32(cache, code, form, lens, nq, nk, hd, heads):  # noqa: F811
    make = tile_problem if form == "tile" else lambda *a, **k: problem(*a, 16, 8, **k)
    p = make("f32", code, lens, nq, nk, hd, seed=nq + hd)
    own, ref, exact = errors(cache, p, "f32", (P.PA8_TILE if form == "tile" else P.PA8_ROWS,), heads)
    two = error(coarse(p, "f32", lambda q: cut(q, 2), as_is), exact)
    parts = error(coarse(p, "f32", as_is, lambda w: rounded(w, 2)), exact)
    assert own <= min(2 * ref, 0.9 * two, 0.9 * parts), (own, ref, two, parts)
