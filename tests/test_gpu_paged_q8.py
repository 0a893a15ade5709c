"""GPU: the paged KV cache in 8 bits against the oracle (float64).

The write: codes and scales equal the oracle's, whatever they were before; nothing
else changes. The read: one rounding. Attention: every slot that no row may
see holds what it must not use (NaN codes and scales, else the largest codes); tolerances
are the oracle's slack (float32 arithmetic, with two more roundings of a score, for the
key's scale and the product with the other, and one of a weight, for the value's) plus, in
bf16, half a step (2^-8) of every weight where it meets V and of the result.
"""
import numpy as np
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged import BATCHES, DEV, DT, HALF, HEADS, TILE_BATCHES, check, f64, i32

pytestmark = pytest.mark.gpu
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
KIND = {"int8": P.INT8, "e4m3": P.E4M3}
CODES = list(CODE)
DTYPES = ["bf16", "f32"]


@pytest.fixture(scope="module")
def cache():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_37241_amd as tri
    c = tri.SpecCache(capacity=4096, auto_install=True)
    yield c
    torch.cuda.synchronize()
    c.close()


def bits(t):
    return t.contiguous().view(torch.uint8 if t.dtype.itemsize == 1 else torch.int32)


def numbers(t):
    """Codes as the numbers they are."""
    return t.to(torch.float32).double().cpu().numpy()


def code_tensor(shape, code, layout):
    """Codes [pages, page, nk, hd] of the layout (as in cache_tensor), the largest ones."""
    n, page, nk, hd = shape
    td, v = CODE[code], 127 if code == "int8" else float("nan")

    def full(*s):
        return torch.full(s, v, dtype=torch.float32, device=DEV).to(td)
    if layout == "slot":
        return full(*shape)
    if layout == "head":
        return full(n, nk, page, hd).transpose(1, 2)
    if layout == "pair":
        return full(n, 2, page, nk, hd)[:, 1]
    return full(n * page * nk * (hd + 3) + 1)[1:].view(n, page, nk, hd + 3)[..., :hd]


def scale_tensor(shape, layout):
    n, blocks, nk = shape
    nan = float("nan")
    if layout in ("slot", "odd"):
        return torch.full(shape, nan, device=DEV)
    if layout == "head":
        return torch.full((n, nk, blocks), nan, device=DEV).transpose(1, 2)
    return torch.full((n, 2, blocks, nk + 1), nan, device=DEV)[:, 1, :, :nk]


def pages_of(lens, page, gen, spare=3):
    """A block table of shuffled pages for requests of lens tokens, and the pool's size."""
    need = [-(-kv // page) for kv, _ in lens]
    cols, pool = max(need + [1]) + 2, sum(need) + spare
    order = torch.randperm(pool, generator=gen, device=DEV).tolist()
    table = [[-1] * cols for _ in lens]
    for r in range(len(lens)):
        for c in range(need[r]):
            table[r][c] = order.pop()
    return table, pool


def problem(dtype, code, lens, nq, nk, hd, page, block, layout="slot", pad=0, seed=0, peak=2.0,
            q_off=0):
    """Attention: requests of lens [(tokens in the cache, new ones of them)] over random codes and
    scales; what is not a request's is poisoned."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    table, pool = pages_of(lens, page, gen)
    shape = (pool, page, nk, hd)
    kc, vc = (code_tensor(shape, code, layout) for _ in range(2))
    ks, vs = (scale_tensor((pool, page // block, nk), layout) for _ in range(2))
    for r, (kv, _) in enumerate(lens):
        for c in range(-(-kv // page)):
            m = min(page, kv - c * page)
            used = -(-m // block)
            for x, s in ((kc, ks), (vc, vs)):
                y = torch.randn((m, nk, hd), generator=gen, device=DEV)
                y = (40 * y).round().clamp(-127, 127) if code == "int8" else (120 * y).clamp(-448, 448)
                x[table[r][c], :m] = y.to(x.dtype)
                y = torch.rand((used, nk), generator=gen, device=DEV)
                s[table[r][c], :used] = (0.5 + y) / (40 if code == "int8" else 120)
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1] + pad
    flat = peak * torch.randn(max(T, 1) * nq * hd + q_off, generator=gen, device=DEV)
    q = flat.to(DT[dtype])[q_off:].view(max(T, 1), nq, hd)[:T]
    return dict(q=q, kc=kc, vc=vc, ks=ks, vs=vs, table=i32(table), kv_len=i32([kv for kv, _ in lens]),
                q_start=i32(starts), scale=hd ** -0.5)


def oracle(p, window=0):
    K, V = (P.values_q8(numbers(p[c]), f64(p[s])) for c, s in (("kc", "ks"), ("vc", "vs")))
    out, written, spread, slack = P.attention(
        f64(p["q"]), K, V, p["table"].cpu().numpy(), p["kv_len"].tolist(), p["q_start"].tolist(),
        float(np.float32(p["scale"])), window, more=2)
    return out, written, spread, slack + 2.0 ** -24


def attend(cache, p, window=0, max_kv=0, out=None, **kw):
    if out is None:
        out = torch.full_like(p["q"], 7.0)
    r = cache.paged_attention_q8(p["q"], p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"],
                                 p["q_start"], p["scale"], window=window, max_kv=max_kv, out=out, **kw)
    torch.cuda.synchronize()
    return r


# ---- the write ---------------------------------------------------------------------------------
def write_problem(dtype, code, lens, nk, hd, page, block, layout="slot", seed=0, spread=2, off=0, pad=0):
    """Rows for requests of lens [(tokens afterwards, new ones of them)]; everything in the
    cache is random, NaN scales and codes among it where nothing is held."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    table, pool = pages_of(lens, page, gen)
    p = problem(dtype, code, [(kv, 0) for kv, _ in lens], 1, nk, hd, page, block, layout, seed=seed)
    assert p["kc"].shape[0] == pool
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1] + pad
    for name in ("k", "v"):
        x = torch.randn((T, nk, hd), generator=gen, device=DEV)
        x = x * 2.0 ** torch.randint(-spread, spread + 1, (T, nk, 1), generator=gen, device=DEV)
        flat = torch.zeros(T * nk * hd + off, device=DEV, dtype=DT[dtype])
        p[name] = flat[off:].view(T, nk, hd)
        p[name].copy_(x)
    p["q_start"] = i32(starts)
    return p


def write(cache, p, **kw):
    r = cache.kv_write_q8(p["k"], p["v"], p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"],
                          p["q_start"], **kw)
    torch.cuda.synchronize()
    assert all(x is y for x, y in zip(r, (p["kc"], p["vc"], p["ks"], p["vs"])))


def written(p, code):
    f32 = lambda t: t.detach().float().cpu().numpy()  # noqa: E731
    return P.kv_write_q8(f64(p["k"]), f64(p["v"]), numbers(p["kc"]), numbers(p["vc"]), f32(p["ks"]),
                         f32(p["vs"]), p["table"].cpu().numpy(), p["kv_len"].tolist(),
                         p["q_start"].tolist(), KIND[code])


def same(p, want):
    for name, w in zip(("kc", "vc", "ks", "vs"), want):
        g = numbers(p[name])
        bad = ~((g == w) | (np.isnan(g) & np.isnan(w)))
        assert not bad.any(), (name, int(bad.sum()), bad.size, g[bad][:5], w[bad][:5])


WRITE_BATCHES = {
    "one token": [(1, 1)],
    "decode": [(1, 1), (17, 1), (64, 1), (65, 1), (200, 1), (33, 1), (48, 1)],
    "prompts": [(5, 5), (70, 70), (1, 1), (33, 33)],
    "chunks": [(100, 30), (64, 64), (300, 129), (31, 1), (257, 2), (40, 0)],
    "empty among": [(0, 0), (40, 0), (0, 0), (50, 9), (20, 0)],
    "short": [(3, 5), (0, 4), (10, 2)],
}


@pytest.mark.parametrize("batch", list(WRITE_BATCHES))
@pytest.mark.parametrize("nk,hd", [(4, 64), (2, 128), (1, 80), (3, 256), (7, 20), (2, 33), (1, 512), (3, 1)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_heads_and_lengths(cache, dtype, code, nk, hd, batch):
    p = write_problem(dtype, code, WRITE_BATCHES[batch], nk, hd, 16, 16, seed=hd + nk)
    want = written(p, code)
    write(cache, p)
    same(p, want)


@pytest.mark.parametrize("layout", ["slot", "head", "odd", "pair"])
@pytest.mark.parametrize("page,block", [(1, 1), (3, 3), (16, 1), (16, 4), (24, 8), (24, 12), (64, 64), (100, 50),
                                        (128, 2)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_pages_blocks_and_layouts(cache, dtype, code, page, block, layout):
    p = write_problem(dtype, code, [(130, 7), (65, 1), (48, 48), (97, 30), (210, 150)], 3, 64, page, block, layout,
                      seed=page + block, pad=3)
    want = written(p, code)
    write(cache, p)
    same(p, want)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_rows_at_any_alignment(cache, dtype, code):
    p = write_problem(dtype, code, WRITE_BATCHES["chunks"], 2, 64, 16, 8, off=1)
    want = written(p, code)
    write(cache, p)
    assert cache.last_selection().variant == P.Q8W_ANY
    same(p, want)
    p = write_problem(dtype, code, WRITE_BATCHES["chunks"], 2, 64, 16, 8)
    for name in ("k", "v"):      # rows in a wider tensor
        wide = torch.full((p[name].shape[0], 2 * 64 + 24), 99.0, dtype=DT[dtype], device=DEV)
        view = wide.as_strided(p[name].shape, (wide.stride(0), 64, 1))
        view.copy_(p[name])
        p[name] = view
    want = written(p, code)
    write(cache, p)
    same(p, want)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd", [32, 20, 7])
def test_write_ties_and_extremes(cache, dtype, code, hd):
    """Quotients in the middle of two codes (the even one), zeros, the smallest and largest
    numbers, and rows whose scale is the least there is."""
    p = write_problem(dtype, code, [(16, 16), (32, 16), (8, 8), (8, 8), (8, 8)], 1, hd, 16, 8)
    most = 127.0 if code == "int8" else 448.0
    i = torch.arange(hd, device=DEV).float()
    k = p["k"].float()
    for t in range(32):
        k[t, 0] = (i - hd // 2) * 4 + t + 0.5
        k[t, 0, 0] = -most               # (a scale of 1)
    if code == "e4m3":
        k[:32, 0, 1:] *= 0.5
        k[3, 0, 1:] = (2 * i[1:] + 1) * 2.0 ** -10
    k[32:40] = 0
    k[33, 0, 2] = -0.0
    k[40:48, 0] = torch.exp2(-140 + 2 * i)[None] if dtype == "f32" else 1e-38
    k[48:56, 0] = -3.3e38 / (1 + i)
    p["k"].copy_(k)
    p["v"].copy_(-3 * k.clamp(-1e38, 1e38))
    want = written(p, code)
    write(cache, p)
    same(p, want)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_write_of_what_is_not_finite(cache, code, bad):
    """The block and head reads as NaN until it is begun anew; its neighbours do not."""
    p = write_problem("bf16", code, [(20, 20), (41, 1), (30, 4)], 2, 64, 16, 8)
    p["k"][3, 1, 5] = bad
    p["v"][20, 0, 0] = bad
    p["k"][22, 1, 63] = bad
    want = written(p, code)
    assert np.isnan(want[2]).sum() > np.isnan(f64(p["ks"])).sum()
    write(cache, p)
    same(p, want)
    # one token more in each: a scale of NaN stays; then all of them begun anew
    p = dict(p, k=p["k"][:3] * 0 + 2, v=p["v"][:3].nan_to_num(0, 0, 0), kv_len=i32([21, 42, 31]),
             q_start=i32([0, 1, 2, 3]))
    want = written(p, code)
    write(cache, p)
    same(p, want)
    p = dict(p, k=torch.ones((93, 2, 64), dtype=torch.bfloat16, device=DEV), kv_len=i32([20, 41, 30]),
             q_start=i32([0, 20, 61, 91]))
    p["v"] = p["k"]
    want = written(p, code)
    write(cache, p)
    same(p, want)
    at = p["table"][0, 0]
    assert torch.isfinite(p["ks"][at]).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_write_token_by_token(cache, dtype, code):
    """A request grown by single tokens, whose blocks' scales grow with them, and the same in
    ragged chunks: every step as the oracle's."""
    p = write_problem(dtype, code, [(50, 50), (50, 50)], 2, 40, 24, 12, spread=4)
    k, v = p["k"].clone(), p["v"].clone()
    for t in range(50):
        q = dict(p, k=torch.stack([k[t], k[50 + t]]), v=torch.stack([v[t], v[50 + t]]),
                 kv_len=i32([t + 1, t + 1]), q_start=i32([0, 1, 2]))
        want = written(q, code)
        write(cache, q)
        same(q, want)
    at = 0
    for n in (1, 2, 13, 24, 10):
        q = dict(p, k=torch.cat([k[at:at + n], k[50 + at:50 + at + n]]),
                 v=torch.cat([v[at:at + n], v[50 + at:50 + at + n]]), kv_len=i32([at + n, at + n]),
                 q_start=i32([0, n, 2 * n]))
        want = written(q, code)
        write(cache, q)
        same(q, want)
        at += n


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("hd", [64, 20])
def test_write_bad_pages_lengths_and_starts(cache, code, hd):
    """Pages outside the pool are skipped, lengths and starts out of range clamped; nothing
    else is written."""
    p = write_problem("bf16", code, [(100, 40), (90, 33)], 2, hd, 16, 8)
    p["table"][0, 4], p["table"][0, 5], p["table"][1, :] = p["kc"].shape[0], -7, 2 ** 31 - 1
    want = written(p, code)
    write(cache, p)
    same(p, want)
    p = write_problem("bf16", code, [(100, 40), (90, 33)], 2, hd, 16, 8)
    for lens, starts in (([2 ** 31 - 1, -5], [0, 40, 73]), ([100, 90], [-4, 40, 2 ** 31 - 1]),
                         ([100, 90], [0, 40, 40]), ([100, 90], [73, 73, 73]), ([100, 90], [-9, -8, -7])):
        q = dict(p, kv_len=i32(lens), q_start=i32(starts))
        want = written(q, code)
        write(cache, q)
        same(q, want)


def test_many_requests(cache):
    """More requests than a round of the search takes, most of a token, some without any."""
    rng = np.random.default_rng(3)
    lens = [(int(rng.integers(1, 40)), 1) if rng.random() < 0.8 else (int(rng.integers(0, 30)), 0)
            for _ in range(700)]
    for code in CODES:
        p = write_problem("bf16", code, lens, 1, 32, 8, 4)
        want = written(p, code)
        write(cache, p)
        same(p, want)
        k, v = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"],
                                p["k"].shape[0])
        read_check(p, k, v, "bf16")


# ---- the read ----------------------------------------------------------------------------------
def read_check(p, k, v, dtype, before=None):
    T = k.shape[0]
    wk, wv, rows = P.kv_read_q8(numbers(p["kc"]), numbers(p["vc"]), f64(p["ks"]), f64(p["vs"]),
                                p["table"].cpu().numpy(), p["kv_len"].tolist(), p["q_start"].tolist(), T)
    for got, want in ((k, wk), (v, wv)):
        # one rounding of the exact product: of 8 by 24 bits, exact in float64
        w = torch.from_numpy(want).to(DT[dtype] if dtype == "f32" else torch.float64)
        if dtype == "bf16":   # (float64 to bf16 in one step)
            g = f64(got)[rows]
            assert (np.abs(g - want[rows]) <= 2.0 ** -8 * np.abs(want[rows])).all()
            continue
        assert (got.cpu()[rows] == w[rows]).all()
    if before is not None:
        assert (f64(k)[~rows] == before).all() and (f64(v)[~rows] == before).all()


@pytest.mark.parametrize("layout", ["slot", "head", "odd", "pair"])
@pytest.mark.parametrize("nk,hd,page,block", [(2, 64, 16, 16), (8, 128, 16, 4), (1, 80, 24, 1), (3, 33, 16, 8),
                                              (1, 512, 3, 3), (5, 1, 128, 64), (3, 24, 100, 50)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_read(cache, dtype, code, nk, hd, page, block, layout):
    lens = [(70, 70), (0, 0), (33, 5), (200, 1), (3, 6)]
    p = problem(dtype, code, lens, 1, nk, hd, page, block, layout, pad=4)
    p["table"][2, 0] = -1
    T = p["q"].shape[0]
    off = 1 if layout == "odd" else 0
    k, v = (torch.full((T * nk * hd + off,), 7.0, dtype=DT[dtype], device=DEV)[off:].view(T, nk, hd)
            for _ in range(2))
    r = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"], T,
                         DT[dtype], k=k, v=v)
    torch.cuda.synchronize()
    assert r[0] is k and r[1] is v
    read_check(p, k, v, dtype, before=7.0)


@pytest.mark.parametrize("code", CODES)
def test_read_of_every_code(cache, code):
    """All 256 bytes, in both types, vector by vector and one by one."""
    b = torch.arange(256, dtype=torch.uint8, device=DEV)
    b = b.view(torch.int8) if code == "int8" else b.view(torch.float8_e4m3fn)
    want = b.float()
    table, n, starts = i32([[0]]), i32([1]), i32([0, 1])
    scale = torch.full((1, 1, 1), 0.75, device=DEV)
    for dtype in DTYPES:
        k, v = cache.kv_read_q8(b.view(1, 1, 1, 256), b.view(1, 1, 1, 256), scale, 2 * scale, table, n, starts,
                                1, DT[dtype])
        assert torch.equal(k.view(-1).nan_to_num(9e9), (want * 0.75).to(k.dtype).nan_to_num(9e9))
        assert torch.equal(v.view(-1).nan_to_num(9e9), (want * 1.5).to(k.dtype).nan_to_num(9e9))
        odd = torch.cat([b.view(torch.uint8)[:1], b.view(torch.uint8)])[1:].view(b.dtype)
        k2, v2 = cache.kv_read_q8(odd.view(1, 1, 1, 256), odd.view(1, 1, 1, 256), scale, 2 * scale, table, n,
                                  starts, 1, DT[dtype])
        assert cache.last_selection().variant == P.Q8R_ANY
        assert torch.equal(bits(k), bits(k2)) and torch.equal(bits(v), bits(v2))


# ---- attention ---------------------------------------------------------------------------------
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("nq,nk,hd", HEADS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_heads_and_lengths(cache, dtype, code, nq, nk, hd, batch):
    p = problem(dtype, code, BATCHES[batch], nq, nk, hd, 16, 8, seed=hd + nq)
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("layout", ["slot", "head", "odd", "pair"])
@pytest.mark.parametrize("page,block", [(1, 1), (3, 3), (16, 1), (16, 16), (24, 8), (24, 2), (64, 32), (100, 50)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_pages_blocks_and_layouts(cache, dtype, code, page, block, layout):
    p = problem(dtype, code, [(130, 7), (65, 1), (48, 48), (97, 1)], 8, 2, 128, page, block, layout, pad=3,
                seed=page)
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("window", [1, 2, 15, 64, 65, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("batch", ["decode", "chunks", "short"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_window(cache, dtype, code, batch, window):
    p = problem(dtype, code, BATCHES[batch], 8, 2, 64, 16, 4, seed=window % 97)
    check(attend(cache, p, window=window), oracle(p, window), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_unaligned_rows_and_in_place(cache, dtype, code):
    p = problem(dtype, code, BATCHES["chunks"], 8, 2, 64, 16, 16, q_off=1)
    check(attend(cache, p), oracle(p), dtype)
    want = oracle(p)
    check(attend(cache, p, out=p["q"]), want, dtype)     # out may be q
    p = problem(dtype, code, BATCHES["chunks"], 8, 2, 64, 16, 16)
    q = torch.zeros((p["q"].shape[0], 8 * 64 + 24), dtype=DT[dtype], device=DEV)
    o = torch.full_like(q, 7.0)
    view = q.as_strided((q.shape[0], 8, 64), (q.stride(0), 64, 1))
    view.copy_(p["q"])
    p["q"] = view
    check(attend(cache, p, out=o.as_strided(view.shape, view.stride())), oracle(p), dtype)
    assert (o[:, 512:] == 7.0).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,nk,hd", [(4, 1, 128), (2, 2, 64), (2, 1, 40)])
@pytest.mark.parametrize("lens", [[(5000, 1)], [(3001, 1), (2, 1), (700, 1)], [(4100, 40)],
                                  [(2500, 3), (0, 0), (1, 1)]])
def test_attention_split_keys(cache, dtype, code, nq, nk, hd, lens):
    p = problem(dtype, code, lens, nq, nk, hd, 16, 16, seed=len(lens), pad=2)
    got = attend(cache, p)
    assert cache.last_selection().n_launches == 2
    want = oracle(p)
    check(got, want, dtype)
    for _ in range(3):
        assert torch.equal(got, attend(cache, p))
    for bound in (1, 100, 600, 10 ** 6):
        check(attend(cache, p, max_kv=bound), want, dtype)
    check(attend(cache, p, window=900), oracle(p, 900), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("hd", [64, 24])
def test_attention_bad_pages_and_lengths(cache, dtype, code, n, hd):
    p = problem(dtype, code, [(200, n), (90, n)], 4, 2, hd, 16, 4)
    p["table"][0, 2] = p["kc"].shape[0]
    p["table"][0, 5] = -7
    p["table"][1, :] = 2 ** 31 - 1                     # no key left
    check(attend(cache, p), oracle(p), dtype)
    assert (f64(attend(cache, p))[n:2 * n] == 0).all()
    p = problem(dtype, code, [(200, n), (90, n)], 4, 2, hd, 16, 4)
    p["kv_len"] = i32([2 ** 31 - 1, -5])
    for c, s in (("kc", "ks"), ("vc", "vs")):
        p[c].copy_(p[c].float().nan_to_num(0.5).to(p[c].dtype))
        p[s].nan_to_num_(0.01)
    check(attend(cache, p), oracle(p), dtype)
    p["kv_len"] = i32([200, 90])
    for starts in ([-4, n, 2 ** 31 - 1], [0, n, n], [n, n, 2 * n], [2 * n, 2 * n, 2 * n],
                   [-9, -8, -7]):
        p["q_start"] = i32(starts)
        check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd", [64, 128, 20])
@pytest.mark.parametrize("lens", [[(100, 100)], [(300, 37), (20, 20)], [(9, 9)]])
def test_attention_nan_in_hidden_places(cache, dtype, code, hd, lens):
    """NaN codes and scales at keys that some rows of a tile see and others must not: rows
    before them are untouched, rows behind take them."""
    p = problem(dtype, code, lens, 4, 2, hd, 16, 1)
    nan = float("nan")
    for i, (r, back) in enumerate([(0, 1), (0, 5), (len(lens) - 1, 3)]):
        x = lens[r][0] - back
        pid = int(p["table"][r, x // 16])
        if code == "e4m3":
            p["vc"][pid, x % 16, i % 2, 3 * i] = torch.tensor(nan, device=DEV).to(CODE[code])
        if i == 1:
            p["ks"][pid, x % 16, 0] = nan
        if i == 2:
            p["vs"][pid, x % 16, 1] = nan
    check(attend(cache, p), oracle(p), dtype)
    check(attend(cache, p, window=4), oracle(p, 4), dtype)
    # in a key that all rows see
    pid = int(p["table"][0, 0])
    p["vs"][pid, 0, 0] = nan
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 50])
def test_attention_special_queries_and_scores(cache, dtype, code, n):
    """Rows with NaN or infinite queries stay alone; scores of -inf weigh nothing, all of them
    -inf give zeros; huge scores do not overflow; scales of 0 and below 0."""
    p = problem(dtype, code, [(120, n)], 4, 2, 64, 16, 8)
    p["q"][0, 1] = float("nan")
    p["q"][n - 1, 2, 5] = float("inf")
    check(attend(cache, p), oracle(p), dtype)
    p = problem(dtype, code, [(120, n)], 4, 2, 64, 16, 8)
    p["q"].abs_()
    p["q"][0] = -float("inf")
    p["kc"].copy_(p["kc"].float().nan_to_num(1.0).abs().clamp(min=1).to(p["kc"].dtype))
    want = oracle(p)
    assert (want[0][0] == 0).all()
    check(attend(cache, p), want, dtype)
    p = problem(dtype, code, [(120, n)], 4, 2, 64, 16, 8, peak=100.0)
    check(attend(cache, p), oracle(p), dtype)
    for scale in (0.0, -0.3):
        p["scale"] = scale
        check(attend(cache, p), oracle(p), dtype)
    p = problem(dtype, code, [(120, n)], 4, 2, 64, 16, 8)   # blocks of zero and negative scales
    p["ks"][int(p["table"][0, 1])] = 0.0
    p["vs"][int(p["table"][0, 2])] *= -1
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("code", CODES)
def test_offsets_beyond_32_bits(cache, code):
    """Codes more than 2^32 bytes into the cache: attention, the write and the read."""
    lens = [(100, 1), (75, 20)]
    p = problem("bf16", code, lens, 8, 2, 128, 16, 16)
    want = oracle(p)
    n, far = p["kc"].shape[0], 600000       # pages of 4 KiB: 2.4 GB of each
    big = torch.zeros((2 * far, 2, 16, 2, 128), dtype=torch.uint8, device=DEV).view(CODE[code])
    scales = torch.zeros((2 * far, 2, 1, 2), device=DEV)
    for i, (c, s) in enumerate((("kc", "ks"), ("vc", "vs"))):
        big[2 * far - n:, i].view(torch.uint8).copy_(p[c].view(torch.uint8))
        scales[2 * far - n:, i] = p[s]
        p[c], p[s] = big[:, i], scales[:, i]
    p["table"] = torch.where(p["table"] >= 0, p["table"] + 2 * far - n, -1).to(torch.int32)
    check(attend(cache, p), want, "bf16")
    k = torch.randn((21, 2, 128), device=DEV).to(torch.bfloat16)
    cache.kv_write_q8(k, -k, p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
    gk, gv = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"], 21)
    torch.cuda.synchronize()
    assert (gk - k).abs().max() < 0.3 and torch.equal(gk[10:], -gv[10:])
    assert (gk[10:].float() / k[10:].float() - 1).abs().median() < 0.05


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,hd,window", [(1, 64, 300), (1, 64, 3000), (1, 20, 300), (150, 64, 300),
                                         (150, 128, 2100)])
def test_attention_at_the_last_position(cache, dtype, code, n, hd, window):
    """2^31 - 4096 keys, the most a request can have; the write and the read of its last rows."""
    page, far = 16, 200
    p = problem(dtype, code, [(far * page, n)], 8, 1, hd, page, 16)
    want = oracle(p, window)
    cols = (1 << 27) - 256
    table = torch.full((1, cols), -1, dtype=torch.int32, device=DEV)
    table[0, cols - far:] = p["table"][0, :far]
    short, p["table"], p["kv_len"] = dict(p), table, i32([cols * page])
    check(attend(cache, p, window), want, dtype)
    k = torch.randn((n, 1, hd), device=DEV).to(DT[dtype])
    short = {**short, **{c: short[c].clone() for c in ("kc", "vc", "ks", "vs")}, "k": k, "v": -k}
    after = written(short, code)
    p["k"], p["v"] = k, -k
    write(cache, p)
    same(p, after)
    gk, gv = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"], n, DT[dtype])
    read_check(short | {c: p[c] for c in ("kc", "vc", "ks", "vs")}, gk, gv, dtype)


# ---- tiles of many rows: every case of these is served by them ------------------------------
TILE_HEADS = [("bf16", 8, 1, 128), ("bf16", 5, 1, 80), ("bf16", 16, 1, 64), ("bf16", 6, 1, 256),
              ("bf16", 10, 2, 96), ("bf16", 33, 3, 48), ("f32", 20, 1, 64), ("f32", 20, 1, 80),
              ("f32", 32, 1, 128), ("f32", 21, 1, 256)]


def tile_problem(dtype, code, lens, nq, nk, hd, page=16, block=8, **kw):
    """A problem whose table is wide: more keys than tiles of few rows serve."""
    p = problem(dtype, code, lens, nq, nk, hd, page, block, **kw)
    wide = torch.full((len(lens), 4200 // page + 1), -1, dtype=torch.int32, device=DEV)
    wide[:, :p["table"].shape[1]] = p["table"]
    return dict(p, table=wide)


def tile_check(cache, p, dtype, window=0, **kw):
    """The result of the form that many rows take: with few tiles and heads of up to 128 in
    bf16 two groups of wavefronts share the keys, else one has them. Rows of nobody make the
    tiles too many for the first; both are compared with the oracle."""
    want = oracle(p, window)
    got = attend(cache, p, window=window, **kw)
    assert cache.last_selection().variant in (P.PA8_TILE, P.PA8_PAIR)
    check(got, want, dtype)
    T, nq, hd = p["q"].shape
    nk = p["kc"].shape[2]
    if dtype == "bf16" and hd <= 128 and cache.last_selection().variant == P.PA8_PAIR:
        more = 300 * 128 * nk // nq
        q = torch.cat([p["q"], torch.zeros((more, nq, hd), dtype=p["q"].dtype, device=DEV)])
        got = attend(cache, dict(p, q=q), window=window)
        assert cache.last_selection().variant == P.PA8_TILE
        assert (got[T:] == 7.0).all()
        check(got[:T], want, dtype)


@pytest.mark.parametrize("batch", list(TILE_BATCHES))
@pytest.mark.parametrize("dtype,nq,nk,hd", TILE_HEADS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("block", [8, 1])
def test_tiles_heads_and_lengths(cache, block, code, dtype, nq, nk, hd, batch):
    tile_check(cache, tile_problem(dtype, code, TILE_BATCHES[batch], nq, nk, hd, block=block, seed=hd), dtype)


@pytest.mark.parametrize("layout", ["slot", "head", "pair"])
@pytest.mark.parametrize("page,block", [(3, 3), (16, 16), (24, 12), (64, 64), (100, 50), (100, 25), (128, 4)])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_tiles_pages_blocks_and_layouts(cache, dtype, code, page, block, layout):
    p = tile_problem(dtype, code, [(300, 129), (65, 40), (200, 30)], 16, 1, 64, page, block, layout=layout, pad=3,
                     seed=page)
    tile_check(cache, p, dtype)


@pytest.mark.parametrize("window", [1, 15, 64, 100, 1000])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block", [16, 2])
def test_tiles_window(cache, dtype, code, block, window):
    p = tile_problem(dtype, code, [(700, 150), (90, 64), (10, 20)], 8, 1, 128, block=block)
    tile_check(cache, p, dtype, window)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_tiles_split_keys(cache, dtype, code, hd):
    """Long contexts before a chunk: split, joined, and the same bits every time."""
    p = problem(dtype, code, [(4300, 40), (2000, 50), (0, 0)], 16, 2, hd, 16, 16, seed=hd, pad=1)
    want = oracle(p)
    got = attend(cache, p)
    assert cache.last_selection().variant in (P.PA8_TILE, P.PA8_PAIR)
    assert cache.last_selection().n_launches == 2
    check(got, want, dtype)
    for _ in range(3):
        assert torch.equal(got, attend(cache, p))
    check(attend(cache, p, window=700), oracle(p, 700), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd", [64, 256])
def test_tiles_nan_in_hidden_places(cache, dtype, code, hd):
    lens = [(300, 137), (220, 120)]
    p = tile_problem(dtype, code, lens, 16, 2, hd, block=1)
    nan = float("nan")
    for i, (r, back) in enumerate([(0, 1), (0, 5), (0, 100), (1, 3), (1, 80)]):
        x = lens[r][0] - back
        pid = int(p["table"][r, x // 16])
        if code == "e4m3":
            p["vc"][pid, x % 16, i % 2, 3 * i] = torch.tensor(nan, device=DEV).to(CODE[code])
        if i == 2:
            p["ks"][pid, x % 16, 0] = nan
        if i in (1, 4):
            p["vs"][pid, x % 16, 1] = nan
    tile_check(cache, p, dtype)
    tile_check(cache, p, dtype, window=90)
    p["q"][3, 1] = nan
    p["q"][50, 9, 5] = float("inf")
    tile_check(cache, p, dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_tiles_bad_pages_and_scores(cache, dtype, code):
    p = tile_problem(dtype, code, [(300, 129), (200, 60)], 16, 2, 64)
    p["table"][0, 2], p["table"][0, 5], p["table"][1, :] = p["kc"].shape[0], -7, 2 ** 31 - 1
    tile_check(cache, p, dtype)
    p = tile_problem(dtype, code, [(300, 129), (200, 60)], 16, 2, 64, peak=100.0)
    tile_check(cache, p, dtype)
    for scale in (0.0, -0.3):
        p = tile_problem(dtype, code, [(300, 129), (200, 60)], 16, 2, 64)
        p["scale"] = scale
        tile_check(cache, p, dtype)
    tile_check(cache, p, dtype, out=p["q"].clone().fill_(7.0))
