"""GPU: the paged KV cache's ops against the oracle (float64).

Every slot that no row may see holds NaN: stale slots behind a request's
length, pages of nobody, the table's unused entries. Tolerances are the
oracle's slack (float32 arithmetic) plus, in bf16, half a step (2^-8) of every
weight where it meets V and of the result.
"""
import numpy as np
import pytest
import torch

from oracle import paged as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def tri():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_37241_amd as tri
    return tri


@pytest.fixture(scope="module")
def cache(tri):
    c = tri.SpecCache(capacity=4096, auto_install=True)
    yield c
    torch.cuda.synchronize()
    c.close()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


def cache_tensor(shape, dtype, layout):
    """A cache [pages, page, nk, hd] of NaN: "slot" packed, "head" with a
    page's slots head by head, "odd" one element off a 16-byte boundary in
    rows with a gap, "pair" K's half of a tensor that holds both."""
    n, page, nk, hd = shape
    td = DT[dtype]
    nan = float("nan")
    if layout == "slot":
        return torch.full(shape, nan, dtype=td, device=DEV)
    if layout == "head":
        return torch.full((n, nk, page, hd), nan, dtype=td, device=DEV).transpose(1, 2)
    if layout == "pair":
        return torch.full((n, 2, page, nk, hd), nan, dtype=td, device=DEV)[:, 1]
    buf = torch.full((n * page * nk * (hd + 3) + 1,), nan, dtype=td, device=DEV)
    return buf[1:].view(n, page, nk, hd + 3)[..., :hd]


def problem(dtype, lens, nq, nk, hd, page, layout="slot", pad=0, seed=0, peak=2.0, q_off=0):
    """Requests of lens [(tokens in the cache, new ones of them)] with a block
    table of shuffled pages; NaN wherever nothing is stored."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    td = DT[dtype]
    need = [-(-kv // page) for kv, _ in lens]
    cols, pool = max(need + [1]) + 2, sum(need) + 3
    order = torch.randperm(pool, generator=gen, device=DEV).tolist()
    table = [[-1] * cols for _ in lens]
    shape = (pool, page, nk, hd)
    kc, vc = cache_tensor(shape, dtype, layout), cache_tensor(shape, dtype, layout)
    for r, (kv, _) in enumerate(lens):
        for c in range(need[r]):
            pid = order.pop()
            table[r][c] = pid
            m = min(page, kv - c * page)
            for x in (kc, vc):
                x[pid, :m] = torch.randn((m, nk, hd), generator=gen, device=DEV).to(td)
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1] + pad
    flat = peak * torch.randn(max(T, 1) * nq * hd + q_off, generator=gen, device=DEV)
    q = flat.to(td)[q_off:].view(max(T, 1), nq, hd)[:T]
    return dict(q=q, kc=kc, vc=vc, table=i32(table), kv_len=i32([kv for kv, _ in lens]),
                q_start=i32(starts), scale=hd ** -0.5)


def oracle(p, window=0):
    return P.attention(f64(p["q"]), f64(p["kc"]), f64(p["vc"]), p["table"].cpu().numpy(),
                       p["kv_len"].tolist(), p["q_start"].tolist(),
                       float(np.float32(p["scale"])), window)


def attend(cache, p, window=0, max_kv=0, out=None, **kw):
    if out is None:
        out = torch.full_like(p["q"], 7.0)
    r = cache.paged_attention(p["q"], p["kc"], p["vc"], p["table"], p["kv_len"], p["q_start"],
                              p["scale"], window=window, max_kv=max_kv, out=out, **kw)
    torch.cuda.synchronize()
    return r


def check(got, want, dtype, before=7.0):
    out, written, spread, slack = want
    g = f64(got)
    assert (g[~written] == before).all(), "a row of no request was written"
    g, out, spread, slack = g[written], out[written], spread[written], slack[written]
    fine = np.isfinite(out)
    # infinities and NaN are theirs exactly
    assert (np.isnan(g) == np.isnan(out)).all()
    inf = np.isinf(out)
    assert (g[inf] == out[inf]).all()
    half = HALF[dtype]
    tol = slack[..., None] * spread + half * np.abs(out) + 1e-30
    if dtype == "bf16":
        tol = tol + half * spread
    g, out = np.where(fine, g, 0.0), np.where(fine, out, 0.0)
    bad = ~(np.abs(g - out) <= tol * (1 + 1e-9)) & fine
    assert not bad.any(), (f"{bad.sum()} of {bad.size} off, worst "
                           f"{np.max((np.abs(g - out) / tol)[fine]):.2f} of the tolerance")


HEADS = [(4, 4, 64), (8, 2, 128), (5, 1, 80), (6, 3, 256), (7, 7, 20), (32, 1, 128), (4, 2, 33),
         (20, 4, 96), (2, 1, 512), (3, 1, 1), (9, 3, 72)]
BATCHES = {
    "one token": [(1, 1)],
    "decode": [(1, 1), (17, 1), (64, 1), (65, 1), (200, 1), (33, 1)],
    "prompts": [(5, 5), (70, 70), (1, 1), (33, 33)],
    "chunks": [(100, 30), (64, 64), (300, 129), (31, 1), (257, 2)],
    "empty among": [(0, 0), (40, 0), (0, 0), (50, 9), (20, 0)],
    "short": [(3, 5), (0, 4), (10, 2)],       # fewer tokens in the cache than new ones
}


@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("nq,nk,hd", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_heads_and_lengths(cache, dtype, nq, nk, hd, batch):
    p = problem(dtype, BATCHES[batch], nq, nk, hd, 16, seed=hd + nq)
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("layout", ["slot", "head", "odd", "pair"])
@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 100])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_pages_and_layouts(cache, dtype, page, layout):
    p = problem(dtype, [(130, 7), (65, 1), (48, 48), (97, 1)], 8, 2, 128, page, layout, pad=3,
                seed=page)
    check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("window", [1, 2, 15, 64, 65, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("batch", ["decode", "chunks", "short"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_window(cache, dtype, batch, window):
    p = problem(dtype, BATCHES[batch], 8, 2, 64, 16, seed=window % 97)
    check(attend(cache, p, window=window), oracle(p, window), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_unaligned_rows_and_in_place(cache, dtype):
    p = problem(dtype, BATCHES["chunks"], 8, 2, 64, 16, q_off=1)
    check(attend(cache, p), oracle(p), dtype)
    want = oracle(p)
    check(attend(cache, p, out=p["q"]), want, dtype)     # out may be q
    wide = problem(dtype, BATCHES["chunks"], 8, 2, 64, 16)
    q = torch.zeros((wide["q"].shape[0], 8 * 64 + 24), dtype=DT[dtype], device=DEV)
    o = torch.full_like(q, 7.0)
    view = q[:, :512].view(-1, 8, 64) if q[:, :512].is_contiguous() else \
        q.as_strided((q.shape[0], 8, 64), (q.stride(0), 64, 1))
    view.copy_(wide["q"])
    wide["q"] = view
    out = o.as_strided(view.shape, view.stride())
    check(attend(cache, wide, out=out), oracle(wide), dtype)
    assert (o[:, 512:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,hd", [(4, 1, 128), (2, 2, 64), (2, 1, 40)])
@pytest.mark.parametrize("lens", [[(5000, 1)], [(3001, 1), (2, 1), (700, 1)], [(4100, 40)],
                                  [(2500, 3), (0, 0), (1, 1)]])
def test_attention_split_keys(cache, dtype, nq, nk, hd, lens):
    """Few rows over many keys: split over workgroups and joined; runs without a
    key among them. The same bits on every run."""
    p = problem(dtype, lens, nq, nk, hd, 16, seed=len(lens), pad=2)
    got = attend(cache, p)
    assert cache.last_selection().n_launches == 2
    check(got, oracle(p), dtype)
    for _ in range(3):
        assert torch.equal(got, attend(cache, p))
    # a bound that is wrong steers the split only
    for bound in (1, 100, 600, 10 ** 6):
        check(attend(cache, p, max_kv=bound), oracle(p), dtype)
    check(attend(cache, p, window=900), oracle(p, 900), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("hd", [64, 24])
def test_attention_bad_pages_and_lengths(cache, dtype, n, hd):
    """Pages outside the pool are not seen; lengths and starts out of range are
    clamped; nothing else is read or written."""
    p = problem(dtype, [(200, n), (90, n)], 4, 2, hd, 16)
    p["table"][0, 2] = p["kc"].shape[0]
    p["table"][0, 5] = -7
    p["table"][1, :] = 2 ** 31 - 1                     # no key left
    check(attend(cache, p), oracle(p), dtype)
    assert (f64(attend(cache, p))[n:2 * n] == 0).all()
    p = problem(dtype, [(200, n), (90, n)], 4, 2, hd, 16)
    p["kv_len"] = i32([2 ** 31 - 1, -5])
    for x in (p["kc"], p["vc"]):
        x.nan_to_num_(0.5)
    check(attend(cache, p), oracle(p), dtype)
    p["kv_len"] = i32([200, 90])
    for starts in ([-4, n, 2 ** 31 - 1], [0, n, n], [n, n, 2 * n], [2 * n, 2 * n, 2 * n],
                   [-9, -8, -7]):
        p["q_start"] = i32(starts)
        check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 20])
@pytest.mark.parametrize("lens", [[(100, 100)], [(300, 37), (20, 20)], [(9, 9)]])
def test_attention_infinities_in_hidden_places(cache, dtype, hd, lens):
    """Infinities and NaN in keys that some rows of a tile see and others must
    not: rows before them are untouched by them, rows behind take them."""
    p = problem(dtype, lens, 4, 2, hd, 16)
    inf, nan = float("inf"), float("nan")
    for i, (r, back) in enumerate([(0, 1), (0, 5), (len(lens) - 1, 3)]):
        x = lens[r][0] - back
        pid = int(p["table"][r, x // 16])
        p["vc"][pid, x % 16, i % 2, 3 * i] = (inf, -inf, nan)[i]
        if i == 1:
            p["kc"][pid, x % 16, 0, 2] = nan
    check(attend(cache, p), oracle(p), dtype)
    check(attend(cache, p, window=4), oracle(p, 4), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 50])
def test_attention_special_queries_and_scores(cache, dtype, n):
    """Rows with NaN or infinite queries stay alone; scores of -inf weigh
    nothing, all of them -inf give zeros; huge scores do not overflow."""
    p = problem(dtype, [(120, n)], 4, 2, 64, 16)
    p["q"][0, 1] = float("nan")
    p["q"][n - 1, 2, 5] = float("inf")
    check(attend(cache, p), oracle(p), dtype)
    p = problem(dtype, [(120, n)], 4, 2, 64, 16)
    p["q"].abs_()
    pid = int(p["table"][0, 1])
    p["kc"][pid, 3] = -float("inf")
    check(attend(cache, p), oracle(p), dtype)
    for x in range(120):
        p["kc"][int(p["table"][0, x // 16]), x % 16] = -float("inf")
    want = oracle(p)
    assert (want[0] == 0).all()
    check(attend(cache, p), want, dtype)
    p = problem(dtype, [(120, n)], 4, 2, 64, 16, peak=100.0)
    check(attend(cache, p), oracle(p), dtype)
    for scale in (0.0, -0.3):
        p["scale"] = scale
        check(attend(cache, p), oracle(p), dtype)


def test_attention_offsets_beyond_32_bits(cache):
    """Slots more than 2^32 bytes into the cache, in the slot and head layouts."""
    lens = [(100, 1), (75, 20)]
    p = problem("bf16", lens, 8, 2, 128, 16)
    want = oracle(p)
    n, far = p["kc"].shape[0], 300000       # pages of 8 KiB: 2.4 GB
    big = torch.zeros((2 * far, 2, 16, 2, 128), dtype=torch.bfloat16, device=DEV)
    for i, x in enumerate(("kc", "vc")):
        big[2 * far - n:, i] = p[x]
        p[x] = big[:, i]
    p["table"] = torch.where(p["table"] >= 0, p["table"] + 2 * far - n, -1).to(torch.int32)
    check(attend(cache, p), want, "bf16")
    k = torch.randn((3, 2, 128), device=DEV).to(torch.bfloat16)
    slots = torch.tensor([(2 * far - 1) * 16 + 15, -1, (far - 1) * 16], device=DEV)
    cache.kv_write(k, -k, slots, p["kc"], p["vc"])
    torch.cuda.synchronize()
    assert torch.equal(p["kc"][-1, 15], k[0]) and torch.equal(p["vc"][far - 1, 0], -k[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hd,window", [(1, 64, 300), (1, 64, 3000), (1, 20, 300), (150, 64, 300),
                                         (150, 64, 2100), (150, 128, 2100)])
def test_attention_at_the_last_position(cache, dtype, n, hd, window):
    """2^31 - 4096 keys, the most a request can have, all but the last 3200 in
    one page: a window sees what it sees in those alone."""
    page, far = 16, 200
    p = problem(dtype, [(far * page, n)], 8, 1, hd, page)
    want = oracle(p, window)
    cols = (1 << 27) - 256
    table = torch.full((1, cols), -1, dtype=torch.int32, device=DEV)
    table[0, cols - far:] = p["table"][0, :far]
    p["table"], p["kv_len"] = table, i32([cols * page])
    check(attend(cache, p, window), want, dtype)


# ---- tiles of many rows: every case of these is served by them ------------------------------
TILE_HEADS = [("bf16", 8, 1, 128), ("bf16", 5, 1, 80), ("bf16", 16, 1, 64), ("bf16", 6, 1, 256),
              ("bf16", 10, 2, 96), ("bf16", 33, 3, 72), ("bf16", 130, 1, 8), ("f32", 20, 1, 64),
              ("f32", 20, 1, 80), ("f32", 32, 1, 128), ("f32", 21, 1, 256), ("f32", 80, 2, 20)]
TILE_BATCHES = {
    "prompts": [(70, 70), (33, 33), (64, 64)],
    "chunks": [(100, 30), (0, 0), (300, 129), (31, 1), (257, 60)],
    "short": [(3, 25), (0, 24), (10, 22)],
    "pages end": [(65, 40), (127, 31), (16, 16), (49, 33)],
}


def tile_problem(dtype, lens, nq, nk, hd, page=16, **kw):
    """A problem whose table is wide: more keys than tiles of few rows serve."""
    p = problem(dtype, lens, nq, nk, hd, page, **kw)
    wide = torch.full((len(lens), 4200 // page + 1), -1, dtype=torch.int32, device=DEV)
    wide[:, :p["table"].shape[1]] = p["table"]
    return dict(p, table=wide)


def tile_check(cache, p, dtype, window=0, **kw):
    """The result of the form that many rows take: with few tiles and heads of
    up to 128 in bf16 two groups of wavefronts share the keys, else one has
    them. Both are compared where both can be had: rows of nobody make the
    tiles too many for the first."""
    got = attend(cache, p, window=window, **kw)
    assert cache.last_selection().variant in (P.PA_TILE, P.PA_PAIR)
    if "out" in kw:
        return got
    T, nq, hd = p["q"].shape
    nk, dev = p["kc"].shape[2], p["q"].device
    rows = (256 // nk + 1) * 128 * nk // nq + 1
    q = torch.cat([p["q"], torch.zeros((rows, nq, hd), dtype=p["q"].dtype, device=dev)])
    many = attend(cache, dict(p, q=q), window=window)
    assert cache.last_selection().variant == P.PA_TILE and (f64(many[T:]) == 7.0).all()
    if cache.last_selection().n_launches == 1:
        check(many[:T], oracle(p, window), dtype)
    return got


@pytest.mark.parametrize("batch", list(TILE_BATCHES))
@pytest.mark.parametrize("dtype,nq,nk,hd", TILE_HEADS)
def test_tile_heads_and_lengths(cache, dtype, nq, nk, hd, batch):
    p = tile_problem(dtype, TILE_BATCHES[batch], nq, nk, hd, seed=nq, pad=2)
    check(tile_check(cache, p, dtype), oracle(p), dtype)


@pytest.mark.parametrize("window", [1, 2, 15, 64, 65, 1000])
@pytest.mark.parametrize("batch", ["chunks", "pages end"])
@pytest.mark.parametrize("dtype,nq,nk,hd", [TILE_HEADS[0], TILE_HEADS[7], TILE_HEADS[3]])
def test_tile_window(cache, dtype, nq, nk, hd, batch, window):
    # (a window bounds the keys: rows of nobody make the tiles too many for the other form)
    p = tile_problem(dtype, TILE_BATCHES[batch], nq, nk, hd, seed=window, pad=150)
    check(tile_check(cache, p, dtype, window), oracle(p, window), dtype)


@pytest.mark.parametrize("layout", ["slot", "head", "pair"])
@pytest.mark.parametrize("page", [1, 3, 24, 64, 100])
@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 16, 2, 128), ("f32", 40, 2, 64)])
def test_tile_pages_and_layouts(cache, dtype, nq, nk, hd, page, layout):
    p = tile_problem(dtype, [(130, 40), (65, 30), (48, 48), (97, 1)], nq, nk, hd, page,
                     layout=layout, seed=page)
    if layout == "pair":                    # K and V in one tensor, V of other strides
        p["vc"] = p["vc"].contiguous()
    check(tile_check(cache, p, dtype), oracle(p), dtype)


@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 8, 1, 128), ("bf16", 10, 2, 64), ("f32", 32, 1, 64),
                                             ("bf16", 5, 1, 80), ("f32", 20, 1, 128)])
@pytest.mark.parametrize("lens", [[(100, 100)], [(300, 37), (60, 60)], [(150, 70)]])
def test_tile_infinities_in_hidden_places(cache, dtype, nq, nk, hd, lens):
    p = tile_problem(dtype, lens, nq, nk, hd, pad=150)
    inf, nan = float("inf"), float("nan")
    for i, (r, back) in enumerate([(0, 1), (0, 5), (len(lens) - 1, 33), (0, 36)]):
        x = lens[r][0] - back
        pid = int(p["table"][r, x // 16])
        p["vc"][pid, x % 16, i % nk, 3 * i] = (inf, -inf, nan, inf)[i]
        if i == 1:
            p["kc"][pid, x % 16, 0, 2] = nan
    check(tile_check(cache, p, dtype), oracle(p), dtype)
    check(tile_check(cache, p, dtype, 4), oracle(p, 4), dtype)
    check(tile_check(cache, p, dtype, 40), oracle(p, 40), dtype)


@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 8, 1, 128), ("f32", 32, 1, 64)])
def test_tile_special_values(cache, dtype, nq, nk, hd):
    n = 50
    p = tile_problem(dtype, [(120, n)], nq, nk, hd)
    p["q"][0, 1] = float("nan")
    p["q"][n - 1, 2, 5] = float("inf")
    check(tile_check(cache, p, dtype), oracle(p), dtype)
    p = tile_problem(dtype, [(120, n)], nq, nk, hd)
    p["q"].abs_()
    p["kc"][int(p["table"][0, 1]), 3] = -float("inf")
    check(tile_check(cache, p, dtype), oracle(p), dtype)
    for x in range(120):
        p["kc"][int(p["table"][0, x // 16]), x % 16] = -float("inf")
    got = tile_check(cache, p, dtype)
    assert (f64(got) == 0).all()
    p = tile_problem(dtype, [(120, n)], nq, nk, hd, peak=100.0)
    check(tile_check(cache, p, dtype), oracle(p), dtype)
    for scale in (0.0, -0.3):
        p["scale"] = scale
        check(tile_check(cache, p, dtype), oracle(p), dtype)
    # scores that rise by more than the softmax's reference allows, and fall
    p = tile_problem(dtype, [(120, n)], nq, nk, hd)
    p["q"][:] = 1.0
    for x in range(120):
        p["kc"][int(p["table"][0, x // 16]), x % 16] = 0.3 * (x if x < 100 else 200 - x)
    check(tile_check(cache, p, dtype), oracle(p), dtype)


@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 8, 1, 128), ("f32", 32, 1, 64)])
def test_tile_bad_pages_in_place_and_rows_with_gaps(cache, dtype, nq, nk, hd):
    p = tile_problem(dtype, [(200, 40), (90, 40)], nq, nk, hd)
    p["table"][0, 2], p["table"][0, 5] = p["kc"].shape[0], -7
    p["table"][1, :] = 2 ** 31 - 1
    got = tile_check(cache, p, dtype)
    check(got, oracle(p), dtype)
    assert (f64(got)[40:80] == 0).all()
    p = tile_problem(dtype, [(200, 40), (90, 40)], nq, nk, hd)
    want = oracle(p)
    wide = torch.full((80, nq * hd + 16), 7.0, dtype=DT[dtype], device=DEV)
    view = wide.as_strided((80, nq, hd), (nq * hd + 16, hd, 1))
    view.copy_(p["q"])
    p["q"] = view
    check(tile_check(cache, p, dtype, out=view), want, dtype)      # out is q
    assert (wide[:, nq * hd:] == 7.0).all()
    for starts in ([-4, 40, 2 ** 31 - 1], [0, 40, 40], [40, 40, 80], [80, 80, 80]):
        p["q_start"] = i32(starts)
        check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("R", [63, 64, 65, 130, 1000, 4096])
@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 2, 1, 16), ("bf16", 40, 1, 8), ("f32", 2, 2, 5)])
def test_attention_many_requests(cache, dtype, nq, nk, hd, R):
    """Requests are found among more than a wavefront has lanes."""
    r = np.random.Generator(np.random.PCG64(R))
    new = r.integers(0, 3, R)
    new[r.random(R) < 0.3] = 0
    lens = [(int(n + c), int(n)) for n, c in zip(new, r.integers(0, 12, R))]
    if nq == 40:
        lens = lens[:1000]
    p = problem(dtype, lens, nq, nk, hd, 8, seed=R, pad=1)
    wide = torch.full((len(lens), p["table"].shape[1] + 5), 2 ** 30, dtype=torch.int32, device=DEV)
    wide[:, :-5] = p["table"]
    p["table"] = wide[:, :-5]                       # rows with a gap
    check(attend(cache, p), oracle(p), dtype)


def large_oracle(p, window=0):
    """oracle() in torch's float64 on the GPU, for one request."""
    q, kv = p["q"].double(), int(p["kv_len"][0])
    n, g = q.shape[0], q.shape[1] // p["kc"].shape[2]
    page = p["kc"].shape[1]
    rows = p["table"][0, :-(-kv // page)].long()
    K, V = (p[x][rows].flatten(0, 1)[:kv].double() for x in ("kc", "vc"))
    j = torch.arange(kv, device=DEV)
    pos = torch.arange(kv - n, kv, device=DEV)[:, None]
    hide = (j > pos) | ((j <= pos - window) if window else False)
    out, spread, slack = torch.empty_like(q), torch.empty_like(q), q[..., 0].clone()
    u, hd = 2.0 ** -24, q.shape[2]
    for h in range(q.shape[1]):
        k, v = K[:, h // g].contiguous(), V[:, h // g].contiguous()
        s = (q[:, h].contiguous() @ k.t().contiguous()) * p["scale"]
        big = (q[:, h].abs().contiguous() @ k.abs().t().contiguous()).masked_fill(hide, 0).amax(1)
        top = s.abs().masked_fill(hide, 0).amax(1)
        w = torch.softmax(s.masked_fill(hide, -float("inf")), 1)
        out[:, h], spread[:, h] = w @ v, w @ v.abs()
        slack[:, h] = 2 * (u * (hd + 3) * big * p["scale"] + 4 * u * top) + (2 * kv + 200) * u
    return f64(out), np.ones(n, dtype=bool), f64(spread), f64(slack)


@pytest.mark.parametrize("dtype,kv,n,nq,nk,hd,window,layout", [
    ("bf16", 5000, 3000, 8, 2, 128, 0, "slot"), ("bf16", 2500, 2500, 5, 1, 64, 700, "head"),
    ("bf16", 1500, 1300, 4, 4, 256, 0, "slot"), ("bf16", 9000, 400, 40, 1, 80, 0, "pair"),
    ("f32", 3000, 2000, 4, 2, 128, 0, "head"), ("f32", 1200, 1200, 2, 2, 256, 300, "slot"),
    ("f32", 40000, 1, 8, 2, 64, 0, "slot"), ("bf16", 70000, 2, 8, 1, 96, 0, "slot"),
    ("bf16", 1100, 1000, 3, 1, 33, 0, "odd")])
def test_attention_long_chunks(cache, dtype, kv, n, nq, nk, hd, window, layout):
    p = problem(dtype, [(kv, n)], nq, nk, hd, 16, layout, seed=kv)
    check(attend(cache, p, window=window), large_oracle(p, window), dtype)


@pytest.mark.parametrize("flag", ["jit", "autotune", "generic", "resident_args"])
def test_other_caches_give_the_same(cache, tri, flag):
    other = tri.SpecCache(auto_install=True, **{flag: True})
    for lens in ([(3000, 1)], [(300, 200), (5, 1)]):
        p = problem("bf16", lens, 4, 2, 64, 16)
        assert torch.equal(attend(cache, p), attend(other, p))
    slots_case(other, *SLOT_CASES[3])
    other.close()


# ---- the store -----------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["slot", "head", "odd", "pair"])
@pytest.mark.parametrize("nk,hd", [(8, 128), (1, 64), (3, 80), (2, 33), (5, 1), (40, 256)])
@pytest.mark.parametrize("T", [1, 7, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write(cache, dtype, T, nk, hd, layout):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T)
    page = 24
    n = -(-2 * T // page) + 1
    kc, vc = (cache_tensor((n, page, nk, hd), dtype, layout) for _ in range(2))
    kc.copy_(torch.randn(kc.shape, generator=gen, device=DEV))
    vc.copy_(torch.randn(vc.shape, generator=gen, device=DEV))
    wide = torch.randn((T, 2, nk, hd), generator=gen, device=DEV).to(DT[dtype])
    k, v = wide[:, 0], wide[:, 1]              # rows of a fused projection
    slots = torch.randperm(n * page, generator=gen, device=DEV)[:T]
    if T > 3:
        slots[1], slots[2], slots[3] = -1, n * page, 2 ** 40
    want = P.kv_write(f64(k), f64(v), slots.tolist(), f64(kc), f64(vc))
    cache.kv_write(k, v, slots, kc, vc)
    torch.cuda.synchronize()
    assert (f64(kc) == want[0]).all() and (f64(vc) == want[1]).all()


def test_write_copies_bits_and_takes_either_of_two_rows(cache):
    k = torch.randint(-2 ** 15, 2 ** 15, (64, 4, 64), device=DEV, dtype=torch.int16)
    kc = torch.zeros((8, 16, 4, 64), device=DEV, dtype=torch.int16)
    vc = kc.clone()
    slots = torch.arange(64, device=DEV)
    b = torch.bfloat16
    cache.kv_write(k.view(b), k.flip(0).contiguous().view(b), slots, kc.view(b), vc.view(b))
    torch.cuda.synchronize()
    assert torch.equal(kc.view(-1, 4, 64)[:64], k)
    assert torch.equal(vc.view(-1, 4, 64)[:64], k.flip(0))
    slots[:] = 5                                # one slot for all: a row's vector each
    cache.kv_write(k.view(b), k.view(b), slots, kc.view(b), vc.view(b))
    torch.cuda.synchronize()
    got, rows = kc.view(-1, 4, 8, 8)[5], k.view(64, 4, 8, 8)
    assert (rows == got).all(-1).any(0).all()
    assert torch.equal(kc.view(-1, 4, 64)[6:64], k[6:])


# ---- the bookkeeping ----------------------------------------------------------------------
SLOT_CASES = [
    # kv_len, new_len, page, cols, free, count, T
    ([0], [1], 16, 4, 8, 8, 1),
    ([15, 16, 17, 0], [1, 1, 1, 1], 16, 4, 8, 8, 6),
    ([5, 0, 40, 3], [0, 33, 7, 0], 8, 9, 30, 20, 50),
    ([5, 0, 40, 3], [12, 33, 7, 9], 8, 9, 30, 4, 50),          # the stack runs out
    ([5, 0, 40, 3], [12, 33, 7, 9], 8, 9, 0, 0, 70),           # no stack at all
    ([60, 2], [30, 5], 8, 9, 30, 30, 35),                      # beyond the table
    ([60, 2, 3], [10, 5, 4], 8, 20, 30, 30, 11),               # fewer rows than tokens
    ([-3, 2 ** 31 - 1, 4], [5, 2 ** 31 - 1, -8], 8, 9, 30, 99, 40),   # out of range
    ([0, 0, 0], [0, 0, 0], 8, 9, 30, 30, 5),
    ([7] * 9, [2 ** 30] * 9, 1, 9, 30, -4, 40),                # sums beyond 32 bits
]


def slots_case(cache, kv, new, page, cols, free, count, T, table=None):
    R = len(kv)
    if table is None:
        table = np.arange(R * cols).reshape(R, cols) + 1000
        table[:, cols // 2] = -1
    fp = list(range(500, 500 + free))
    want = P.kv_slots(kv, new, table, fp, count, page, T)
    t = i32(table.tolist())
    got = cache.kv_slots(i32(kv), i32(new), t, i32(fp), i32([count, 123]), page, T)
    torch.cuda.synchronize()
    assert (t.cpu().numpy() == want[0]).all()
    for g, w, name in zip(got, want[1:], ("slots", "pos", "q_start", "kv_len", "free")):
        assert g.tolist() == list(w), name


@pytest.mark.parametrize("case", SLOT_CASES, ids=range(len(SLOT_CASES)))
def test_slots(cache, case):
    slots_case(cache, *case)


@pytest.mark.parametrize("R", [1, 63, 64, 65, 255, 256, 257, 1000, 4096])
def test_slots_many_requests(cache, R):
    r = np.random.Generator(np.random.PCG64(R))
    kv, new = r.integers(0, 300, R), r.integers(0, 9, R)
    new[r.random(R) < 0.3] = 0
    need = int(sum(-(-(a + b) // 16) + (-a // 16) for a, b in zip(kv, new)))
    slots_case(cache, kv.tolist(), new.tolist(), 16, 20, need + 5, need + 5 - (R % 2) * 7,
               int(new.sum()) + R % 3)


def test_slots_without_rows(cache):
    slots_case(cache, [5, 0], [4, 9], 4, 5, 6, 6, 0)


def test_slots_long_prompt(cache):
    slots_case(cache, [100, 5], [20000, 3], 16, 1400, 2000, 2000, 20005)
