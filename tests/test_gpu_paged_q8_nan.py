"""GPU: NaN among the inputs of attention over the 8-bit cache, where a form takes a number
apart or lets several K heads share its products."""
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged import DEV, check
from tests.test_gpu_paged_q8 import CODES, attend, cache, oracle, problem, tile_problem  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0x7F800001, 0xFF800001, 0x7F80FFFF, 0xFF801000, 0x7FC00000])
@pytest.mark.parametrize("scale", [0.125, -0.3])
@pytest.mark.parametrize("form,lens,hd", [("rows", [(1, 1)], 64), ("rows", [(300, 1), (40, 1)], 128),
                                          ("rows", [(3000, 1)], 256), ("tile", [(200, 150)], 64),
                                          ("tile", [(300, 40), (9, 9)], 128), ("any", [(70, 3)], 20)])
@pytest.mark.parametrize("code", CODES)
def test_float32_queries_of_any_nan(cache, code, form, lens, hd, scale, bits):  # noqa: F811
    """A NaN whose bits lie in the lower half alone: taken for an infinity it would give scores of
    -inf at every key of the K head whose codes have the other sign, and zeros for the row."""
    if form == "tile":
        p = tile_problem("f32", code, lens, 16, 2, hd)
    else:
        p = problem("f32", code, lens, 4, 2, hd, 16, 8)
    p["scale"] = scale
    for h, c in ((0, 3), (1, -3)):
        p["kc"][:, :, h, 5] = torch.tensor(float(c), device=DEV).to(p["kc"].dtype)
    p["q"].view(torch.int32)[0, :, 5] = bits - (1 << 32 if bits >> 31 else 0)
    want = oracle(p)
    got = attend(cache, p)
    v = cache.last_selection().variant
    assert v in {"rows": (P.PA8_ROWS,), "tile": (P.PA8_TILE,), "any": (P.PA8_ANY,)}[form]
    assert torch.isnan(got[0]).all() and torch.isfinite(got[1:]).all()
    check(got, want, "f32")


# ---- NaN codes of V where several K heads share a tile's products: other heads' weights of 0 meet them -----
def plant(p, r, key, head, element):
    """A NaN code in V, and where: (request, key, K head, element)."""
    page = p["vc"].shape[1]
    pid = int(p["table"][r, key // page])
    p["vc"][pid, key % page, head, element] = torch.tensor(float("nan"), device=DEV).to(p["vc"].dtype)
    return r, key, head, element


def spoilt(p, planted, window=0):
    """The outputs that see a planted code, from the positions alone: True in [T, nq, hd]."""
    T, nq, hd = p["q"].shape
    g = nq // p["vc"].shape[2]
    out = torch.zeros((T, nq, hd), dtype=torch.bool, device=DEV)
    starts, lens = p["q_start"].tolist(), p["kv_len"].tolist()
    for r, key, head, element in planted:
        for t in range(starts[r], starts[r + 1]):
            at = lens[r] - (starts[r + 1] - t)
            if key <= at and (window == 0 or key > at - window):
                out[t, head * g:(head + 1) * g, element] = True
    return out


def nan_check(cache, p, planted, dtype, heads, window=0, **kw):  # noqa: F811
    got = attend(cache, p, window=window, **kw)
    s = cache.last_selection()
    assert s.variant == P.PA8_ROWS
    # (few requests take one head a tile where they see few keys)
    assert s.key[3] >> 25 & 3 == heads or (len(p["kv_len"]) < 10 and 0 < window <= 1024)
    assert torch.equal(torch.isnan(got), spoilt(p, planted, window))
    check(got, oracle(p, window), dtype)
    return s


SHARED = [(16, 4, 128, 2), (8, 8, 64, 2), (12, 6, 64, 1), (32, 4, 128, 1), (24, 4, 80, 1), (8, 4, 256, 2)]


@pytest.mark.parametrize("nq,nk,hd,heads", SHARED)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_codes_stay_with_their_head(cache, dtype, nq, nk, hd, heads):  # noqa: F811
    """Requests of one part and of many: the element of the rows of the code's own K head alone."""
    lens = [(2300, 1), (1, 1), (0, 0), (513, 1), (700, 1), (0, 1), (40, 1)]
    p = problem(dtype, "e4m3", lens, nq, nk, hd, 16, 8, seed=nq + hd, pad=1)
    planted = [plant(p, 0, 100, 1, 3), plant(p, 0, 2290, nk - 1, hd - 1), plant(p, 4, 650, 0, 17),
               plant(p, 6, 39, 0, 0), plant(p, 6, 0, nk - 1, 9)]
    assert nan_check(cache, p, planted, dtype, heads).n_launches == 2
    for window in (1, 130, 1500):
        nan_check(cache, p, planted, dtype, heads, window)
    nan_check(cache, p, planted, dtype, heads, max_kv=1100)


@pytest.mark.parametrize("nq,nk,hd,heads", [x for x in SHARED if 2 * (x[0] // x[1]) <= 16 >> x[3]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_codes_that_one_row_of_a_tile_sees(cache, dtype, nq, nk, hd, heads):  # noqa: F811
    """Two new tokens: codes at the last key, the one before, and where windows begin."""
    lens = [(2300, 2), (1, 1), (513, 2), (2, 2), (40, 2)]
    p = problem(dtype, "e4m3", lens, nq, nk, hd, 16, 8, seed=nq, pad=1)
    planted = [plant(p, 0, 2299, 1, 3), plant(p, 0, 2298, 0, 5), plant(p, 2, 512, nk - 1, 2),
               plant(p, 3, 1, 0, hd - 1), plant(p, 4, 10, 1, 7), plant(p, 4, 29, nk - 1, 8)]
    for window in (0, 1, 2, 10, 29, 1200):
        nan_check(cache, p, planted, dtype, heads, window)


@pytest.mark.parametrize("nq,nk,hd,heads", [(32, 4, 128, 1), (16, 4, 64, 2), (4, 4, 256, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_codes_in_whole_tiles(cache, dtype, nq, nk, hd, heads):  # noqa: F811
    """Many short requests, several of them a workgroup, no parts: what is done before and after
    a request with such codes stays as it is."""
    lens = [(1 + (37 * i) % 290, 1) for i in range(400)]
    p = problem(dtype, "e4m3", lens, nq, nk, hd, 16, 16, seed=nq)
    clean = attend(cache, p)
    planted = [plant(p, r, lens[r][0] * k // 4, (r + k) % nk, (7 * r + k) % hd)
               for r in (0, 1, 2, 57, 200, 201, 398, 399) for k in range(3)]
    assert nan_check(cache, p, planted, dtype, heads).n_launches == 1
    got, there = attend(cache, p), spoilt(p, planted)
    assert torch.equal(got[~there], clean[~there])
    nan_check(cache, p, planted, dtype, heads, 64)
