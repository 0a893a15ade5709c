"""GPU: kv_write_q8 beside the middle of two codes, where the scale's last bit decides."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged import DEV, DT, i32
from tests.test_gpu_paged_q8 import cache, code_tensor, same, scale_tensor, write, written  # noqa: F401

pytestmark = pytest.mark.gpu


def beside_borders(tokens, hd, seed):
    """Rows [tokens, hd] of float32: the largest magnitude a, with a / 127 rounded unlike a times the
    float32 nearest to 1 / 127, then values that lie between the middles of two codes of the one
    scale and of the other (zeros where there are no more)."""
    rng = np.random.default_rng(seed)
    rows = np.zeros((tokens, hd), dtype=np.float32)
    n = np.arange(127) + 0.5
    for t in range(tokens):
        while True:
            a = np.float32(rng.uniform(0.5, 8))
            s, r = a / np.float32(127), a * np.float32(1 / 127)
            if s == r:
                continue
            lo, hi = n * min(np.float64(s), r), n * max(np.float64(s), r)
            x = lo.astype(np.float32)
            x = np.where(np.float64(x) <= lo, np.nextafter(x, np.float32(np.inf)), x)
            x = x[np.float64(x) < hi]
            if len(x):
                break
        assert (np.rint(np.float64(x) / s) != np.rint(np.float64(x) / r)).all()
        x = x[:hd - 1] * rng.choice([-1, 1], len(x[:hd - 1])).astype(np.float32)
        rows[t, 0], rows[t, 1:1 + len(x)] = a, x
    return rows


@pytest.mark.parametrize("hd", [64, 128, 33])
def test_codes_of_a_scale_divided_once(cache, hd):  # noqa: F811
    """An int8 scale is a / 127 rounded once, a code the nearest to x / scale: with a scale off by its
    last bit these values would take the next code."""
    T, page = 400, 16
    rows = beside_borders(T, hd, hd)
    assert (np.abs(rows) > 0).sum() > 2 * T
    pool = T // page
    p = {c: code_tensor((pool, page, 1, hd), "int8", "slot") for c in ("kc", "vc")}
    p.update({s: scale_tensor((pool, page, 1), "slot") for s in ("ks", "vs")})
    x = torch.from_numpy(rows).to(DEV).to(DT["f32"]).view(T, 1, hd)
    p.update(k=x, v=-x, table=i32([list(range(pool))]), kv_len=i32([T]), q_start=i32([0, T]))
    want = written(p, "int8")
    write(cache, p)
    same(p, want)
    # as the definition says it, apart from the oracle
    s = np.abs(rows).max(1) / np.float32(127)
    assert (p["ks"].cpu().numpy().ravel() == s).all()
    codes = np.rint(rows.astype(np.float64) / s[:, None])
    assert (p["kc"].cpu().numpy().reshape(T, hd) == codes).all()
    assert P.CODE_MAX[P.INT8] == np.abs(codes).max()


def beside_ties():
    """(code, scale): e4m3 values and float32 scales below 1 whose product is not in the middle of two
    codes, but the float32 nearest to it is, and the even one of the two is the farther."""
    codes = np.arange(1, 127, dtype=np.uint8)
    v = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    middles = (v[:-1] + v[1:]) / 2
    found = []
    for c in v:
        for m in middles[(middles < c) & (middles > 0.3 * c)]:
            near = np.float32(m / c)
            for s in (np.nextafter(near, np.float32(0)), near, np.nextafter(near, np.float32(1))):
                z = c * np.float64(s)
                if z != m and np.float32(z) == np.float32(m) and s < 1:
                    if P.nearest_code(z, P.E4M3) != P.nearest_code(m, P.E4M3):
                        found.append((c, s))
    return found


@pytest.mark.parametrize("hd", [64, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_held_codes_of_scales_that_are_no_powers_of_two(cache, dtype, hd):  # noqa: F811
    """A block that goes on and whose scale grows to 1: held codes become the nearest to c s, also
    in a cache filled elsewhere, whose e4m3 scales are any numbers."""
    found = beside_ties()
    assert len(found) > 200
    n, page = len(found), 4
    p = {c: code_tensor((n, page, 1, hd), "e4m3", "slot") for c in ("kc", "vc")}
    p.update({s: scale_tensor((n, 1, 1), "slot") for s in ("ks", "vs")})
    held = torch.tensor([c for c, _ in found], dtype=torch.float32, device=DEV).view(n, 1, 1, 1).expand(n, 3, 1, hd)
    scales = torch.from_numpy(np.array([s for _, s in found], dtype=np.float32)).to(DEV).view(n, 1, 1)
    for c, s, sign in (("kc", "ks", 1), ("vc", "vs", -1)):
        p[c][:, :3] = (sign * held).to(p[c].dtype)
        p[s].copy_(scales)
    x = torch.full((n, 1, hd), 448.0, dtype=DT[dtype], device=DEV)
    p.update(k=x, v=x, table=i32([[r] for r in range(n)]), kv_len=i32([4] * n), q_start=i32(list(range(n + 1))))
    want = written(p, "e4m3")
    assert (want[2] == 1).all()
    write(cache, p)
    same(p, want)
