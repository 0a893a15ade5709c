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
