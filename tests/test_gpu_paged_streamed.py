"""GPU: attention whose K and V outgrow the last-level cache, by the bound on the
keys that the host has, reads them with nontemporal loads (tiles of 16 rows)."""
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged import (BATCHES, DEV, attend, cache, check, large_oracle,  # noqa: F401
                                  oracle, problem, tri)

pytestmark = pytest.mark.gpu
CACHE = 256 << 20


def streamed(cache, p, dtype, bound=0):
    """The result of a call that the host's rule streams."""
    n, page, nk, hd = p["kc"].shape
    R, cols = p["table"].shape
    T, nq, es = p["q"].shape[0], p["q"].shape[1], 2 if dtype == "bf16" else 4
    keys = min(cols * page, bound or cols * page)
    assert 2 * R * keys * nk * hd * es > CACHE and -(-T // R) * (nq // nk) <= 16
    got = attend(cache, p, max_kv=bound)
    assert cache.last_selection().variant == P.PA_ROWS
    return got


def widen(p, keys):
    """The table with room for `keys` keys, all but the first entries unused."""
    table = p["table"]
    cols = max(keys // p["kc"].shape[1] + 1, table.shape[1])
    wide = torch.full((table.shape[0], cols), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    return dict(p, table=wide)


@pytest.mark.parametrize("layout", ["slot", "head", "pair"])
@pytest.mark.parametrize("batch", ["one token", "decode", "empty among", "short"])
@pytest.mark.parametrize("dtype,nq,nk,hd", [("bf16", 4, 4, 64), ("bf16", 4, 2, 128), ("bf16", 6, 3, 80),
                                             ("bf16", 2, 1, 256), ("bf16", 4, 4, 96), ("f32", 4, 2, 64),
                                             ("f32", 2, 1, 128), ("f32", 2, 2, 256), ("f32", 3, 3, 20)])
def test_streamed_by_the_bound(cache, dtype, nq, nk, hd, batch, layout):  # noqa: F811
    """NaN wherever nothing is stored, as in every problem."""
    p = problem(dtype, BATCHES[batch], nq, nk, hd, 16, layout, seed=hd, pad=1)
    want = oracle(p)
    es, R = 2 if dtype == "bf16" else 4, len(BATCHES[batch])
    p = widen(p, CACHE // (2 * R * nk * hd * es) + 1)
    got = streamed(cache, p, dtype)
    check(got, want, dtype)


@pytest.mark.parametrize("dtype,lens,nq,nk,hd,layout", [
    ("bf16", [(70000, 1)], 16, 8, 128, "slot"), ("bf16", [(70000, 2)], 8, 8, 128, "head"),
    ("bf16", [(66000, 1)], 4, 4, 256, "pair"), ("f32", [(35000, 3)], 8, 4, 256, "slot"),
    ("f32", [(70000, 1)], 8, 8, 64, "head"), ("bf16", [(140000, 1)], 8, 8, 64, "slot")])
def test_streamed_in_full(cache, dtype, lens, nq, nk, hd, layout):  # noqa: F811
    p = problem(dtype, lens, nq, nk, hd, 16, layout, seed=nq)
    got = streamed(cache, p, dtype, lens[0][0])
    check(got, large_oracle(p), dtype)
    assert torch.equal(got, attend(cache, p, max_kv=lens[0][0]))


def test_streamed_many_requests(cache):  # noqa: F811
    """64 requests of 600 to 9000 keys, 1.2 GB: each is what it is alone."""
    lens = [(600 + 133 * i, 1) for i in range(64)]
    p = problem("bf16", lens, 8, 8, 128, 64, seed=1)
    got = streamed(cache, p, "bf16", 9000)
    for r in (0, 1, 17, 40, 63):
        one = dict(p, q=p["q"][r:r + 1], table=p["table"][r:r + 1], kv_len=p["kv_len"][r:r + 1],
                   q_start=torch.tensor([0, 1], dtype=torch.int32, device=DEV))
        check(got[r:r + 1], large_oracle(one), "bf16")
