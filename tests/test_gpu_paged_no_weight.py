"""GPU: rows of attention whose scores are all -inf are zero, whatever V holds
at their keys, in each form, split and not."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged import check, f64, oracle
from tests.test_gpu_paged_large_scores import CASES, cache, make, run  # noqa: F401

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def fill(p, name, r, x, value):
    page = p["kc"].shape[1]
    p[name][int(p["table"][r, x // page]), x % page] = value


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("case", list(CASES))
def test_scores_of_minus_infinity_alone(cache, case, bad):  # noqa: F811
    """V holds infinities or NaN at keys that all rows of a tile see and at keys
    that some see; no key has a weight."""
    p, rows = make(case, 7)
    p["q"].abs_().add_(0.5)
    for r, (kv, n) in enumerate(CASES[case][1]):
        for x in range(kv):
            fill(p, "kc", r, x, -INF)
        for x in {0, kv // 3, kv - n, kv - 1}:
            fill(p, "vc", r, x, bad)
    for window in (0, 20):
        assert (run(cache, case, p, window)[:rows] == 0).all()


@pytest.mark.parametrize("case", list(CASES))
def test_the_last_rows_alone_have_a_weight(cache, case):  # noqa: F811
    """The last key of a request has finite scores: the last row is its V (NaN in
    an element where a key of score -inf holds one), the rows before are zero."""
    dtype, lens = CASES[case][:2]
    p, rows = make(case, 8)
    p["q"].abs_().add_(0.5)
    for r, (kv, _) in enumerate(lens):
        for x in range(kv - 1):
            fill(p, "kc", r, x, -INF)
        for x in {0, kv // 3, max(kv - 2, 0)}:
            fill(p, "vc", r, x, 1.0)
            page = p["kc"].shape[1]
            p["vc"][int(p["table"][r, x // page]), x % page, 0, 3] = NAN
    got = run(cache, case, p)
    real = dict(p, q=p["q"][:rows])
    want = oracle({k: v for k, v in real.items() if k != "max_kv"})
    check(torch.from_numpy(got[:rows]), want, dtype)
    starts = p["q_start"].tolist()
    for r, (kv, n) in enumerate(lens):
        assert (got[starts[r]:starts[r + 1] - 1] == 0).all()
        last = got[starts[r + 1] - 1]
        assert np.isnan(last[:, 3]).any() and np.isfinite(np.delete(last, 3, axis=1)).all()


@pytest.mark.parametrize("case", list(CASES))
def test_half_the_keys_have_no_weight(cache, case):  # noqa: F811
    """Scores of -inf in every other 64 keys, so that a group of wavefronts, a
    wavefront or a split may be without any weight."""
    dtype, lens = CASES[case][:2]
    for odd in (0, 1):
        p, rows = make(case, 9)
        p["q"].abs_().add_(0.5)
        for r, (kv, _) in enumerate(lens):
            for x in range(kv):
                if x // 64 % 2 == odd:
                    fill(p, "kc", r, x, -INF)
        got = run(cache, case, p)
        want = oracle({k: v for k, v in dict(p, q=p["q"][:rows]).items() if k != "max_kv"})
        check(torch.from_numpy(got[:rows]), want, dtype)
        assert np.isfinite(f64(torch.from_numpy(got[:rows]))).all()


@pytest.mark.parametrize("gap", [3.0, 60.0, 300.0, 650.0])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("case", list(CASES))
def test_infinities_behind_small_weights(cache, case, back, gap):  # noqa: F811
    """An infinity or NaN in V at a key whose score is `gap` below the largest is
    in the element of each row that sees the key, as it is: also where float32
    has the weight as 0, and whatever the other rows of the tile see. The key is
    an early one, which all rows of a tile see, or one of the last that some
    do not; the largest score is far from it or beside it."""
    dtype, lens = CASES[case][:2]
    hd = CASES[case][4]
    p, rows = make(case, 10)
    p["q"][:] = 1.0
    page = p["kc"].shape[1]
    for far in (True, False):
        q = dict(p, kc=p["kc"].clone(), vc=p["vc"].clone())
        for r, (kv, n) in enumerate(lens):
            for x in range(kv):
                fill(q, "kc", r, x, 0.0)
            marks = sorted({max(kv - n, 0), kv - 1, kv - 1 - n // 2} if back else {0, 1, kv // 4})
            top = (0 if back else kv - n) if far else max(marks[0] - 1, 0)
            if top in marks:
                marks.remove(top)
            fill(q, "kc", r, top, gap / (hd * float(np.float32(p["scale"]))))
            for i, x in enumerate(marks):
                q["vc"][int(q["table"][r, x // page]), x % page, :, i % hd] = (INF, -INF, NAN)[i]
        got = run(cache, case, q)
        want = oracle({k: v for k, v in dict(q, q=q["q"][:rows]).items() if k != "max_kv"})
        check(torch.from_numpy(got[:rows]), want, dtype)
