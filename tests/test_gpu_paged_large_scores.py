"""GPU: attention over pages with scores beyond what float32 resolves.

From about 2^24 on a float32 score is a multiple of one or more, so weights are
compared with what holds whatever the rounding: equal scores weigh the same, a
score that is larger by more than its rounding and the range of a float32 power
takes all, and every result is a mean of the V that its row sees. Each form
(any alignment, tiles of 16 rows, of 128, pairs), with keys split and not.
"""
import numpy as np
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_paged import DEV, DT, HALF, attend, f64, problem, tile_problem

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# dtype, requests (tokens, new ones), nq, nk, hd, the form it takes and whether
# the keys are split
CASES = {
    "any": ("bf16", [(70, 9), (33, 33)], 4, 2, 36, P.PA_ANY, False),
    "any split": ("f32", [(3000, 1)], 2, 1, 33, P.PA_ANY, True),
    "rows": ("bf16", [(70, 3), (41, 1)], 4, 2, 128, P.PA_ROWS, False),
    "rows f32": ("f32", [(70, 9), (33, 33)], 4, 2, 64, P.PA_ROWS, False),
    "rows wide": ("bf16", [(90, 2)], 2, 1, 256, P.PA_ROWS, False),
    "rows split": ("bf16", [(3000, 1)], 4, 1, 128, P.PA_ROWS, True),
    "rows split f32": ("f32", [(2500, 2)], 4, 1, 64, P.PA_ROWS, True),
    "pair": ("bf16", [(150, 70), (64, 64)], 8, 1, 128, P.PA_PAIR, False),
    "pair split": ("bf16", [(2100, 70)], 8, 1, 64, P.PA_PAIR, True),
    "tile": ("bf16", [(150, 70), (64, 64)], 8, 1, 128, P.PA_TILE, False),
    "tile wide": ("bf16", [(150, 70)], 8, 1, 256, P.PA_TILE, False),
    "tile f32": ("f32", [(150, 70)], 32, 1, 64, P.PA_TILE, False),
    "tile split f32": ("f32", [(1200, 70)], 32, 1, 64, P.PA_TILE, True),
}


@pytest.fixture(scope="module")
def cache():
    import paper_2609_37241_amd as tri
    c = tri.SpecCache(capacity=1024, auto_install=True)
    yield c
    torch.cuda.synchronize()
    c.close()


def make(case, seed):
    dtype, lens, nq, nk, hd, form, split = CASES[case]
    p = (tile_problem if form in (P.PA_TILE, P.PA_PAIR) else problem)(dtype, lens, nq, nk, hd, 16,
                                                                     seed=seed)
    rows = p["q"].shape[0]
    if split:
        return p, rows
    if form in (P.PA_TILE, P.PA_PAIR):      # rows of nobody: as many tiles as leave none to split
        more = (200 if form == P.PA_PAIR else 260) * 128 // nq
        p["q"] = torch.cat([p["q"], torch.zeros((more, nq, hd), dtype=DT[dtype], device=DEV)])
    else:
        p["max_kv"] = 1
    return p, rows


def run(cache, case, p, window=0):
    form, split = CASES[case][5:]
    got = attend(cache, {k: v for k, v in p.items() if k != "max_kv"}, window=window,
                 max_kv=p.get("max_kv", 0))
    s = cache.last_selection()
    if not window:      # (a window bounds the keys, which bounds the splits)
        assert (s.variant, s.n_launches) == (form, 1 + split)
    return f64(got)


def seen(p, window=0):
    """(row, K head, keys [n, hd], values [n, hd], query heads) of every row."""
    kc, vc, table = f64(p["kc"]), f64(p["vc"]), p["table"].cpu().numpy()
    page, nk = kc.shape[1:3]
    g = p["q"].shape[1] // nk
    starts = p["q_start"].tolist()
    for r, kv in enumerate(p["kv_len"].tolist()):
        for t in range(starts[r], starts[r + 1]):
            at = kv - (starts[r + 1] - t)
            x = np.arange(max(0, at - window + 1) if window else 0, at + 1)
            for h in range(nk):
                where = table[r, x // page], x % page, h
                yield t, kc[where], vc[where], slice(h * g, (h + 1) * g)


@pytest.mark.parametrize("value,scale", [(24576.0, None), (40960.0, None), (1.0e4, 1e28),
                                         (2.0, 3e38), (-2.0, -3e38), (1.5, 3.4e38), (300.0, 1e-44)])
@pytest.mark.parametrize("case", list(CASES))
def test_equal_scores_give_the_mean(cache, case, value, scale):
    """All products of a row are the same sum of the same numbers, so every
    weight is the same power of two's rounding, 1 where it is the maximum's:
    the mean of V to 2 n + 200 roundings of float32 (the oracle's count for
    powers and sums) and one to the dtype."""
    dtype = CASES[case][0]
    p, _ = make(case, 1)
    p["q"][:] = value
    p["kc"].nan_to_num_(0.0).fill_(abs(value))
    if scale is not None:
        p["scale"] = scale
    for window in (0, 50):
        got = run(cache, case, p, window)
        for t, _, v, heads in seen(p, window):
            mean, size = v.mean(0), np.abs(v).mean(0)
            tol = (2 * len(v) + 200) * U * size + HALF[dtype] * np.abs(mean) + 1e-30
            assert (np.abs(got[t, heads] - mean) <= tol).all(), (t, window)


@pytest.mark.parametrize("size", [1e3, 3e4, 1e6, 1e9])
@pytest.mark.parametrize("case", list(CASES))
def test_the_largest_score_takes_all(cache, case, size):
    """Random large scores: a row whose largest exceeds the next by more than
    the rounding of both and 2^8 (a float32 power ends at 2^-150) is that key's
    V; any other is a mean of what it sees, within the bounds of V and their
    rounding (2 n + 200 roundings of the sums; bf16: half a step of every weight
    and of the result)."""
    dtype = CASES[case][0]
    p, rows = make(case, 2)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    p["q"].copy_(size * torch.randn(p["q"].shape, generator=gen, device=DEV))
    p["kc"].copy_(torch.where(p["kc"].isnan(), p["kc"], p["kc"] * size))
    p["vc"].copy_(torch.where(p["vc"].isnan(), p["vc"], p["vc"].abs() + 1))
    got = run(cache, case, p)
    q, hd = f64(p["q"]), CASES[case][4]
    scale, clear = float(np.float32(p["scale"])), 0
    half = HALF[dtype]
    for t, k, v, heads in seen(p):
        for h in range(heads.start, heads.stop):
            s = (k * q[t, h]).sum(-1) * scale
            off = U * (hd + 4) * (np.abs(k) * np.abs(q[t, h])).sum(-1).max() * abs(scale)
            i = int(s.argmax())
            rest = np.delete(s, i)
            if not len(rest) or s[i] - rest.max() > 2 * off + 256:
                assert (np.abs(got[t, h] - v[i]) <= 4 * U * v[i]).all(), (t, h)
                clear += 1
            else:
                slack = 2 * half + (2 * len(v) + 200) * U
                assert (got[t, h] >= v.min(0) * (1 - slack)).all(), (t, h)
                assert (got[t, h] <= v.max(0) * (1 + slack)).all(), (t, h)
    if size >= 3e4:
        assert clear > rows * q.shape[1] // 2


@pytest.mark.parametrize("case", list(CASES))
def test_a_scale_of_zero_or_nearly(cache, case):
    """Scores that the scale makes 0 weigh the same, however large the
    products are (1e37: differences that 1e-36 would still see)."""
    dtype = CASES[case][0]
    for scale in (0.0, 1e-45, -1e-45):
        p, _ = make(case, 4)
        p["q"].copy_(torch.where(p["q"] > 0, 1e18, -1e18))
        p["kc"].copy_(torch.where(p["kc"].isnan(), p["kc"], torch.where(p["kc"] > 0, 1e17, -1e17)))
        p["scale"] = scale
        got = run(cache, case, p)
        # |scale q.k| <= 1e-45 * 512 * 1e35: below 2^-24, so weights are 1 to a
        # few roundings; in bf16 exactly 1 or half a step below, of each
        for t, _, v, heads in seen(p):
            mean, size = v.mean(0), np.abs(v).mean(0)
            tol = (2 * len(v) + 200) * U * size + HALF[dtype] * np.abs(mean) + 1e-30
            if dtype == "bf16":
                tol = tol + HALF[dtype] * size
            assert (np.abs(got[t, heads] - mean) <= tol).all(), (t, scale)


@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("case", list(CASES))
def test_scores_that_grow_by_steps(cache, case, falling):
    """Scores of 1 at a row's first key that grow by a quarter from key to key
    (or fall so): small and huge ones in one row, references of every size."""
    dtype = CASES[case][0]
    p, _ = make(case, 5)
    p["q"][:] = 1.0
    page = p["kc"].shape[1]
    table = p["table"].cpu()
    for r, kv in enumerate(p["kv_len"].tolist()):
        for x in range(kv):
            e = min((kv - 1 - x) if falling else x, 110)
            p["kc"][int(table[r, x // page]), x % page] = 1.25 ** e
    p["vc"].copy_(torch.where(p["vc"].isnan(), p["vc"], p["vc"].abs() + 1))
    got = run(cache, case, p)
    scale, hd = float(np.float32(p["scale"])), CASES[case][4]
    for t, k, v, heads in seen(p):
        s = k.sum(-1) * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        # scores are off by hd + 4 roundings of themselves; where that is more
        # than 2^-8 only what exceeds it by 256 is compared
        off = U * (hd + 4) * s.max()
        ties = s >= s.max() - 2 * off - 256
        if off > 2.0 ** -8:
            lo, hi = v[ties].min(0), v[ties].max(0)
            slack = 2 * HALF[dtype] + (2 * len(v) + 200) * U
            assert (got[t, heads] >= lo * (1 - slack)).all() and (got[t, heads] <= hi * (1 + slack)).all()
        else:
            want, rel = (w[:, None] * v).sum(0), 2 * off + (2 * len(v) + 200) * U
            rel += HALF[dtype] * (2 if dtype == "bf16" else 1)
            assert (np.abs(got[t, heads] - want) <= rel * np.abs(want)).all(), t
