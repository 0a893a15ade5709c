"""The oracle of the paged KV cache in 8 bits against hand-worked cases and bounds (CPU)."""
import numpy as np
import pytest
import torch

from oracle import paged as P


def _e4m3():
    """Every finite value of the type, by its bits."""
    out = []
    for b in range(128):
        e, m = b >> 3, b & 7
        if b != 127:
            out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(sorted(out + [-x for x in out]))


def test_nearest_e4m3_against_all_codes():
    codes = _e4m3()
    assert codes.max() == 448 and len(set(codes)) == 253
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 2.0 ** rng.integers(-14, 6, 4000),
                        codes, (codes[1:] + codes[:-1]) / 2])
    got = P.nearest_code(y, P.E4M3)
    off = np.abs(y[:, None] - codes[None])
    assert np.isin(got, codes).all() and (np.abs(got - y) == off.min(1)).all()
    # the middle of two: the one whose last bit is clear, as torch's own conversion has it
    want = torch.tensor(y, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy()
    assert (got[-len(codes) + 1:] == want[-len(codes) + 1:]).all()


def test_scales_by_hand():
    f = np.float32
    assert P.scale_for(127.0, P.INT8) == 1 and P.scale_for(1.0, P.INT8) == f(1) / f(127)
    assert P.scale_for(448.0, P.E4M3) == 1 and P.scale_for(449.0, P.E4M3) == 2
    assert P.scale_for(448.0 * 2 ** 20, P.E4M3) == 2 ** 20 and P.scale_for(7.0, P.E4M3) == 2.0 ** -6
    assert P.scale_for(7.0000005, P.E4M3) == 2.0 ** -5
    for code in (P.INT8, P.E4M3):
        assert P.scale_for(0.0, code) == f(2.0 ** -100) == P.scale_for(1e-38, code)
        assert np.isnan(P.scale_for(np.inf, code)) and np.isnan(P.scale_for(np.nan, code))


def test_write_by_hand():
    """One head of one element, pages of 4 in blocks of 2: a block begun, one that goes on with
    its scale, one whose scale grows."""
    kc, ks = np.zeros((3, 4, 1, 1)), np.full((3, 2, 1), 9.0, np.float32)
    k = np.array([254.0, 10.0, 127.0]).reshape(3, 1, 1)
    # tokens 0 .. 2 of a request in page 2
    kc, vc, ks, vs = P.kv_write_q8(k, k, kc, kc, ks, ks, [[2]], [3], [0, 3], P.INT8)
    assert kc[2, :, 0, 0].tolist() == [127, 5, 127, 0] and ks[2, :, 0].tolist() == [2, 1]
    # token 3 needs less than its block has, in V twice as much
    new = np.array([[[63.4]]])
    kc, vc, ks, vs = P.kv_write_q8(new, 4 * new, kc, vc, ks, vs, [[2]], [4], [0, 1], P.INT8)
    assert kc[2, 2:, 0, 0].tolist() == [127, 63] and ks[2, 1, 0] == 1
    assert vs[2, 1, 0] == np.float32(4 * 63.4) / np.float32(127)
    assert vc[2, 2:, 0, 0].tolist() == [round(127 / float(vs[2, 1, 0])), 127]
    assert (kc[:2] == 0).all() and (ks[:2] == 9).all()
    # NaN: the block's scale, and zeros
    kc, vc, ks, vs = P.kv_write_q8(new * np.nan, new, kc, vc, ks, vs, [[2]], [4], [0, 1], P.INT8)
    assert np.isnan(ks[2, 1, 0]) and kc[2, 2:, 0, 0].tolist() == [127, 0] and vs[2, 1, 0] < 4
    # rows without a place: before the first token, pages outside the pool
    before = kc.copy()
    for lens, table in (([0], [[1]]), ([2], [[3]]), ([2], [[-1]])):
        assert (P.kv_write_q8(k, k, kc, kc, ks, ks, table, lens, [0, 2], P.INT8)[0] == before).all()


@pytest.mark.parametrize("code", [P.INT8, P.E4M3])
def test_what_a_write_leaves_is_near(code):
    """A prompt in one call: within half a step of every value; token by token: and half a step
    more for each growth (int8), which the powers of two of e4m3 do without."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((64, 2, 8)) * 2.0 ** rng.integers(-2, 3, (64, 1, 1))
    shape, scales = (4, 16, 2, 8), (4, 2, 2)
    at = [[3, 0, 1, 2]]
    state = [np.zeros(shape), np.zeros(shape), np.ones(scales, np.float32), np.ones(scales, np.float32)]
    once = P.kv_write_q8(x, x, *state, at, [64], [0, 64], code)
    got, _, _ = P.kv_read_q8(*once, at, [64], [0, 64], 64)
    step = np.repeat(once[2][at[0]].reshape(8, 2).astype(np.float64), 8, 0)[..., None]   # of each token
    bound = 0.5 * step if code == P.INT8 else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)
    assert (np.abs(got - x) <= bound * (1 + 1e-12)).all()
    for i in range(64):
        state = P.kv_write_q8(x[i:i + 1], x[i:i + 1], *state, at, [i + 1], [0, 1], code)
    assert (state[2] == once[2]).all()
    got, _, _ = P.kv_read_q8(*state, at, [64], [0, 64], 64)
    # up to 7 growths, each of at least 0: half a step each at most
    assert (np.abs(got - x) <= (bound + (3.5 * step if code == P.INT8 else 2.0 ** -10 * step)) * (1 + 1e-12)).all()


def test_read_of_tokens_without_a_place():
    c, s = np.ones((2, 2, 1, 1)), np.full((2, 1, 1), 3.0, np.float32)
    k, v, written = P.kv_read_q8(c, c, s, s, [[1, 5]], [4], [1, 6], 8)
    assert k[:, 0, 0].tolist() == [0, 0, 3, 3, 0, 0, 0, 0]
    assert written.tolist() == [False] + [True] * 5 + [False] * 2
