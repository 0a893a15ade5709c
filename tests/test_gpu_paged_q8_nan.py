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
