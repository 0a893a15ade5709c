"""CPU: calls of the 8-bit cache's ops that would write K's and V's at one place are refused;
what is only read may be shared."""
import ctypes as C

import pytest

from paper_2609_37241_amd import _lib as L
from tests.test_host_paged_q8 import INVALID, at, attn, fresh, kv, last, lib, q8, rows, stats  # noqa: F401


@pytest.mark.parametrize("kw", [dict(cache=kv(k=at(1), v=at(1))), dict(scales=q8(k_scale=at(7), v_scale=at(7)))])
def test_write_into_one_place(lib, fresh, kw):  # noqa: F811
    h = fresh()
    assert lib.tri_kv_write_quant(h, C.byref(rows(**kw)), None) == INVALID
    assert last(lib, h).status == INVALID and last(lib, h).op == L.OP_KV_WRITE_Q8
    assert lib.trifake_launch_count() == 0 and stats(lib, h)["errors"] == 1
    # read, and attended over, K may be V
    assert lib.tri_kv_read_quant(h, C.byref(rows(**kw)), None) == 0
    a = attn(cache=kw["cache"]) if "cache" in kw else attn()
    assert lib.tri_paged_attention_quant(h, C.byref(a), C.byref(kw.get("scales", q8())), None) == 0


def test_read_into_one_place(lib, fresh):  # noqa: F811
    h = fresh()
    assert lib.tri_kv_read_quant(h, C.byref(rows(k=at(3), v=at(3))), None) == INVALID
    assert last(lib, h).op == L.OP_KV_READ_Q8 and lib.trifake_launch_count() == 0
    # the same rows may be K's and V's of a write
    assert lib.tri_kv_write_quant(h, C.byref(rows(k=at(3), v=at(3))), None) == 0
