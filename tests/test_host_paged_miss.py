"""The record of a miss of the paged ops whose install the call made itself (CPU)."""
import ctypes as C

import pytest

from paper_2609_37241_amd import _lib as L
from tests.native_libs import load_fake
from tests.test_host_paged import at, attn, kv, last, launches, slots_args


@pytest.fixture
def lib():
    return load_fake()


@pytest.fixture
def fresh(lib):
    lib.trifake_reset()
    h = C.c_void_p()
    assert lib.tri_spec_cache_create(C.byref(h), 0, L.AUTO_INSTALL) == 0
    yield h
    lib.tri_spec_cache_destroy(h)


def test_last_miss_after_an_automatic_install(lib, fresh):
    """tri_spec_install_last_miss describes the call that missed, not an earlier
    one, also where the call installed the version and was launched."""
    h, s = fresh, L.Selection()

    def attention(cols, T):
        a = attn(T=T, R=T, cols=cols)
        a.workspace_bytes = lib.tri_paged_attention_workspace(C.byref(a))
        a.workspace = at(31) if a.workspace_bytes else None
        return lib.tri_paged_attention(h, C.byref(a), None)

    calls = [lambda: attention(50, 4), lambda: lib.tri_kv_slots(h, C.byref(slots_args(T=4000)), None),
             lambda: attention(2000, 300), lambda: attention(2000, 1),
             lambda: lib.tri_kv_write(h, L.BF16, at(3), 128, at(4), 128, at(5), 900, C.byref(kv()), None)]
    seen = set()
    for call in calls:
        assert call() == 0
        got = last(lib, h)
        assert lib.tri_spec_install_last_miss(h, C.byref(s)) == 0
        assert tuple(s.key) == tuple(got.key) and s.variant == got.variant
        assert launches(s) == launches(got) and all(g and b for _, g, b in launches(s))
        seen.add(tuple(launches(s)))
    assert len(seen) == len(calls)
