"""What the paged ops hand on (CPU): the record of a miss whose install the call
made itself, the choice of streamed loads."""
import ctypes as C

import pytest

from paper_2609_37241_amd import _lib as L
from tests.native_libs import load_fake
from tests.test_host_paged import at, attn, kv, last, launches, read_args, slots_args


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


def stream_flag(lib, h, *a, **kw):
    """`stream` of the argument block of an attention call's first launch."""
    lib.trifake_reset()
    x = attn(*a, **kw)
    assert lib.tri_paged_attention(h, C.byref(x), None) == 0
    return int.from_bytes(read_args(lib, 0)[1][198:200], "little")


def test_what_outgrows_the_cache_is_streamed(lib, fresh):
    """More than 256 MiB of K and V, by the bound on the keys that the host has,
    read by one tile of 16 rows: nontemporal loads."""
    c = kv(n_pages=9, nk=8, hd=128)
    row = 2 * 8 * 128 * 2                       # bytes of a key, bf16
    most = (1 << 28) // row
    assert stream_flag(lib, fresh, L.BF16, 1, 1, 32, most // 16, c) == 0
    assert stream_flag(lib, fresh, L.BF16, 1, 1, 32, most // 16 + 1, c) == 1
    assert stream_flag(lib, fresh, L.BF16, 4, 4, 32, most // 64 + 1, c) == 1
    assert stream_flag(lib, fresh, L.BF16, 1, 1, 32, 1 << 20, c, max_kv=most) == 0
    assert stream_flag(lib, fresh, L.BF16, 1, 1, 32, 1 << 20, c, window=most + 1) == 1
    # five rows of four heads: two tiles read the keys, the second from the cache
    assert stream_flag(lib, fresh, L.BF16, 4, 1, 32, 1 << 20, c) == 1
    assert stream_flag(lib, fresh, L.BF16, 5, 1, 32, 1 << 20, c) == 0


def test_the_bytes_of_the_largest_caches(lib, fresh):
    """2^64 bytes by the bound on the keys, and more: streamed as any large one."""
    c = kv(n_pages=9, page=65536, nk=4096, hd=256)
    for R, cols in ((2048, 1 << 14), (1024, (1 << 15) - 1), (4095, (1 << 15) - 1)):
        assert stream_flag(lib, fresh, L.F32, 1, R, 4096, cols, c) == 1
