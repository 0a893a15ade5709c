"""What the paged ops hand on (CPU): the record of a miss whose install the call
made itself, the choice of streamed loads."""
import ctypes as C

import pytest

from oracle import paged as P
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


@pytest.mark.parametrize("R,T,nq,nk,form", [
    (15, 15 * 64, 32, 8, P.PA_PAIR), (16, 16 * 64, 32, 8, P.PA_TILE),     # 240, 256 equal tiles
    (14, 14 * 60, 32, 8, P.PA_PAIR), (11, 11 * 70, 32, 8, P.PA_TILE),     # 224, 264
    (1, 1024, 32, 8, P.PA_PAIR), (1, 1025, 32, 8, P.PA_TILE),             # 256, 264 of one request
    (22, 800, 32, 8, P.PA_PAIR), (23, 831, 32, 8, P.PA_TILE),             # 288, 296 ragged ones
    (24, 1740, 16, 2, P.PA_PAIR), (3, 1027, 32, 8, P.PA_TILE), (40, 601, 32, 4, P.PA_PAIR), (48, 1301, 32, 4, P.PA_TILE)])
def test_pairs_where_no_unit_gets_two_tiles(lib, fresh, R, T, nq, nk, form):
    c = kv(n_pages=9, nk=nk, hd=128)
    a = attn(L.BF16, T, R, nq, 400, c)
    assert lib.tri_paged_attention(fresh, C.byref(a), None) == 0
    s = last(lib, fresh)
    assert s.variant == form
    assert launches(s) == P.attention_selection(1, T, R, nq, nk, 128, True, 6400, 0)[1]
