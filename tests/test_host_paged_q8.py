"""The paged cache in 8 bits in the native cache core (CPU, recording backend):
refusals, selections against the model, argument blocks, misses, keys, statistics."""
import ctypes as C
import os
import random
import subprocess
import sys

import pytest

from oracle import paged as P
from paper_2609_37241_amd import _lib as L
from tests.native_libs import load_fake
from tests.test_host_paged import (ATTN_REFUSALS, at, attn, kv, last, launches, read_args, stats)
from tests.test_host_sanitized import ROOT, _runtime

INVALID, UNSUPPORTED = L.E_INVALID, L.E_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return load_fake()


@pytest.fixture
def fresh(lib):
    caches = []

    def make(capacity=0, flags=L.AUTO_INSTALL):
        lib.trifake_reset()
        h = C.c_void_p()
        assert lib.tri_spec_cache_create(C.byref(h), capacity, flags) == 0
        caches.append(h)
        return h
    yield make
    for h in caches:
        lib.tri_spec_cache_destroy(h)


def q8(code=L.INT8, page=16, block=16, nk=2, **kw):
    n = page // block if block > 0 else 1
    x = dict(code=code, block=block, k_scale=at(7), v_scale=at(8), k_ps=n * nk, k_bs=nk, k_hs=1,
             v_ps=n * nk, v_bs=nk, v_hs=1)
    x.update(kw)
    return L.KvQ8(**x)


def rows(dtype=L.BF16, T=8, R=3, cols=10, cache=None, scales=None, **kw):
    c = cache if cache is not None else kv()
    w = c.nk * c.hd
    x = dict(dtype=dtype, R=R, T=T, k=at(3), k_ts=w, v=at(4), v_ts=w, table=at(22), table_rs=cols,
             kv_len=at(23), q_start=at(24), cols=cols, kv=c,
             q8=scales if scales is not None else q8(page=max(c.page, 1), block=max(c.page, 1), nk=c.nk))
    x.update(kw)
    return L.KvRowsArgs(**x)


def both(lib):
    return (lib.tri_kv_write_quant, lib.tri_kv_read_quant)


# ---- refusals ------------------------------------------------------------------------------
SCALE_REFUSALS = [
    dict(code=2), dict(code=-1), dict(block=0), dict(block=-16), dict(block=3), dict(block=32),
    dict(k_scale=None), dict(v_scale=None), dict(k_scale=at(7, 2)), dict(v_scale=at(8, 1)),
    dict(k_ps=1), dict(k_ps=-2), dict(v_hs=0), dict(v_hs=-1), dict(v_ps=0), dict(k_ps=1 << 60),
    dict(block=4, k_bs=1), dict(block=4, v_ps=7), dict(block=4, v_bs=0),
]


@pytest.mark.parametrize("kw", SCALE_REFUSALS, ids=range(len(SCALE_REFUSALS)))
def test_scale_refusals(lib, fresh, kw):
    h = fresh()
    s = q8(**kw)
    for f in both(lib):
        assert f(h, C.byref(rows(scales=s)), None) == INVALID
    assert lib.tri_paged_attention_quant(h, C.byref(attn()), C.byref(s), None) == INVALID
    assert lib.trifake_launch_count() == 0 and stats(lib, h)["errors"] == 3


@pytest.mark.parametrize("kw", [
    dict(block=1), dict(block=8), dict(k_ps=9, v_ps=64), dict(k_hs=100, k_ps=1),   # pages innermost
    dict(block=4, k_bs=1, k_hs=4, v_bs=100, v_ps=400), dict(k_bs=-3, v_bs=0)])     # one block a page
def test_scale_layouts_taken(lib, fresh, kw):
    h = fresh()
    s = q8(**kw)
    for f in both(lib):
        assert f(h, C.byref(rows(scales=s)), None) == 0
    assert lib.tri_paged_attention_quant(h, C.byref(attn()), C.byref(s), None) == 0


ROWS_REFUSALS = [
    (dict(dtype=2), INVALID), (dict(T=-1), INVALID), (dict(T=(1 << 22) + 1), UNSUPPORTED),
    (dict(R=0), INVALID), (dict(R=4097), UNSUPPORTED), (dict(cols=0), INVALID),
    (dict(cols=1 << 27, table_rs=1 << 27), UNSUPPORTED), (dict(table=None), INVALID),
    (dict(table=at(22, 2)), INVALID), (dict(table_rs=9), INVALID), (dict(table_rs=1 << 60), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(kv_len=None), INVALID),
    (dict(q_start=None), INVALID), (dict(k=at(3, 1)), INVALID), (dict(v=at(4, 1)), INVALID),
    (dict(kv_len=at(23, 2)), INVALID), (dict(q_start=at(24, 1)), INVALID), (dict(k_ts=127), INVALID),
    (dict(v_ts=-128), INVALID), (dict(v_ts=1 << 60), INVALID),
    (dict(cache=kv(n_pages=0)), INVALID), (dict(cache=kv(page=65537)), UNSUPPORTED),
    (dict(cache=kv(hd=513)), UNSUPPORTED), (dict(cache=kv(k=None)), INVALID),
    (dict(cache=kv(k_hs=63)), INVALID), (dict(cache=kv(v_ps=16 * 128 - 1)), INVALID),
    (dict(cache=kv(v_ps=1 << 47)), INVALID),
]


@pytest.mark.parametrize("kw,want", ROWS_REFUSALS, ids=range(len(ROWS_REFUSALS)))
def test_rows_refusals(lib, fresh, kw, want):
    h = fresh()
    for f, op in zip(both(lib), (L.OP_KV_WRITE_Q8, L.OP_KV_READ_Q8)):
        assert f(h, C.byref(rows(**kw)), None) == want
        assert last(lib, h).status == want and last(lib, h).op == op
    assert lib.trifake_launch_count() == 0 and stats(lib, h)["errors"] == 2


@pytest.mark.parametrize("kw,want", ATTN_REFUSALS, ids=range(len(ATTN_REFUSALS)))
def test_attention_refusals(lib, fresh, kw, want):
    h = fresh()
    assert lib.tri_paged_attention_quant(h, C.byref(attn(**kw)), C.byref(q8()), None) == want
    assert lib.trifake_launch_count() == 0 and last(lib, h).status == want


def test_edges(lib, fresh):
    h = fresh()
    for f in both(lib):
        assert f(None, C.byref(rows()), None) == INVALID
        assert f(h, None, None) == INVALID
        assert f(h, C.byref(L.KvRowsArgs(dtype=L.BF16, T=0)), None) == 0
        # codes lie at any address; the largest of all
        assert f(h, C.byref(rows(cache=kv(k=at(1, 1), v=at(2, 3), k_ps=16 * 128 + 1))), None) == 0
        assert f(h, C.byref(rows(T=1 << 22, R=4096, cols=32767, cache=kv(page=65536, nk=4096, hd=512))),
                 None) == 0
    f = lib.tri_paged_attention_quant
    assert f(None, C.byref(attn()), C.byref(q8()), None) == INVALID
    assert f(h, None, C.byref(q8()), None) == INVALID and f(h, C.byref(attn()), None, None) == INVALID
    assert f(h, C.byref(L.AttentionArgs(dtype=L.F32, T=0)), None, None) == 0
    size = lib.tri_paged_attention_quant_workspace
    assert size(None) == 0 and size(C.byref(attn(nq=7))) == 0
    assert size(C.byref(L.AttentionArgs(dtype=L.F32, T=0))) == 0
    assert size(C.byref(attn(cols=(1 << 27) - 255))) == 0
    assert lib.trifake_launch_count() == 4
    assert f(h, C.byref(attn(cols=(1 << 27) - 256, table_rs=1 << 27)), C.byref(q8()), None) == 0


def test_attention_beyond_a_launch(lib, fresh):
    """2^24 rows of heads of 9 (no tiles) go round; tiles of many rows, 2^32 work-items
    and more, do not fit."""
    h = fresh()
    c = kv(nk=4096, hd=16, page=1)
    s = q8(page=1, block=1, nk=4096)
    big = attn(L.F32, 1 << 18, 4096, 4096, 9, c)
    assert lib.tri_paged_attention_quant(h, C.byref(big), C.byref(s), None) == UNSUPPORTED
    assert lib.trifake_launch_count() == 0
    c = kv(nk=4096, hd=9, page=1)
    ok = attn(L.F32, 1 << 18, 4096, 4096, 9, c)
    assert lib.tri_paged_attention_quant(h, C.byref(ok), C.byref(s), None) == 0


# ---- selections ----------------------------------------------------------------------------
def test_rows_selection(lib, fresh):
    h = fresh(4096)
    r = random.Random(1)
    teams = set()
    for i in range(4000):
        if i % 2000 == 1999:
            h = fresh(4096)
        dt, code = r.choice([0, 1]), r.choice([0, 1])
        T, R = r.choice([1, 3, 64, 300, 8192, 16384, 70000, 1 << 22]), r.choice([1, 2, 16, 300, 4096])
        nk, hd = r.choice([1, 2, 3, 8, 40]), r.choice([1, 20, 33, 64, 80, 128, 512])
        page = r.choice([1, 16, 24, 64, 256])
        block = r.choice([b for b in (1, 8, 16, 24, 256) if page % b == 0])
        off, back = r.choice([0, 0, 16, 4]), r.choice([0, 0, 0, 8, 4, 2, 1])
        es = 2 if dt else 4
        c = kv(n_pages=9, page=page, nk=nk, hd=hd, k=at(1, back))
        a = rows(dt, T, R, 3, c, q8(code, page, block, nk), k=at(3, off))
        codes = 16 // es                      # bytes of a vector's codes
        aligned = off % 16 == 0 and (T == 1 or nk * hd * es % 16 == 0) and back % codes == 0 \
            and page * nk * hd % codes == 0 and (page == 1 or nk * hd % codes == 0) \
            and (nk == 1 or hd % codes == 0)
        for f, op in zip(both(lib), (P.OP_KV_WRITE_Q8, P.OP_KV_READ_Q8)):
            assert f(h, C.byref(a), None) == 0
            key, want = P.kv_rows_q8_selection(op, dt, code, T, R, nk, hd, block, aligned)
            s = last(lib, h)
            assert tuple(s.key) == key and launches(s) == want
            teams.add((op, want[0][0], key[3] >> 16 & 3))
    w, x = P.OP_KV_WRITE_Q8, P.OP_KV_READ_Q8
    assert teams == {(w, P.Q8W_ANY, 0), (x, P.Q8R_ANY, 0), (x, P.Q8R_VEC, 0)} | \
        {(w, P.Q8W_VEC, t) for t in range(3)}


def test_attention_selection(lib, fresh):
    h = fresh(4096)
    r = random.Random(2)
    forms = set()
    for i in range(8000):
        if i % 2000 == 1999:
            h = fresh(4096)
        dt, code, nk = r.choice([0, 1]), r.choice([0, 1]), r.choice([1, 2, 3, 8, 12])
        nq, hd = nk * r.choice([1, 2, 4, 5, 40]), r.choice([1, 20, 24, 64, 80, 128, 256, 320, 512])
        R = r.choice([1, 2, 16, 300, 4096])
        T = min(1 << 22, R * r.choice([1, 1, 1, 2, 4, 16, 200]) + r.choice([0, 0, 3]))
        page, cols = r.choice([1, 16, 100]), r.choice([1, 7, 300, 20000])
        off, back, es = r.choice([0, 0, 0, 8]), r.choice([0, 0, 0, 8]), 2 if dt else 4
        window, bound = r.choice([0, 0, 5, 3000]), r.choice([0, 0, 1, 2000, 10 ** 9])
        c = kv(n_pages=9, page=page, nk=nk, hd=hd, v=at(2, back))
        a = attn(dt, T, R, nq, cols, c, q=at(20, off), window=window, max_kv=bound)
        keys = min(x for x in (cols * page, bound or 1 << 40, window or 1 << 40))
        aligned = off == 0 and back == 0 and (T == 1 or nq * hd * es % 16 == 0) \
            and nk * hd * page % 16 == 0 and (page == 1 or nk * hd % 16 == 0) \
            and (nk == 1 or hd % 16 == 0)
        need = lib.tri_paged_attention_quant_workspace(C.byref(a))
        plan = P.attention_q8_plan(dt, T, R, nq, nk, hd, aligned, keys, cols * page, 1 << 62)
        assert need == P.attention_workspace(T, nq, hd, plan[1])
        forms.add((plan[0], plan[1] > 1, plan[4]))
        given = r.choice([0, need // 2, need, need + 100])
        if given:
            a.workspace, a.workspace_bytes = at(31), given
        form, _, grids, block, _, _ = P.attention_q8_plan(dt, T, R, nq, nk, hd, aligned, keys, cols * page,
                                                          given)
        too_many = form > 1 and grids[0] * block >= 1 << 32
        s = q8(code, page, page, nk)
        want = UNSUPPORTED if too_many else 0
        assert lib.tri_paged_attention_quant(h, C.byref(a), C.byref(s), None) == want
        if too_many:
            continue
        key, want = P.attention_q8_selection(dt, code, T, R, nq, nk, hd, aligned, keys, cols * page, given)
        got = last(lib, h)
        assert tuple(got.key) == key and launches(got) == want
    assert forms == {(f, s, 0) for f in range(4) for s in (False, True)} | \
        {(1, s, x) for s in (False, True) for x in (1, 2)}


def test_rows_argument_block(lib, fresh):
    h = fresh()
    c = kv(page=24, nk=2, hd=40)
    a = rows(L.F32, 300, 5, 9, c, q8(L.E4M3, 24, 8, 2, v_ps=100), v_ts=96)
    assert lib.tri_kv_write_quant(h, C.byref(a), None) == 0
    v, raw, _ = read_args(lib, 0)
    word = lambda i, n=4: int.from_bytes(raw[i:i + n], "little", signed=True)  # noqa: E731
    assert v == P.Q8W_VEC
    assert [word(8 * i, 8) for i in range(2)] == [at(3), at(4)]
    assert [word(16 + 8 * i, 8) for i in range(8)] == [at(1), 1920, 80, 40, at(2), 1920, 80, 40]
    assert [word(80 + 8 * i, 8) for i in range(8)] == [at(7), 6, 2, 1, at(8), 100, 2, 1]
    assert [word(144 + 8 * i, 8) for i in range(6)] == [at(22), at(23), at(24), 80, 96, 9]
    assert [word(192 + 4 * i) for i in range(8)] == [300, 5, 9, 100, 24, 2, 40, 8]
    # vectors of a row; 300 / 8 + 10 blocks, fewer than rows; every head for itself
    assert [word(248 + 4 * i) for i in range(4)] == [10, 47, 0, 1]


def test_attention_argument_block(lib, fresh):
    h = fresh()
    a = attn(L.F32, T=3, R=2, nq=16, cols=500, cache=kv(nk=4, hd=128), scale=-0.25)
    need = lib.tri_paged_attention_quant_workspace(C.byref(a))
    a.workspace, a.workspace_bytes = at(31), need
    s = q8(L.INT8, 16, 4, 4)
    assert need > 0 and lib.tri_paged_attention_quant(h, C.byref(a), C.byref(s), None) == 0
    _, splits, grids, _, heads, shift = P.attention_q8_plan(0, 3, 2, 16, 4, 128, True, 8000, 8000, need)
    v, raw, _ = read_args(lib, 0)
    w, raw2, _ = read_args(lib, 1)
    assert (v, w) == (P.PA8_ROWS, P.PA8_JOIN) and raw[:312] == raw2[:312]
    word = lambda i, n=4: int.from_bytes(raw[i:i + n], "little", signed=True)  # noqa: E731
    assert word(104, 8) == at(31) and word(112, 8) == at(31) + 3 * 16 * splits * 128 * 4
    assert word(112, 8) + 3 * 16 * splits * 8 == at(31) + need
    assert (heads, splits) == (1, 128) and word(180) == splits
    # the maxima of the parts are in powers of two already
    assert C.c_float.from_buffer_copy(raw[192:196]).value == 1.0 and raw[196:198] == b"\x01\0"
    assert [word(216 + 8 * i, 8) for i in range(8)] == [at(7), 16, 4, 1, at(8), 16, 4, 1]
    assert abs(C.c_float.from_buffer_copy(raw[280:284]).value - 0.25 * 1.4426950408889634) < 1e-7
    assert word(284) == 4 and [word(296 + 4 * i) for i in range(4)] == [grids[0], shift, 1, (2 ** 31 - 1) // 2]


def test_steps_stay_in_31_bits(lib, fresh):
    """The steps of all tiles are numbered on the device: the host makes them longer
    where a table's lengths could take more than 2^31."""
    h = fresh()
    a = attn(L.BF16, 65536, 4096, 64, (1 << 27) - 256, kv(nk=64, hd=64))
    s = q8(nk=64)
    assert lib.tri_paged_attention_quant(h, C.byref(a), C.byref(s), None) == 0
    _, raw, _ = read_args(lib, 0)
    heads = last(lib, h).key[3] >> 25 & 3
    shift = int.from_bytes(raw[300:304], "little")
    tiles = (a.T // (16 >> heads) + a.R) * (64 >> heads)
    per = -(-a.cols * 16 // (1 << shift))
    assert tiles * per < 1 << 31 <= tiles * -(-a.cols * 16 // (1 << shift - 1))


# ---- misses, keys, failures ---------------------------------------------------------------
def test_miss_install_and_record(lib, fresh):
    h = fresh(flags=0)
    a, s = attn(T=4, R=4, cols=2000), q8(L.E4M3)
    a.workspace_bytes = lib.tri_paged_attention_quant_workspace(C.byref(a))
    a.workspace = at(31)
    f = lib.tri_paged_attention_quant
    assert a.workspace_bytes and f(h, C.byref(a), C.byref(s), None) == L.MISS
    assert lib.trifake_launch_count() == 0
    x = L.Selection()
    assert lib.tri_spec_install_last_miss(h, C.byref(x)) == 0
    assert f(h, C.byref(a), C.byref(s), None) == 0
    got = last(lib, h)
    assert launches(x) == launches(got) and tuple(x.key) == tuple(got.key) and len(launches(x)) == 2
    for f, op in zip(both(lib), (P.OP_KV_WRITE_Q8, P.OP_KV_READ_Q8)):
        assert f(h, C.byref(rows()), None) == L.MISS
        assert lib.tri_spec_install_last_miss(h, C.byref(x)) == 0
        assert launches(x) == P.kv_rows_q8_selection(op, 1, 0, 8, 3, 2, 64, 16, True)[1]
    assert stats(lib, h) == dict(stats(lib, h), calls=4, hits=1, misses=3, installs=3)


def test_a_failed_launch_stops_the_call(lib, fresh):
    h = fresh()
    a = attn(T=1, R=1, cols=2000)
    a.workspace_bytes = lib.tri_paged_attention_quant_workspace(C.byref(a))
    a.workspace = at(31)
    for n, seen in ((0, 1), (1, 2)):
        lib.trifake_reset()
        lib.trifake_fail_at(n)
        assert lib.tri_paged_attention_quant(h, C.byref(a), C.byref(q8()), None) == L.E_LAUNCH
        assert lib.trifake_launch_count() == seen
    for f in both(lib):
        lib.trifake_reset()
        lib.trifake_fail_at(0)
        assert f(h, C.byref(rows()), None) == L.E_LAUNCH
    lib.trifake_fail_at(-1)


def test_versions_do_not_grow_with_lengths(lib, fresh):
    """One version per form, heads a tile and split or not, however lengths vary."""
    h = fresh()
    for cols in range(1, 3000, 37):
        a = attn(T=4, R=4, cols=cols)
        need = lib.tri_paged_attention_quant_workspace(C.byref(a))
        if need:
            a.workspace, a.workspace_bytes = at(31), need
        assert lib.tri_paged_attention_quant(h, C.byref(a), C.byref(q8()), None) == 0
        assert lib.tri_kv_read_quant(h, C.byref(rows(cols=cols)), None) == 0
    assert stats(lib, h)["n_versions"] == 3


def test_keys_export_and_import(lib, fresh):
    h = fresh()
    for f in both(lib):
        assert f(h, C.byref(rows(L.F32)), None) == 0
    assert lib.tri_paged_attention_quant(h, C.byref(attn()), C.byref(q8()), None) == 0
    assert lib.tri_paged_attention_quant(h, C.byref(attn(T=2, R=1, cols=500)), C.byref(q8(L.E4M3)),
                                         None) == 0
    n = C.c_uint32()
    buf = (C.c_uint64 * 24)()
    assert lib.tri_spec_export_keys(h, buf, 4, C.byref(n)) == 0 and n.value == 4
    g = fresh(flags=0)
    done = C.c_uint32()
    assert lib.tri_spec_import_keys(g, buf, 4, C.byref(done)) == 0 and done.value == 4
    for f in both(lib):
        assert f(g, C.byref(rows(L.F32)), None) == 0
    assert lib.tri_paged_attention_quant(g, C.byref(attn()), C.byref(q8()), None) == 0
    assert buf[21] >> 25 & 3 == 1                     # two heads a tile
    common = [(0, 1 << 25), (0, 1 << 40), (1, 5), (2, 1 << 60), (3, 1), (3, 1 << 33), (3, 1 << 40),
              (4, 1), (5, 1)]
    bad = {0: common + [(2, 1 << 16), (3, 3 << 16), (3, 1 << 24)],
           1: common + [(2, 1 << 16), (3, 1 << 16), (3, 1 << 24)],
           # forms 0 and 5 of aligned rows; heads that do not divide, too many, of another form
           2: common + [(2, 1 << 16), (3, 1 << 16), (3, 1 << 18), (3, 2 << 25), (3, 1 << 28)],
           3: common + [(3, 3 << 25), (3, 3 << 16), (3, 1 << 27)]}
    for i, changes in bad.items():
        for word, bit in changes:
            k = list(buf[6 * i:6 * i + 6])
            k[word] ^= bit
            one = (C.c_uint64 * 6)(*k)
            assert lib.tri_spec_import_keys(g, one, 1, C.byref(done)) == INVALID, (i, word, bit)


@pytest.mark.parametrize("flags", [L.JIT, L.AUTOTUNE, L.GENERIC, L.RESIDENT_ARGS])
def test_other_cache_flags(lib, fresh, flags):
    """Nothing is compiled, timed or held for these ops; a generic version
    serves every token bucket."""
    h = fresh(flags=L.AUTO_INSTALL | flags)
    for T in (1, 9, 1000):
        for f in both(lib):
            assert f(h, C.byref(rows(T=T, R=1, scales=q8(block=1))), None) == 0
    assert lib.trifake_compile_count() == 0 and lib.trifake_launch_count() == 6
    assert stats(lib, h)["n_versions"] == (2 if flags == L.GENERIC else 6)
    info = L.ResidentInfo()
    lib.tri_spec_resident_info(h, C.byref(info))
    assert info.held == 0


def test_under_sanitizers():
    """These tests again, on the core built with the address and the undefined
    behaviour sanitizer."""
    asan, ubsan = _runtime("libasan.so"), _runtime("libubsan.so")
    if not asan or not ubsan:
        pytest.skip("gcc sanitizer runtimes not found")
    env = dict(os.environ, TRI_FAKE_SANITIZE="1", LD_PRELOAD=f"{asan}:{ubsan}",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        "-k", "not sanitizers", "tests/test_host_paged_q8.py"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in tail and "runtime error:" not in tail, tail
