"""GPU: the ops of the 8-bit cache together, as a serving loop calls them, and their calls
through every route: prepared, captured, other streams, the Python form, other caches.

A run of steps (prompts, then single tokens, requests of other lengths) keeps a second
cache by the oracle's write; codes and scales stay equal to it throughout, attention and
the read are compared over what it holds.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged as P
from tests.test_gpu_output_streams import owner
from tests.test_gpu_paged import DEV, DT, check, f64, i32
from tests.test_gpu_paged_q8 import (CODE, CODES, DTYPES, KIND, attend, numbers, oracle, problem, read_check,
                                     same, write, write_problem, written)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tri():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_37241_amd as tri
    return tri


@pytest.fixture
def cache(tri):
    c = tri.SpecCache(capacity=1024, auto_install=True)
    yield c
    torch.cuda.synchronize()
    c.close()


@pytest.fixture(params=["native", "python"])
def either(tri, request):
    c = tri.SpecCache(auto_install=True)
    if request.param == "python":
        c._fast = tri._PythonForm()
    yield c
    torch.cuda.synchronize()
    c.close()


def start(p, R, page, cols, pages):
    p["table"] = torch.full((R, cols), -1, dtype=torch.int32, device=DEV)
    return torch.randperm(pages, device=DEV).to(torch.int32), i32([pages, 0]), i32([0] * R)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype,nq,nk,hd,page,block", [("bf16", 8, 2, 128, 8, 8), ("f32", 4, 4, 64, 8, 2),
                                                       ("bf16", 6, 3, 40, 6, 3), ("f32", 5, 1, 33, 8, 4)])
def test_serving_steps(cache, code, dtype, nq, nk, hd, page, block):
    """Bookkeeping, RoPE, quantised store and attention over six steps, then all rows read back."""
    R, pages = 4, 64
    shape = (pages, page, nk, hd)
    nan = torch.full(shape, 100.0, device=DEV).to(CODE[code])
    p = {c: nan.clone() for c in ("kc", "vc")}
    p.update({s: torch.full((pages, page // block, nk), float("nan"), device=DEV) for s in ("ks", "vs")})
    free, count, held = start(p, R, page, 12, pages)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(hd)
    p["scale"] = hd ** -0.5
    total = [0] * R
    for new in ([5, 17, 0, 1], [1, 1, 30, 1], [1, 0, 1, 9], [1, 1, 1, 1], [0, 0, 0, 1], [3, 1, 1, 1]):
        T = sum(new) + 2                                   # two rows of nobody
        slots, pos, starts, lens, left = cache.kv_slots(held, i32(new), p["table"], free, count, page, T)
        q, k, v = (2.0 ** torch.randint(-2, 3, (T, 1, 1), generator=gen, device=DEV)
                   * torch.randn((T, h, hd), generator=gen, device=DEV) for h in (nq, nk, nk))
        q, k, v = (x.to(DT[dtype]) for x in (q, k, v))
        if hd % 2 == 0:
            cache.rope_qk(q, k, pos, 10000.0)
        p.update(q=q, k=k, v=v, kv_len=lens, q_start=starts)
        torch.cuda.synchronize()
        want = written(p, code)
        write(cache, p)
        same(p, want)
        check(attend(cache, p), oracle(p), dtype)
        total = [a + b for a, b in zip(total, new)]
        assert lens.tolist() == total and left[1] == 0
        held, count = lens, left
    p["q_start"] = i32([0] + np.cumsum(total).tolist())
    gk, gv = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"],
                              sum(total), DT[dtype])
    assert gk.dtype == gv.dtype == DT[dtype] and gk.shape == (sum(total), nk, hd)
    read_check(p, gk, gv, dtype)


def test_a_prefix_read_written_and_attended_again(cache):
    """What kv_read_q8 gives back and kv_write_q8 stores again keeps every value, by either code:
    the largest magnitude of a block is a code's largest, or the scales are powers of two."""
    for code, block in (("int8", 4), ("e4m3", 16)):
        p = write_problem("f32", code, [(100, 100), (37, 37)], 2, 64, 16, block)
        write(cache, p)
        a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
        k, v = cache.kv_read_q8(*a, 137, torch.float32)
        p.update(k=k, v=v)
        want = written(p, code)
        write(cache, p)
        same(p, want)
        k2, v2 = cache.kv_read_q8(*a, 137, torch.float32)
        # one more rounding of a scale, of a code's product: 2^-24 of the largest each
        for x, y in ((k, k2), (v, v2)):
            assert (x - y).abs().max() <= 2.0 ** -22 * x.abs().max()


def test_pages_that_are_missing(cache):
    """The stack runs out: the tokens without a slot are not stored, their keys
    are not seen, they read as zeros, and nothing else changes."""
    p = write_problem("bf16", "int8", [(40, 0)], 1, 64, 4, 4)
    free, count, held = start(p, 2, 4, 5, 3)
    slots, pos, starts, lens, left = cache.kv_slots(held, i32([6, 9]), p["table"], free, count, 4, 15)
    q, p["k"], p["v"] = (torch.randn((15, 1, 64), device=DEV).to(torch.bfloat16) for _ in range(3))
    p.update(q=q, kv_len=lens, q_start=starts, scale=0.125)
    torch.cuda.synchronize()
    want = written(p, "int8")
    write(cache, p)
    same(p, want)
    check(attend(cache, p), oracle(p), "bf16")
    gk, gv = cache.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], lens, starts, 15)
    read_check(p, gk, gv, "bf16")
    assert left.tolist() == [0, 2] and (gk[10:] == 0).all() and (gk[:10] != 0).any()


# ---- attention with several K heads a tile, many requests, many parts -----------------------
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,nk,hd,heads", [(16, 4, 128, 2), (12, 12, 64, 2), (12, 6, 64, 1), (24, 4, 80, 1),
                                            (32, 2, 48, 0), (9, 9, 64, 0), (8, 4, 256, 2), (40, 8, 64, 1)])
def test_several_heads_a_tile(cache, code, dtype, nq, nk, hd, heads):
    """Every number of K heads that a tile can take, with groups that do not fill its rows,
    NaN in hidden places, windows, requests from no key to many parts."""
    lens = [(2300, 1), (1, 1), (0, 0), (513, 1), (700, 1), (0, 1)]
    p = problem(dtype, code, lens, nq, nk, hd, 16, 8, seed=nq, pad=1)
    p["vs"][int(p["table"][4, 9]), 1, nk - 1] = float("nan")
    p["ks"][int(p["table"][3, 2]), 0, 0] = float("nan")
    want = oracle(p)
    got = attend(cache, p)
    s = cache.last_selection()
    assert s.variant == P.PA8_ROWS and s.key[3] >> 25 & 3 == heads and s.n_launches == 2
    check(got, want, dtype)
    assert torch.equal(got.nan_to_num(3.0), attend(cache, p).nan_to_num(3.0))
    for w in (1, 130, 1500):
        check(attend(cache, p, window=w), oracle(p, w), dtype)
    if 2 * (nq // nk) <= 16 >> heads:                      # two new tokens of each
        lens = [(n, min(n, 2)) for n, _ in lens]
        p = problem(dtype, code, lens, nq, nk, hd, 16, 8, seed=nq)
        p["vs"][int(p["table"][0, 143]), 1, 0] = float("nan")     # slots 2296 .. 2299
        check(attend(cache, p), oracle(p), dtype)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("nq,nk,hd", [(8, 2, 64), (4, 4, 128), (20, 1, 64)])
@pytest.mark.parametrize("R", [63, 64, 65, 300, 1025])
def test_many_requests(cache, code, nq, nk, hd, R):
    """More requests than a wavefront has lanes, a few of them long, many empty."""
    rng = np.random.default_rng(R)
    lens = [(int(rng.integers(0, 40)), 1) for _ in range(R)]
    lens = [(n, min(n, 1)) for n, _ in lens]
    for r in (0, R // 2, R - 1):
        lens[r] = (1500 + r, 1)
    p = problem("bf16", code, lens, nq, nk, hd, 16, 16, seed=R, pad=2)
    want = oracle(p)
    check(attend(cache, p), want, "bf16")
    assert nk == 1 or cache.last_selection().variant == P.PA8_ROWS
    check(attend(cache, p, max_kv=600), want, "bf16")      # no parts


@pytest.mark.parametrize("part", [0.0, 0.02, 0.3, 1.0])
def test_workspaces_of_any_size(cache, tri, part):
    """The C entry with less memory for parts than it would use, and none: fewer parts, and
    nothing is written behind them."""
    L = tri._lib
    for lens, nq, nk, hd in (([(5000, 1), (40, 1)], 8, 4, 128), ([(3000, 300)], 8, 1, 128),
                             ([(4000, 2)], 3, 1, 20)):
        p = problem("bf16", "int8", lens, nq, nk, hd, 16, 8)
        if nq == 8 and nk == 1:
            wide = torch.full((1, 400), -1, dtype=torch.int32, device=DEV)
            wide[:, :p["table"].shape[1]] = p["table"]
            p["table"] = wide
        out = torch.full_like(p["q"], 7.0)
        kv, q8 = tri._kv_q8(p["kc"], p["vc"], p["ks"], p["vs"], 0)
        t, T = p["table"], p["q"].shape[0]
        a = L.AttentionArgs(L.BF16, nq, T, len(lens), t.shape[1], p["q"].data_ptr(), nq * hd, out.data_ptr(),
                            nq * hd, t.data_ptr(), t.stride(0), p["kv_len"].data_ptr(),
                            p["q_start"].data_ptr(), p["scale"], 0, 0, None, 0, kv)
        need = tri._dll.tri_paged_attention_quant_workspace(C.byref(a))
        assert need > 0
        n = int(need * part) // 16 * 16
        space = torch.full((n + 4096,), 255, dtype=torch.uint8, device=DEV)
        a.workspace, a.workspace_bytes = (space.data_ptr() if n else None), n
        stream = torch.cuda.current_stream().cuda_stream
        assert tri._dll.tri_paged_attention_quant(cache._h, C.byref(a), C.byref(q8), stream) == 0
        torch.cuda.synchronize()
        check(out, oracle(p), "bf16")
        assert (space[n:] == 255).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("R", [3, 64, 301])
@pytest.mark.parametrize("hd", [64, 20])
def test_starts_that_fall(cache, code, R, hd):
    """Requests whose rows overlap (a caller's mistake): what they leave is theirs, but no more
    work is done than the rows allow and nothing else is written."""
    T, page = 40, 16
    p = problem("bf16", code, [(600, 1)] * R, 8, 2, hd, page, 8)
    p["q_start"] = i32([0, T] * ((R + 1) // 2) + [0] * ((R + 1) % 2))
    flat = torch.full((T + 8, 8, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    p["q"] = torch.randn((T, 8, hd), device=DEV).to(torch.bfloat16)
    attend(cache, p, out=flat[4:-4])
    attend(cache, p, max_kv=600, out=flat[4:-4])
    assert (flat[:4] == 7.0).all() and (flat[-4:] == 7.0).all()
    rows = torch.full((2, T + 8, 2, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
    cache.kv_read_q8(*a, T, k=rows[0, 4:-4], v=rows[1, 4:-4])
    torch.cuda.synchronize()
    assert (rows[:, :4] == 7.0).all() and (rows[:, -4:] == 7.0).all()
    spare = sorted(set(range(p["kc"].shape[0])) - set(p["table"].view(-1).tolist()))
    before = [p[c][spare].view(torch.uint8).clone() for c in ("kc", "vc", "ks", "vs")]
    cache.kv_write_q8(rows[0, 4:-4], rows[1, 4:-4], *a)
    torch.cuda.synchronize()
    assert spare and all(torch.equal(p[c][spare].view(torch.uint8), b)
                         for c, b in zip(("kc", "vc", "ks", "vs"), before))
    p = problem("bf16", code, [(600, 1)] * 3, 8, 2, hd, page, 8)
    check(attend(cache, p), oracle(p), "bf16")


# ---- routes -----------------------------------------------------------------------------------
@pytest.mark.parametrize("lens", [[(40, 1), (9, 1)], [(3000, 1)], [(300, 200)], [(1500, 33)]])
@pytest.mark.parametrize("code", CODES)
def test_captured_and_replayed(cache, code, lens):
    """A step in a graph: replays follow the data behind the pointers, with
    eager calls and synchronizations between them."""
    p = write_problem("bf16", code, lens, 2, 128, 16, 8)
    p["q"] = torch.randn((p["k"].shape[0], 8, 128), device=DEV).to(torch.bfloat16)
    before = {c: p[c].clone() for c in ("kc", "vc", "ks", "vs")}
    out, T = torch.full_like(p["q"], 7.0), p["k"].shape[0]
    rows = [torch.empty_like(p["k"]) for _ in range(2)]

    def step():
        a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
        cache.kv_write_q8(p["k"], p["v"], *a)
        cache.paged_attention_q8(p["q"], *a, p["scale"], out=out)
        return cache.kv_read_q8(*a, T, k=rows[0], v=rows[1])

    def reset():
        for c, t in before.items():
            p[c].view(torch.uint8).copy_(t.view(torch.uint8))
        out.fill_(7.0)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        for x in ("q", "k", "v"):
            p[x].normal_()
        reset()
        want = written(p, code)
        g.replay()
        torch.cuda.synchronize()
        same(p, want)
        got = [x.clone() for x in (out, *rows)]
        check(got[0], oracle(p), "bf16")
        read_check(p, *got[1:], "bf16")
        reset()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, *rows)))


def test_two_graphs_at_once(cache):
    """Two captured calls that split their keys, replayed on two streams together:
    each has its own workspace."""
    ps = [problem("bf16", "int8", [(6000, 1)], 4, 1, 128, 16, 16, seed=i) for i in range(2)]
    want = [attend(cache, p) for p in ps]
    assert cache.last_selection().n_launches == 2
    graphs, outs = [], []
    for p in ps:
        out = torch.full_like(p["q"], 7.0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend_async(cache, p, out)
        graphs.append(g)
        outs.append(out)
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(20):
        for out in outs:
            out.fill_(7.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    g.replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            assert torch.equal(out, w)


def attend_async(c, p, out, **kw):
    return c.paged_attention_q8(p["q"], p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"],
                                p["q_start"], p["scale"], out=out, **kw)


def test_two_streams_at_once(cache, tri):
    """Calls of two caches and of one, on two streams, split and not."""
    other = tri.SpecCache(auto_install=True)
    ps = [problem("bf16", "e4m3", [(5000, 1), (70, 1)], 4, 1, 128, 16, 8, seed=i) for i in range(2)]
    want = [attend(cache, p) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for second in (other, cache):
        outs = [[torch.full_like(p["q"], 7.0) for _ in range(10)] for p in ps]
        torch.cuda.synchronize()
        for i in range(10):
            for c, p, s, out in zip((cache, second), ps, streams, outs):
                if i % 2:
                    attend_async(c, p, out[i], stream=s)
                else:
                    with torch.cuda.stream(s):
                        attend_async(c, p, out[i])
                        junk = torch.full((1 << 16,), float("nan"), device=DEV)   # reuses what is free
                        del junk
        torch.cuda.synchronize()
        for w, out in zip(want, outs):
            for x in out:
                assert torch.equal(x, w)
    other.close()


def test_made_outputs_and_streams(either):
    """Outputs and workspaces that a call makes come from the call's stream's memory, whatever
    stream is the current one."""
    p = write_problem("bf16", "int8", [(5000, 2)], 1, 64, 16, 16)
    a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
    q = torch.randn((2, 4, 64), device=DEV).to(torch.bfloat16)
    here, there = torch.cuda.current_stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    want = None
    for stream in (None, there, torch.cuda.ExternalStream(there.cuda_stream, device=there.device)):
        torch.cuda.empty_cache()
        before = {s["address"] for s in torch.cuda.memory_snapshot()}
        either.kv_write_q8(p["k"], p["v"], *a, stream=stream)
        made = (either.paged_attention_q8(q, *a, stream=stream), *either.kv_read_q8(*a, 2, stream=stream))
        torch.cuda.synchronize()
        on = here if stream is None else there
        assert all(owner(t) == on.cuda_stream for t in made) and torch.cuda.current_stream() == here
        assert all(s["stream"] == on.cuda_stream for s in torch.cuda.memory_snapshot()
                   if s["address"] not in before)
        want = made if want is None else want
        assert all(torch.equal(x, y) for x, y in zip(made, want))


def test_prepared_calls(cache):
    """A prepared call keeps its operands and its workspace; its data may change."""
    p = problem("bf16", "int8", [(4000, 1), (50, 1)], 8, 2, 128, 16, 8)
    a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
    call = cache.prepare("paged_attention_q8", p["q"], *a, p["scale"])
    junk = [torch.full((1 << 18,), float("nan"), device=DEV) for _ in range(20)]
    del junk
    for i in range(3):
        p["q"].normal_()
        got = call()
        torch.cuda.synchronize()
        check(got, oracle(p), "bf16")
    p["k"], p["v"] = (torch.randn((2, 2, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    store, load = cache.prepare("kv_write_q8", p["k"], p["v"], *a), cache.prepare("kv_read_q8", *a, 2)
    torch.cuda.empty_cache()
    for i in range(2):
        p["k"].normal_()
        want = written(p, "int8")
        store()
        k, v = load()
        torch.cuda.synchronize()
        same(p, want)
        read_check(p, k, v, "bf16")


def test_native_and_python_forms_agree(cache, tri):
    if tri._native is None:
        pytest.skip("the binding's extension module is not built")
    python = tri.SpecCache(auto_install=True)
    python._fast = tri._PythonForm()
    for dtype, code, lens, nk, hd in (("bf16", "int8", [(3000, 1)], 2, 128),
                                      ("f32", "e4m3", [(77, 30), (9, 2)], 3, 48)):
        res = []
        for c in (cache, python):
            p = write_problem(dtype, code, lens, nk, hd, 16, 8, "odd")
            a = (p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"])
            T = p["k"].shape[0]
            r = c.kv_write_q8(p["k"], p["v"], *a)
            assert all(x is y for x, y in zip(r, a[:4])) and len(r) == 4
            q = p["k"].repeat(1, 2, 1)
            x = [t.float().nan_to_num(3.0) for t in a[:4]]
            x.append(c.paged_attention_q8(q, *a, window=500))
            out = torch.empty_like(q)
            assert c.paged_attention_q8(q, *a, p["scale"], 500, 0, out) is out
            x.append(out)
            x += c.kv_read_q8(*a, T, DT[dtype])
            k, v = torch.empty_like(p["k"]), torch.empty_like(p["k"])
            made = c.kv_read_q8(*a, T, DT[dtype], k, None)
            assert made[0] is k and made[1] is not v
            x += made
            made = c.kv_read_q8(*a, T, dtype=DT[dtype], v=v)
            assert made[1] is v
            x += [*made, *c.kv_read_q8(*a, 0, DT[dtype])]
            torch.cuda.synchronize()
            res.append(x)
        for x, y in zip(*res):
            assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y)
    python.close()


@pytest.mark.parametrize("kw", [dict(jit=True), dict(autotune=True), dict(generic=True), dict(resident_args=True)])
def test_other_caches(tri, kw):
    """Caches that compile, time or hold argument blocks serve these ops as the others do."""
    c = tri.SpecCache(auto_install=True, **kw)
    for T in (1, 40):
        p = write_problem("bf16", "e4m3", [(2000, T)], 2, 64, 16, 8)
        p["q"] = torch.randn((T, 4, 64), device=DEV).to(torch.bfloat16)
        for _ in range(3):
            want = written(p, "e4m3")
            write(c, p)
            same(p, want)
            check(attend(c, p), oracle(p), "bf16")
            k, v = c.kv_read_q8(p["kc"], p["vc"], p["ks"], p["vs"], p["table"], p["kv_len"], p["q_start"], T)
            read_check(p, k, v, "bf16")
    c.close()


def test_binding_refusals(either, tri):
    p = write_problem("bf16", "int8", [(20, 2)], 2, 64, 16, 8)
    ok = dict(k_cache=p["kc"], v_cache=p["vc"], k_scale=p["ks"], v_scale=p["vs"], block_table=p["table"],
              kv_len=p["kv_len"], q_start=p["q_start"])
    bad = [dict(k_cache=p["kc"].cpu()), dict(v_cache=p["vc"][:1]), dict(k_cache=p["kc"][..., ::2]),
           dict(v_cache=p["vc"].view(torch.float8_e4m3fn)), dict(k_cache=p["kc"].view(torch.uint8)),
           dict(k_cache=p["kc"].bfloat16(), v_cache=p["vc"].bfloat16()), dict(k_scale=p["ks"].double()),
           dict(k_scale=p["ks"][:1]), dict(v_scale=p["vs"].half()), dict(v_scale=p["vs"][:, :1]),
           dict(k_scale=p["ks"].cpu()), dict(k_scale=p["ks"][:, 0]), dict(v_scale=p["vs"][..., :1]),
           dict(k_scale=p["ks"].repeat(1, 3, 1), v_scale=p["vs"].repeat(1, 3, 1)),
           dict(k_scale=p["ks"][:, :0], v_scale=p["vs"][:, :0]), dict(k_scale=p["ks"][:, :1].expand(-1, 2, -1)),
           dict(block_table=p["table"].long()), dict(block_table=p["table"][0]),
           dict(kv_len=p["kv_len"].long()), dict(kv_len=i32([1, 2])), dict(q_start=i32([0])),
           dict(q_start=i32([0, 9, 2])[::2])]
    q = p["k"].repeat(1, 2, 1)
    calls = either.stats()["hits"] + either.stats()["installs"]
    for kw in bad:
        for f in (lambda a: either.kv_write_q8(p["k"], p["v"], **a), lambda a: either.kv_read_q8(T=2, **a),
                  lambda a: either.paged_attention_q8(q, **a)):
            with pytest.raises((ValueError, TypeError, tri.TriError)):
                f({**ok, **kw})
    for k, v in ((p["k"].half(), p["v"].half()), (p["k"], p["v"].float()), (p["k"][:, :1], p["v"][:, :1]),
                 (p["k"], p["v"][:1]), (p["k"].transpose(0, 1), p["v"].transpose(0, 1)),
                 (p["k"].cpu(), p["v"].cpu()), (p["k"][0], p["v"][0])):
        with pytest.raises((ValueError, TypeError)):
            either.kv_write_q8(k, v, **ok)
    for kw in (dict(T=-1), dict(T=2, dtype=torch.float16), dict(T=2, k=p["k"].float()), dict(T=3, v=p["v"]),
               dict(T=2, dtype=torch.float32, k=p["k"])):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            either.kv_read_q8(**ok, **kw)
    for kw in (dict(scale=float("nan")), dict(window=-1), dict(max_kv=-1), dict(out=q.float()), dict(out=q[:1]),
               dict(window=1 << 32), dict(max_kv=1 << 64)):
        with pytest.raises((tri.TriError, ValueError, OverflowError, RuntimeError)):
            either.paged_attention_q8(q, **ok, **kw)
    for x in (q[:, :3], q.half(), q[..., :32].contiguous()):
        with pytest.raises((tri.TriError, ValueError, TypeError)):
            either.paged_attention_q8(x, **ok)
    assert either.stats()["hits"] + either.stats()["installs"] == calls
    torch.cuda.synchronize()
