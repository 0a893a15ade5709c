"""GPU: outputs and workspaces that a call makes belong, for torch's allocator,
to the stream that the call runs on, in the native and the Python marshalling."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def tri():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_37241_amd as tri
    return tri


@pytest.fixture(params=["native", "python"])
def cache(tri, request):
    c = tri.SpecCache(auto_install=True)
    if request.param == "python":
        c._fast = tri._PythonForm()
    yield c
    torch.cuda.synchronize()
    c.close()


def owner(t):
    """The stream whose pool a tensor's memory came from."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


def operands():
    f = lambda *s: torch.randn(s, device=DEV).to(torch.bfloat16)  # noqa: E731
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    x, w, mask = f(6, 64), f(64), torch.zeros(6, 64, dtype=torch.uint8, device=DEV)
    kc = f(4, 16, 2, 64)
    return {
        "rmsnorm": (x, w), "residual_rmsnorm": (x, x.clone(), w), "swiglu": (x, x.clone()),
        "silu": (x,), "add": (x, x.clone()), "masked_fill": (x, mask, 1.0),
        "embedding": (f(9, 64), i([1, 2, 3])),
        "kv_slots": (i([3, 4]), i([1, 1]), i([[0, 1], [2, 3]]), i([7]), i([1]), 16, 3),
        "paged_attention": (f(2, 4, 64), kc, kc.clone(), i([[0, 1, 2, 3]]), i([50]), i([0, 2])),
        "decode_chain": (x, x.clone(), w, f(6, 2, 64), f(6, 1, 64), i([0] * 6), x.clone(), x.clone()),
    }


OPS = ["rmsnorm", "residual_rmsnorm", "swiglu", "silu", "add", "masked_fill", "embedding", "kv_slots",
       "paged_attention", "decode_chain"]


@pytest.mark.parametrize("op", OPS)
def test_made_outputs(cache, op):
    args = operands()[op]
    here, there = torch.cuda.current_stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outside = torch.cuda.ExternalStream(there.cuda_stream, device=there.device)
    for stream, want in ((there, there), (None, here), (outside, there)):
        made = getattr(cache, op)(*args, stream=stream)
        torch.cuda.synchronize()
        for t in made if isinstance(made, tuple) else (made,):
            assert owner(t) == want.cuda_stream
        assert torch.cuda.current_stream() == here
    with torch.cuda.stream(there):
        made = getattr(cache, op)(*args)
    torch.cuda.synchronize()
    assert owner(made[0] if isinstance(made, tuple) else made) == there.cuda_stream


@pytest.mark.parametrize("op", OPS)
def test_the_default_stream_from_another(cache, op):
    args = operands()[op]
    there, default = torch.cuda.Stream(), torch.cuda.default_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(there):
        made = getattr(cache, op)(*args, stream=default)
        assert torch.cuda.current_stream() == there
        torch.cuda.synchronize()
    for t in made if isinstance(made, tuple) else (made,):
        assert owner(t) == default.cuda_stream


@pytest.mark.parametrize("op", ["rmsnorm", "paged_attention"])
def test_a_stream_that_torch_did_not_make(cache, op):
    """Anything with the address of a stream is taken as before."""
    class Bare:
        def __init__(self, s):
            self.cuda_stream = s.cuda_stream
    args = operands()[op]
    there = torch.cuda.Stream()
    torch.cuda.synchronize()
    made = getattr(cache, op)(*args, stream=Bare(there))
    torch.cuda.synchronize()
    assert owner(made) == there.cuda_stream
    assert torch.equal(made, getattr(cache, op)(*args))


def test_made_workspaces(cache):
    """Split keys: the workspace comes from the call's stream, whether the
    output was given or not; the result is the one of the current stream."""
    gen = lambda *s: torch.randn(s, device=DEV).to(torch.bfloat16)  # noqa: E731
    q, kc, vc = gen(1, 4, 128), gen(320, 16, 1, 128), gen(320, 16, 1, 128)
    table = torch.arange(320, dtype=torch.int32, device=DEV)[None]
    lens = torch.tensor([5000], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    want = cache.paged_attention(q, kc, vc, table, lens, starts)
    assert cache.last_selection().n_launches == 2
    for out in (torch.empty_like(q), None):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        there = torch.cuda.Stream()
        before = {s["address"] for s in torch.cuda.memory_snapshot()}
        got = cache.paged_attention(q, kc, vc, table, lens, starts, out=out, stream=there)
        torch.cuda.synchronize()
        new = [s for s in torch.cuda.memory_snapshot() if s["address"] not in before]
        assert new and all(s["stream"] == there.cuda_stream for s in new)
        assert torch.equal(got, want)
