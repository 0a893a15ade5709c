"""GPU: attention's error against 64 bits beside that of the plain computation in
32 bits (products, maximum, powers and sums in torch, rounded once at the end),
as root mean squares over all outputs of a call."""
import pytest
import torch

from tests.test_gpu_paged import DT, attend, cache, f64, problem, tile_problem, tri  # noqa: F401

pytestmark = pytest.mark.gpu


def plain(p, dtype, bits):
    """softmax(scale q k) v of the rows of every request, in `bits`."""
    out = torch.empty(p["q"].shape, dtype=bits, device=p["q"].device)
    page, nk = p["kc"].shape[1:3]
    g, starts = p["q"].shape[1] // nk, p["q_start"].tolist()
    for r, kv in enumerate(p["kv_len"].tolist()):
        a, b = starts[r], starts[r + 1]
        used = p["table"][r, :-(-kv // page)].long()
        hidden = torch.arange(kv, device=out.device) > torch.arange(kv - (b - a), kv, device=out.device)[:, None]
        for h in range(nk if b > a else 0):
            k, v = (p[x][used, :, h].flatten(0, 1)[:kv].to(bits) for x in ("kc", "vc"))
            q = p["q"][a:b, h * g:(h + 1) * g].to(bits).transpose(0, 1).reshape(-1, k.shape[1])
            s = (q @ k.t().contiguous()).view(g, b - a, kv) * p["scale"]
            s = s.masked_fill(hidden, -float("inf"))
            w = torch.exp(s - s.amax(-1, keepdim=True))
            o = w.view(-1, kv) @ v / w.sum(-1).view(-1, 1)
            out[a:b, h * g:(h + 1) * g] = o.view(g, b - a, -1).transpose(0, 1)
    return out if bits == torch.float64 else out.to(DT[dtype])


def error(x, exact):
    return ((x.double() - exact).pow(2).sum() / exact.pow(2).sum()).sqrt().item()


def compare(cache, p, dtype):
    exact = plain(p, dtype, torch.float64)
    return error(attend(cache, p), exact), error(plain(p, dtype, torch.float32), exact)


SHORT = [(1 + i % 10, 1) for i in range(200)]
CHUNKS = [(600, 50), (90, 90), (1500, 129), (40, 1)]


@pytest.mark.parametrize("lens,nq,nk,hd", [(SHORT, 20, 4, 64), (SHORT, 4, 4, 64), (CHUNKS, 8, 2, 64),
                                           (SHORT, 20, 4, 128), (CHUNKS, 8, 2, 128), (CHUNKS, 4, 1, 256),
                                           ([(9000, 1)], 8, 2, 64), ([(700, 1)] * 5, 8, 1, 64)])
def test_float32(cache, lens, nq, nk, hd):  # noqa: F811
    """As good as the plain form: at most a tenth above it."""
    own, ref = compare(cache, problem("f32", lens, nq, nk, hd, 16, seed=nq + hd), "f32")
    assert own <= 1.1 * ref, (own, ref)


ROWS = [(SHORT, 16, 4, 64), (SHORT, 4, 4, 128), (SHORT, 4, 2, 256), ([(9000, 1)], 8, 2, 64),
        ([(5000, 1), (700, 2), (40, 1)], 8, 2, 128), ([(700, 1)] * 5, 8, 1, 256)]


@pytest.mark.parametrize("lens,nq,nk,hd", ROWS)
def test_bfloat16_in_tiles_of_16_rows(cache, lens, nq, nk, hd):  # noqa: F811
    """The weights are off by 2^-16, a 256th of the rounding of the result (at most
    2^-8, in both): the same error but for results that a rounding of float32
    moves over a border, far less than a hundredth of them."""
    own, ref = compare(cache, problem("bf16", lens, nq, nk, hd, 16, seed=nq + hd), "bf16")
    assert abs(own / ref - 1) <= 0.01, (own, ref)


@pytest.mark.parametrize("lens,nq,nk,hd", [(CHUNKS, 8, 2, 64), (CHUNKS, 8, 2, 128), (CHUNKS, 4, 1, 256),
                                           ([(900, 900)], 4, 2, 128)])
def test_bfloat16_in_tiles_of_128_rows(cache, lens, nq, nk, hd):  # noqa: F811
    """The weights are rounded as the result is, and independent of it: at most
    the square root of two times the error of the result's rounding alone."""
    p = tile_problem("bf16", lens, nq, nk, hd, seed=nq + hd)
    own, ref = compare(cache, p, "bf16")
    assert own <= 1.42 * ref, (own, ref)
