"""GPU: numbers that the fields of a call do not hold are refused, in the native
and the Python marshalling, and nothing is launched."""
import pytest
import torch

from tests.test_gpu_output_streams import cache, operands, tri  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 16, (1 << 64) + 16, -(1 << 32) + 16, 1 << 70])
def test_beyond_32_bits(cache, tri, n):  # noqa: F811
    kv, new, table, free, count, _, T = operands()["kv_slots"]
    before = table.clone()
    attention = operands()["paged_attention"]
    for call in (lambda: cache.kv_slots(kv, new, table, free, count, n, T),
                 lambda: cache.paged_attention(*attention, window=n)):
        calls = cache.stats()["hits"] + cache.stats()["installs"]
        with pytest.raises((ValueError, OverflowError, tri.TriError)):
            call()
        assert cache.stats()["hits"] + cache.stats()["installs"] == calls
    torch.cuda.synchronize()
    assert torch.equal(table, before)


@pytest.mark.parametrize("n", [(1 << 64) + 3, (1 << 64) + 1000, -(1 << 64) + 3])
def test_beyond_64_bits(cache, tri, n):  # noqa: F811
    kv, new, table, free, count, page, _ = operands()["kv_slots"]
    attention = operands()["paged_attention"]
    for call in (lambda: cache.kv_slots(kv, new, table, free, count, page, n),
                 lambda: cache.paged_attention(*attention, max_kv=n)):
        with pytest.raises((ValueError, OverflowError, RuntimeError)):
            call()


def test_numbers_that_are_no_integers(cache):  # noqa: F811
    args = operands()["kv_slots"]
    attention = operands()["paged_attention"]
    for call in (lambda: cache.kv_slots(*args[:5], 16.0, 3),
                 lambda: cache.paged_attention(*attention, window=2.5),
                 lambda: cache.paged_attention(*attention, max_kv="9")):
        with pytest.raises(TypeError):
            call()
