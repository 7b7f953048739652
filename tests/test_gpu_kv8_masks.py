"""Attention over the 8-bit cache where a query's bits may depend on nothing but
what it sees: the other queries of its tile, the codes of tokens that no query
sees, and every border of a mask or a split, one token at a time."""
import pytest

from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _int32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _randn(shape, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


# ------------------------------------------------------------- wide arguments
def test_windows_and_sinks_past_32_bits():
    """A window or a number of first tokens past 2^31 covers everything."""
    import torch
    cache = B.kv8_cache(1, 1, 256, 64)
    B.op_kv8_append(cache, _randn((1, 1, 256, 64), 1), _randn((1, 1, 256, 64), 2), _int32([0]))
    q = _randn((1, 2, 1, 64), 3)
    want = B.op_attention_kv8(q, cache, _int32([200]))
    for window, sinks in (((1 << 32) + 16, 0), (1 << 31, 0), (16, (1 << 32) + 3)):
        assert torch.equal(B.op_attention_kv8(q, cache, _int32([200]), window=window, sinks=sinks), want)
