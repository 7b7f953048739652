"""Attention over the 8-bit cache where a query's bits may depend on nothing but
what it sees: the other queries of its tile, the codes of tokens that no query
sees, and every border of a mask or a split, one token at a time."""
import numpy as np
import pytest

import lowbit_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _int32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _randn(shape, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


# --------------------------------------------------- the queries beside a query
# (cap, Hq, Hkv, T, border of two splits): a tile of 16 columns, one of 256
FORMS = {"few": (1088 * 2, 2, 2, 16, 1024), "many": (1216, 8, 1, 300, 640)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
def test_a_quotient_does_not_depend_on_the_tile(form, hd):
    """Values whose means over a window lie halfway between two bf16 numbers, at
    480 keys, where the sum times the rounded reciprocal of 480 falls to the
    other side than the quotient: a query gives the same bits whether its tile
    ends before the border of two splits or behind it, and in whichever row of
    the call it is.  (Of 32 tokens 4 d + 1 have 2 and the others 1.875 in dim d,
    so a window's mean is 1.875 + (4 d + 1) / 256; queries of zero weigh alike,
    and all sums are exact.)"""
    import torch
    cap, Hq, Hkv, T, border = FORMS[form]
    if form == "few" and hd == 128:
        cap, border = 1088, 512
    log(f"quotient {form} hd={hd}")
    j, d = torch.arange(cap, device="cuda")[:, None], torch.arange(hd, device="cuda")[None, :]
    v = torch.where(j % 32 < 4 * (d % 8) + 1, 2.0, 1.875).to(torch.bfloat16).expand(1, Hkv, cap, hd).contiguous()
    cache = B.kv8_cache(1, Hkv, cap, hd)
    B.op_kv8_append(cache, _randn((1, Hkv, cap, hd), 1), v, _int32([0]))
    q = torch.zeros((1, Hq, T, hd), dtype=torch.bfloat16, device="cuda")
    want = {}
    for n in (border - T, border - 20, border - 10, border - 6, border - 1):
        for count in (6, 10, T):
            out = B.op_attention_kv8(q, cache, _int32([n]), _int32([count]), window=480).reshape(T, -1)
            for t in range(count):
                row = want.setdefault(n + t, out[t].clone())
                assert torch.equal(row, out[t]), (n, count, t)
    assert len(want) > T


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 8, 2), (16, 2, 2), (40, 4, 2), (300, 16, 2)])
def test_a_query_does_not_depend_on_the_others(T, Hq, Hkv):
    """The same positions through other lengths and counts, over random values."""
    import torch
    hd, cap = 128, 1216
    log(f"queries T={T} heads {Hq}/{Hkv}")
    cache = B.kv8_cache(2, Hkv, cap, hd)
    B.op_kv8_append(cache, _randn((2, Hkv, cap, hd), 1), _randn((2, Hkv, cap, hd), 2), _int32([0, 0]))
    all_q = _randn((2, Hq, cap, hd), 3)  # by position
    want = {}
    for n in (500, 509, 600, 620, 639 - T // 2):
        for count in (1, (T + 1) // 2, T):
            lens = [n, n + 3]
            q = torch.stack([all_q[b, :, m:m + T] for b, m in enumerate(lens)]).contiguous()
            out = B.op_attention_kv8(q, cache, _int32(lens), _int32([count, T]), window=333, sinks=5).reshape(2, T, -1)
            for b, (m, c) in enumerate(zip(lens, (count, T))):
                for t in range(c):
                    row = want.setdefault((b, m + t), out[b, t].clone())
                    assert torch.equal(row, out[b, t]), (b, m, t)


# ------------------------------------------------------------ unseen tokens
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 2), (1, 24, 1), (5, 4, 2), (20, 2, 1), (100, 4, 2), (300, 16, 2)])
def test_codes_of_unseen_tokens_count_for_nothing(hd, T, Hq, Hkv):
    """Codes that are no numbers (0x7f, 0xff) in every token that no query sees,
    in blocks that are partly seen too, change no bit."""
    import torch
    cap = 1216
    log(f"unseen codes hd={hd} T={T} heads {Hq}/{Hkv}")
    cache = B.kv8_cache(1, Hkv, cap, hd)
    B.op_kv8_append(cache, _randn((1, Hkv, cap, hd), 1), _randn((1, Hkv, cap, hd), 2), _int32([0]))
    q = _randn((1, Hq, T, hd), 3)
    for n, window, sinks in ((0, 0, 0), (1, 0, 0), (37, 20, 0), (400, 0, 0), (447, 100, 0), (448, 90, 7), (700, 333, 70), (850, 64, 1)):
        want = B.op_attention_kv8(q, cache, _int32([n]), window=window, sinks=sinks)
        j = np.arange(cap)
        unseen = j >= n + T
        if window:
            unseen |= (j <= n - window) & (j >= sinks)
        bad = [t.clone() for t in cache]
        for codes, index in ((bad[0], R.key_index(hd)), (bad[2], R.value_index(hd))):
            blk, at = np.nonzero(unseen)[0] // 64, index[np.nonzero(unseen)[0] % 64]
            blk, at = torch.from_numpy(blk).cuda()[:, None], torch.from_numpy(at).cuda()
            codes[0][:, blk, at] = torch.where(at % 3 == 0, 0xff, 0x7f).to(torch.uint8)
        got = B.op_attention_kv8(q, bad, _int32([n]), window=window, sinks=sinks)
        assert torch.isfinite(want).all() and torch.equal(got, want), (n, window, sinks)


# ------------------------------------------------------------------- borders
def _marks(n, T, cap, window, sinks, hd):
    """hd tokens next to the borders of a call: of the mask for the first, a
    middle and the last query, and of 64 and of every length that a split may
    have."""
    at = set()
    for p in (n, n + T // 2, n + T - 1):
        for j in (p, p - window, sinks):
            at |= {j - 1, j, j + 1}
    g = np.random.default_rng(n + T + window)
    at |= {0, cap - 1, n - 1, n}
    at = {j for j in at if 0 <= j < cap}
    blocks = np.arange(64, cap, 64)
    near = [j + e for j in g.permutation(blocks) for e in (-1, 0)]
    at = list(at) + [j for j in near if j not in at]
    return np.array(at[:hd] if len(at) >= hd else at + [0] * (hd - len(at)))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("cap,T,Hq,window,sinks", [
    (1 << 18, 1, 2, 0, 0), (1 << 18, 1, 2, 100000, 5000), (1 << 18, 20, 1, 0, 0), (1 << 18, 20, 1, 100000, 64), (1 << 18, 600, 4, 3000, 4),
    (1 << 15, 600, 4, 0, 0), (4096, 1, 4, 0, 0), (4096, 70, 2, 1000, 3), (4096, 700, 4, 0, 0), (4096, 700, 4, 600, 130), (1088, 3, 2, 64, 1)])
def test_every_key_counts_once(hd, cap, T, Hq, window, sinks):
    """Queries of zero weigh all keys alike, and in dim d a single token has the
    value 448, the others none: a result is 448 over the number of keys that the
    query sees, or zero, exactly, where it does not see the token.  Weights,
    their sum (below 2^24) and the product are exact; the reciprocal and its
    product are off by 2^-23, bf16 by 2^-8."""
    import torch
    log(f"borders hd={hd} cap={cap} T={T} heads {Hq} window {window} sinks {sinks}")
    k = _randn((1, 1, cap, hd), 1)
    for n in (cap - T, cap - T - 65, cap // 2 + 1):
        at = _marks(n, T, cap, window, sinks, hd)
        v = torch.zeros((1, 1, cap, hd), dtype=torch.bfloat16, device="cuda")
        v[0, 0, torch.from_numpy(at).cuda(), torch.arange(hd, device="cuda")] = 448.0
        cache = B.kv8_cache(1, 1, cap, hd)
        B.op_kv8_append(cache, k, v, _int32([0]))
        q = torch.zeros((1, Hq, T, hd), dtype=torch.bfloat16, device="cuda")
        out = B.op_attention_kv8(q, cache, _int32([n]), window=window, sinks=sinks).double().cpu().numpy().reshape(T, Hq, hd)
        pos = n + np.arange(T)
        low = np.maximum(pos - window, -1) if window else np.full(T, -1)
        seen = (pos - low) + np.minimum(sinks if window else 0, low + 1)
        sees = (at[None] <= pos[:, None]) & ((at[None] > low[:, None]) | (at[None] < sinks))
        want = np.where(sees, 448.0 / seen[:, None], 0.0)[:, None]
        assert (np.abs(out - want) <= (2.0 ** -8 + 2.0 ** -22) * want).all(), n


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
