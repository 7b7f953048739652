"""The 8-bit key/value cache and attention over it against plain float64
references, and a decoder layer's step made of the operators in fewer bits."""
import numpy as np
import pytest

import lowbit_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def _host(t):
    import torch
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _int32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _kv(shape, seed, grow=0.0):
    """bf16 keys or values whose magnitude changes along the tokens (scales grow and fall)."""
    g = np.random.default_rng(seed)
    T = shape[2]
    return _bf16(g.standard_normal(shape) * np.exp(grow * g.standard_normal((shape[0], shape[1], T, 1))))


def _same(cache, ref):
    for got, want, name in zip(cache, ref.buffers(), ("key codes", "key scales", "value codes", "value scales")):
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=name.endswith("scales")), name


# -------------------------------------------------------------------- append
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("steps", [[1] * 70, [64, 64], [63, 1, 1, 63], [5, 130, 1, 20], [200], [1, 62, 2, 65]])
def test_append(hd, steps):
    log(f"append hd={hd} {steps[:6]}")
    Bn, H, cap = 2, 2, 256
    cache, ref = B.kv8_cache(Bn, H, cap, hd), R.Cache(Bn, H, cap, hd)
    lens = np.array([0, 3])
    k0, v0 = _kv((Bn, H, 3, hd), 1), _kv((Bn, H, 3, hd), 2)
    B.op_kv8_append(cache, k0, v0, _int32([0, 0]), _int32([0, 3]))
    ref.append(_host(k0), _host(v0), [0, 0], [0, 3])
    for i, T in enumerate(steps):
        k, v = _kv((Bn, H, T, hd), 10 + i, 1.5), _kv((Bn, H, T, hd), 50 + i, 1.5)
        B.op_kv8_append(cache, k, v, _int32(lens))
        ref.append(_host(k), _host(v), lens)
        lens = lens + T
    _same(cache, ref)


def test_append_counts_and_the_end_of_the_cache():
    """Ragged rows, sequences with no token, lengths at, past and before the
    cache's ends: nothing outside the tokens is touched."""
    Bn, H, cap, hd, T = 7, 1, 128, 64, 40
    cache, ref = B.kv8_cache(Bn, H, cap, hd), R.Cache(Bn, H, cap, hd)
    for t in cache[0], cache[2]:
        t.fill_(0x35)
    for c in ref.codes:
        c[:] = 0x35
    lens, counts = [0, 10, 100, 127, 128, -1, 64], [40, 0, 40, 5, 40, 40, -3]
    k, v = _kv((Bn, H, T, hd), 3), _kv((Bn, H, T, hd), 4)
    B.op_kv8_append(cache, k, v, _int32(lens), _int32(counts))
    ref.append(_host(k), _host(v), lens, counts)
    _same(cache, ref)


def test_append_after_tokens_are_dropped():
    """Lengths that go back (tokens that were tried and not taken), into a block
    and to a block's start, one sequence at a time."""
    Bn, H, cap, hd = 2, 2, 256, 64
    cache, ref = B.kv8_cache(Bn, H, cap, hd), R.Cache(Bn, H, cap, hd)
    for i, (lens, T) in enumerate((([0, 0], 150), ([140, 64], 8), ([128, 70], 5), ([3, 75], 1), ([4, 76], 130))):
        k, v = _kv((Bn, H, T, hd), 10 + i, 1.5), _kv((Bn, H, T, hd), 50 + i, 1.5)
        B.op_kv8_append(cache, k, v, _int32(lens))
        ref.append(_host(k), _host(v), lens)
        _same(cache, ref)


def test_append_special_values():
    """Zeros, tiny and huge values; a NaN or an infinity marks its block until
    the block is begun anew, and leaves the other blocks alone."""
    import torch
    Bn, H, cap, hd = 1, 1, 256, 64
    cache, ref = B.kv8_cache(Bn, H, cap, hd), R.Cache(Bn, H, cap, hd)
    k = torch.zeros(1, 1, 200, hd, device="cuda")
    k[..., 0:64, :] = 1e-30
    k[..., 64:128, :] = 3e38
    k[..., 130, 7] = float("inf")
    v = torch.randn(1, 1, 200, hd, device="cuda")
    v[..., 199, 3] = float("nan")
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    B.op_kv8_append(cache, k, v, _int32([0]))
    ref.append(_host(k), _host(v), [0])
    _same(cache, ref)
    more = _kv((1, 1, 2, hd), 9)
    B.op_kv8_append(cache, more, more, _int32([190]))
    ref.append(_host(more), _host(more), [190])
    _same(cache, ref)
    assert torch.isnan(cache[1][0, 0, 2]) and torch.isnan(cache[3][0, 0, 3])
    B.op_kv8_append(cache, more, more, _int32([128]))  # begun anew
    ref.append(_host(more), _host(more), [128])
    _same(cache, ref)
    assert not torch.isnan(cache[1][0, 0, 2])


def test_append_again_changes_nothing():
    import torch
    cache = B.kv8_cache(2, 3, 192, 128)
    a, b = _kv((2, 3, 90, 128), 1, 1.0), _kv((2, 3, 90, 128), 2, 1.0)
    B.op_kv8_append(cache, a, b, _int32([0, 0]))
    c, d = _kv((2, 3, 50, 128), 3, 1.0), _kv((2, 3, 50, 128), 4, 1.0)
    B.op_kv8_append(cache, c, d, _int32([90, 70]))
    once = [t.clone() for t in cache]
    B.op_kv8_append(cache, c, d, _int32([90, 70]))
    assert all(torch.equal(x, y) for x, y in zip(once, cache))


# ----------------------------------------------------------------- attention
def _filled(Bn, Hkv, cap, hd, tokens, seed, grow=0.5):
    """A device cache with `tokens` tokens of every sequence, its values in float64, and the codes' check."""
    cache = B.kv8_cache(Bn, Hkv, cap, hd)
    k, v = _kv((Bn, Hkv, tokens, hd), seed, grow), _kv((Bn, Hkv, tokens, hd), seed + 1, grow)
    B.op_kv8_append(cache, k, v, _int32([0] * Bn))
    return cache, _values(cache, hd)


def _values(cache, hd):
    out = []
    for codes, scales, index in ((cache[0], cache[1], R.key_index(hd)), (cache[2], cache[3], R.value_index(hd))):
        c, s = codes.cpu().numpy(), scales.cpu().numpy().astype(np.float64)
        x = R.E4M3[c[..., index.reshape(-1)]] * s[..., None]
        out.append(x.reshape(c.shape[0], c.shape[1], -1, hd))
    return out


def _heads(Hkv, T):
    """Query heads: two to a key/value head, and with 100 queries and more so
    many that the form for many columns (over 2048) runs."""
    return Hkv * (2 if T < 100 else -(-2100 // T))


def _check_attention(got, q, kv, lens, counts=None, window=0, sinks=0):
    """The output's rounding to bf16 (2^-8 of it), the probabilities' rounding
    to bf16 in the sum (2^-8 of sum p |v|) and in the sum that divides it
    (2^-8 of the result), and float32 scores and exponentials (2^-11)."""
    Bn, Hq, T, hd = q.shape
    ref, spread, there = R.attention(_host(q), kv, lens, counts, window, sinks)
    got = _host(got).reshape(Bn, T, Hq, hd).astype(np.float64)
    err = np.abs(got - ref)[there]
    tol = (2 * 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -11) * spread + 1e-30)[there]
    assert (err <= tol).all(), (err / tol).max()
    return there


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 2), (16, 1), (12, 1)])
@pytest.mark.parametrize("T,lens", [(1, [0, 63]), (1, [64, 255]), (1, [256, 511]), (1, [700, 13]), (2, [254, 62]), (3, [0, 500]),
                                    (16, [240, 1]), (17, [100, 0]), (40, [0, 600]), (70, [63, 250]), (130, [500, 0])])
def test_attention(hd, Hq, Hkv, T, lens):
    log(f"attention hd={hd} heads {Hq}/{Hkv} T={T} lens={lens}")
    cap = 768
    cache, kv = _filled(2, Hkv, cap, hd, cap, 5)
    q = _kv((2, Hq, T, hd), 9)
    out = B.op_attention_kv8(q, cache, _int32(lens))
    _check_attention(out, q, kv, lens)


@pytest.mark.parametrize("T,lens", [(1, [700, 20]), (5, [320, 0]), (50, [0, 300]), (200, [400, 100])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (64, 70), (200, 4), (300, 300), (5000, 2), (1 << 30, 1 << 30)])
def test_attention_window_and_sinks(T, lens, window, sinks):
    log(f"window {window} sinks {sinks} T={T} lens={lens}")
    cache, kv = _filled(2, 2, 768, 64, 768, 15)
    q = _kv((2, _heads(2, T), T, 64), 19)
    out = B.op_attention_kv8(q, cache, _int32(lens), window=window, sinks=sinks)
    _check_attention(out, q, kv, lens, window=window, sinks=sinks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("T,masks", [(1, [(0, 0), (100000, 5000), (70, 0)]), (20, [(100000, 5000), (70, 0)]), (600, [(3000, 4)])])
def test_attention_over_a_long_cache(hd, T, masks):
    """More tokens than the largest number of splits has by itself: longer
    splits, a lane for each in the join; windows that leave some of them out."""
    log(f"long cache hd={hd} T={T}")
    cap, Hq = 1 << 18, 2
    cache, kv = _filled(1, 1, cap, hd, cap, 35)
    q = _kv((1, Hq, T, hd), 39)
    n = cap - 700
    for window, sinks in masks:
        out = B.op_attention_kv8(q, cache, _int32([n]), window=window, sinks=sinks)
        _check_attention(out, q, kv, [n], window=window, sinks=sinks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5), (700, 0), (64, 600)])
def test_attention_prompt_in_splits(hd, window, sinks):
    """Few tiles and a cache of several splits: parts joined, some of them empty
    for all of a tile's queries, some for a few of them."""
    log(f"prompt splits hd={hd} window {window} sinks {sinks}")
    cap, T, lens, counts = 2368, 300, [0, 1900, 560], [300, 300, 17]
    cache, kv = _filled(3, 2, cap, hd, cap, 85)
    q = _kv((3, _heads(2, T), T, hd), 89)
    out = B.op_attention_kv8(q, cache, _int32(lens), _int32(counts), window=window, sinks=sinks)
    _check_attention(out, q, kv, lens, counts, window=window, sinks=sinks)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,T", [(2, 2, 130), (24, 8, 11), (5, 1, 51), (255, 1, 1), (256, 1, 1), (1024, 1, 1), (34, 2, 15), (3, 3, 256), (341, 1, 3), (682, 1, 3)])
def test_attention_few_columns(hd, Hq, Hkv, T):
    """Tiles of 16 columns up to 2048 of them, heads that are no power of two."""
    log(f"few columns hd={hd} heads {Hq}/{Hkv} T={T}")
    cap, lens = 1216 * (128 // hd), [0, 900 * (128 // hd)]  # two splits
    cache, kv = _filled(2, Hkv, cap, hd, cap, 95)
    q = _kv((2, Hq, T, hd), 99)
    for window, sinks in ((500, 2), (0, 0)):
        out = B.op_attention_kv8(q, cache, _int32(lens), window=window, sinks=sinks)
        _check_attention(out, q, kv, lens, window=window, sinks=sinks)


@pytest.mark.parametrize("T", [1, 20, 90, 300])
def test_attention_nan_queries_stay_in_their_rows(T):
    import torch
    cache, _ = _filled(1, 2, 640, 64, 640, 105)
    q = _kv((1, _heads(2, T), T, 64), 109)
    clean = B.op_attention_kv8(q, cache, _int32([300])).reshape(T, -1, 64)
    q[0, 1, T // 2, 7] = float("nan")
    q[0, 2, T - 1, 3] = float("inf")
    out = B.op_attention_kv8(q, cache, _int32([300])).reshape(T, -1, 64)
    bad = torch.zeros(clean.shape[:2], dtype=torch.bool, device="cuda")
    bad[T // 2, 1] = bad[T - 1, 2] = True
    assert torch.equal(out[~bad], clean[~bad]) and torch.isnan(out[bad]).any(-1).all()


@pytest.mark.parametrize("T", [1, 40, 200])
def test_attention_and_append_past_32_bits(T):
    """Codes past 4 GB and blocks past the last sequence's 2^31 bytes: the last
    sequence's tokens, seen through a window, as in a small cache."""
    import torch
    Bn, Hkv, Hq, hd, cap, window = 3, 16, 32, 128, 1 << 20, 100
    cache = tuple(torch.empty(s, dtype=dt, device="cuda") for s, dt in
                  ((((Bn, Hkv, cap // 64, 64 * hd)), torch.uint8), ((Bn, Hkv, cap // 64), torch.float32)) * 2)
    first = cap - 64 * 20
    k, v = _kv((1, Hkv, 1280, hd), 45), _kv((1, Hkv, 1280, hd), 46)
    three = lambda t: t.expand(Bn, -1, -1, -1).contiguous()
    B.op_kv8_append(cache, three(k), three(v), _int32([0, 0, first]), _int32([0, 0, 1280]))
    small = B.kv8_cache(1, Hkv, 1280, hd)
    B.op_kv8_append(small, k, v, _int32([0]))
    assert all(torch.equal(c[2:, :, -20:], s) for c, s in zip(cache, small))
    q = _kv((1, Hq, T, hd), 49)
    out = B.op_attention_kv8(three(q), cache, _int32([0, 0, first + 150]), _int32([0, 0, T]), window=window)
    _check_attention(out.reshape(Bn, T, -1)[2], q, _values(small, hd), [150], window=window)


def test_attention_refuses_lengths_on_the_host():
    import torch
    cache, _ = _filled(1, 1, 64, 64, 64, 1)
    q, k = _kv((1, 1, 1, 64), 2), _kv((1, 1, 1, 64), 3)
    host = torch.tensor([5], dtype=torch.int32)
    for call in (lambda: B.op_attention_kv8(q, cache, host), lambda: B.op_kv8_append(cache, k, k, host),
                 lambda: B.op_kv8_append(cache, k.cpu(), k, _int32([5])),
                 lambda: B.op_attention_kv8(q, cache, _int32([5]), host)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("T", [1, 3, 33, 150])
def test_attention_ragged_rows_are_left(T):
    """counts, lengths at and past the cache's ends: rows without a token keep what they held."""
    import torch
    Bn, Hq, Hkv, hd, cap = 7, _heads(2, T), 2, 64, 320
    lens, counts = [0, 10, 300, 319, 320, -5, 64], [T, 0, T, T, T, T, max(1, T - 2)]
    cache, kv = _filled(Bn, Hkv, cap, hd, cap, 25)
    q = _kv((Bn, Hq, T, hd), 29)
    out = torch.full((Bn * T, Hq * hd), 7.0, dtype=torch.bfloat16, device="cuda")
    B.op_attention_kv8(q, cache, _int32(lens), _int32(counts), out=out)
    there = _check_attention(out, q, kv, lens, counts)
    rows = _host(out).reshape(Bn, T, -1)
    assert (rows[~there] == 7).all()
    assert not there[1].any() and not there[4].any() and not there[5].any()


@pytest.mark.parametrize("T", [1, 20, 100, 150])
def test_attention_masked_tokens_count_for_nothing(T):
    """Blocks with a NaN scale (keys or values) behind the window and past the
    last token change no bit; a visible one gives NaN."""
    import torch
    cap, hd, n = 512, 64, 300
    cache, _ = _filled(1, 1, cap, hd, cap, 35)
    q = _kv((1, _heads(1, T), T, hd), 39)
    clean = B.op_attention_kv8(q, cache, _int32([n]), window=64, sinks=0)
    bad = [t.clone() for t in cache]
    first = (n - 63) // 64       # block of the first query's first key
    last = (n + T - 1) // 64
    for t in (bad[1], bad[3]):
        t[..., :first] = float("nan")
        t[..., last + 1:] = float("nan")
    assert torch.equal(B.op_attention_kv8(q, bad, _int32([n]), window=64, sinks=0), clean)
    for which in (1, 3):
        b2 = [t.clone() for t in cache]
        b2[which][..., last] = float("nan")
        out = B.op_attention_kv8(q, b2, _int32([n]), window=64, sinks=0).reshape(T, -1)
        sees = torch.arange(n, n + T, device="cuda") >= 64 * last
        assert torch.isnan(out[sees]).all() and torch.equal(out[~sees], clean.reshape(T, -1)[~sees])


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_extreme_scores(hd):
    """Scores far above and below, equal everywhere, and a block of zero values."""
    import torch
    cap = 576
    k, v = _kv((1, 2, cap, hd), 45), _kv((1, 2, cap, hd), 46)
    k[..., 100, :] *= 40
    k[..., 200:264, :] = 0
    v[..., 300:400, :] = 0
    cache = B.kv8_cache(1, 2, cap, hd)
    B.op_kv8_append(cache, k, v, _int32([0]))
    kv = _values(cache, hd)
    for T, n in ((1, 575), (30, 500), (200, 376), (300, 276)):
        for f in (0.0, 1.0, 6.0):
            q = _kv((1, _heads(2, T), T, hd), 47) * f
            _check_attention(B.op_attention_kv8(q, cache, _int32([n])), q, kv, [n])


@pytest.mark.parametrize("T", [1, 4, 30, 90, 150])
def test_attention_queries_do_not_depend_on_others(T):
    """A sequence alone gives the bits it has in a batch; and a few queries
    (whose splits have a length of their own) those of a wider cache."""
    import torch
    cap, hd, Hkv = 1152, 128, 2
    cache, _ = _filled(3, Hkv, cap, hd, cap, 55)
    q = _kv((3, _heads(Hkv, T), T, hd), 59)
    lens = [1000, 30, 513]
    whole = B.op_attention_kv8(q, cache, _int32(lens), window=400, sinks=3).reshape(3, T, -1)
    for b in range(3):
        one = [t[b:b + 1].contiguous() for t in cache]
        out = B.op_attention_kv8(q[b:b + 1].contiguous(), one, _int32(lens[b:b + 1]), window=400, sinks=3)
        assert torch.equal(out.reshape(T, -1), whole[b])
        if 2 * T > 32:
            continue
        big = B.kv8_cache(1, Hkv, 4096, hd)
        for t, o in zip(big, one):
            t[:, :, :cap // 64] = o
        out = B.op_attention_kv8(q[b:b + 1].contiguous(), big, _int32(lens[b:b + 1]), window=400, sinks=3)
        assert torch.equal(out.reshape(T, -1), whole[b])


def test_attention_in_graphs():
    """Append and attention captured once, replayed as the lengths move on the
    device, with eager work between the replays."""
    import torch
    Bn, Hq, Hkv, hd, cap = 2, 4, 2, 64, 512
    eager, cap_cache = B.kv8_cache(Bn, Hkv, cap, hd), B.kv8_cache(Bn, Hkv, cap, hd)
    k0, v0 = _kv((Bn, Hkv, 250, hd), 61), _kv((Bn, Hkv, 250, hd), 62)
    for c in (eager, cap_cache):
        B.op_kv8_append(c, k0, v0, _int32([0, 0]), _int32([250, 190]))
    k, v, q = (torch.zeros((Bn, h, 1, hd), dtype=torch.bfloat16, device="cuda") for h in (Hkv, Hkv, Hq))
    lens = _int32([250, 190])
    ws = B.workspace(B.kv8_workspace(Bn, Hq, Hkv, 1, hd, cap))
    out = torch.empty((Bn, Hq * hd), dtype=torch.bfloat16, device="cuda")

    def step():
        B.op_kv8_append(cap_cache, k, v, lens)
        B.op_attention_kv8(q, cap_cache, lens, out=out, ws=ws)
        lens.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    saved = [t.clone() for t in cap_cache]
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t, s in zip(cap_cache, saved):
        t.copy_(s)
    lens.copy_(_int32([250, 190]))
    for i in range(8):
        nk, nv, nq = _kv((Bn, Hkv, 1, hd), 70 + i, 1.0), _kv((Bn, Hkv, 1, hd), 90 + i, 1.0), _kv((Bn, Hq, 1, hd), 110 + i)
        k.copy_(nk), v.copy_(nv), q.copy_(nq)
        g.replay()
        torch.cuda.synchronize()
        now = _int32([250 + i, 190 + i])
        B.op_kv8_append(eager, nk, nv, now)
        want = B.op_attention_kv8(nq, eager, now)
        assert torch.equal(out, want), i
        assert all(torch.equal(a, b) for a, b in zip(eager, cap_cache))


def test_other_streams():
    import torch
    cache, kv = _filled(1, 2, 512, 64, 512, 81)
    q = _kv((1, 4, 2, 64), 82)
    want = B.op_attention_kv8(q, cache, _int32([400]))
    lens = _int32([400])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [B.op_attention_kv8(q, cache, lens, stream=s, ws=B.workspace(B.kv8_workspace(1, 4, 2, 2, 64, 512))) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


# ------------------------------------------------------------- run together
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_decoder_layer_steps(fmt):
    """Half a decoder layer (add + norm, QKV product, append, attention, O
    product with the residual) over a prompt and then single tokens, each
    operator fed by the one before, against float64 on the same codes."""
    import torch
    Bn, Hq, Hkv, hd, cap, d = 2, 4, 2, 64, 256, 256
    nq, nkv = Hq * hd, Hkv * hd
    g = torch.Generator(device="cuda").manual_seed(7)

    def weight(n, k):
        codes, scales = B.op_mx_quantize(torch.randn(n, k, generator=g, device="cuda") * k ** -0.5, "fp4")
        w = B.op_mx_dequantize(codes, scales, "fp4", k).double().cpu().numpy()
        return B.op_mx_block(codes, scales, k), w

    (wq, wqs), wqkv = weight(nq + 2 * nkv, d)
    (wo, wos), wout = weight(d, nq)
    gain = torch.ones(d, device="cuda")
    cache = B.kv8_cache(Bn, Hkv, cap, hd)
    lens = np.array([0, 0])
    for T in (90, 1, 1, 1):
        h = torch.randn(Bn * T, d, generator=g, device="cuda")
        x = torch.randn(Bn * T, d, generator=g, device="cuda").to(torch.bfloat16)
        codes, scales = B.op_add_norm_mx(h, x, gain, 1e-5, fmt, out=h)
        y = B.op_mx_dequantize(codes, scales, fmt, d).double().cpu().numpy()
        qkv = B.op_gemm_mx(codes, scales, fmt, wq, wqs, nq + 2 * nkv, d, "bf16")
        assert (np.abs(_host(qkv) - y @ wqkv.T) <= _mm_tol(y, wqkv)).all()
        heads = qkv.reshape(Bn, T, Hq + 2 * Hkv, hd).transpose(1, 2)
        q, k, v = (t.contiguous() for t in heads.split([Hq, Hkv, Hkv], dim=1))
        tl = _int32(lens)
        B.op_kv8_append(cache, k, v, tl)
        o = B.op_attention_kv8(q, cache, tl)
        _check_attention(o, q, _values(cache, hd), lens)
        oc, osc = B.op_mx_quantize(o, fmt)
        ov = B.op_mx_dequantize(oc, osc, fmt, nq).double().cpu().numpy()
        before = h.double().cpu().numpy()
        B.op_gemm_mx(oc, osc, fmt, wo, wos, d, nq, "store", add=h, out=h)
        assert (np.abs(_host(h) - (before + ov @ wout.T)) <= _mm_tol(ov, wout) + 2.0 ** -23 * np.abs(before)).all()
        lens = lens + T


def _mm_tol(a, b):
    """Both formats: the bf16 rounding of the result, and a step's dropped bits (2^-18 of its largest product, 128 products)."""
    ref, mag = np.abs(a @ b.T), np.abs(a) @ np.abs(b).T
    drop = sum(128 * 2.0 ** -18 * np.outer(np.abs(a[:, k:k + 128]).max(1), np.abs(b[:, k:k + 128]).max(1))
               for k in range(0, a.shape[1], 128))
    return 2.0 ** -8 * ref + 2.0 ** -20 * mag + 1.01 * drop
