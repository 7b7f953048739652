"""Calls of the rotary positions and the paged cache that have to be refused before
anything is launched, and what the host computes for them."""
import numpy as np
import pytest

from paper_2409_17836_amd import binding as B

EINVAL, ESIZE, EUNSUPPORTED = -1, -4, -6
AT = [0x10000000000 + (i << 36) for i in range(14)]  # addresses that are never read


# --------------------------------------------------------------- frequencies
@pytest.mark.parametrize("rot", [2, 6, 32, 128, 512])
def test_frequencies(rot):
    i = np.arange(rot // 2)
    plain = 10000.0 ** (-2.0 * i / rot)
    # pow is within an ulp or two; factors, quotients and the ramp add some more
    def near(a, b):
        np.testing.assert_allclose(a, b, rtol=2.0 ** -49, atol=0)
    near(B.rope_frequencies(rot), plain)
    near(B.rope_frequencies(rot, scaling="linear", factor=8.0), plain / 8)
    if rot > 2:
        near(B.rope_frequencies(rot, 500.0, "ntk", 4.0), (500.0 * 4.0 ** (rot / (rot - 2))) ** (-2.0 * i / rot))
    f = B.rope_frequencies(rot, 10000.0, "yarn", 16.0, 2048)
    turns = 2048 * plain / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    near(f, plain * keep + plain / 16 * (1 - keep))
    # fast dims keep their angles, slow ones are interpolated as a whole
    near(f[turns > 32], plain[turns > 32])
    near(f[turns < 1], plain[turns < 1] / 16)


def test_frequencies_refusals():
    for kw in (dict(rot=3), dict(rot=0), dict(rot=514), dict(rot=8, theta=0.0), dict(rot=8, theta=float("nan")),
               dict(rot=8, scaling="linear", factor=0.5), dict(rot=8, scaling="yarn", factor=float("inf")), dict(rot=2, scaling="ntk", factor=2.0),
               dict(rot=8, scaling="yarn", factor=2.0, orig=0), dict(rot=8, scaling="yarn", factor=2.0, slow=4, fast=4)):
        with pytest.raises(B.LMGCError) as e:
            B.rope_frequencies(**kw)
        assert e.value.code == EINVAL
    assert B.lib().lmgc_rope_frequencies(1e4, 8, 0, 1.0, 1.0, 1.0, 2.0, None) == EINVAL
    assert B.lib().lmgc_rope_frequencies(1e4, 8, 4, 1.0, 1.0, 1.0, 2.0, None) == EINVAL


# ------------------------------------------------------------------ refusals
def _table(**kw):
    import ctypes
    f = (ctypes.c_double * 256)(*[1.0] * 256)
    a = dict(freqs=f, rot=64, mscale=1.0, n_pos=128, table=AT[0])
    a.update(kw)
    return B.lib().lmgc_op_rope_table(a["freqs"], a["rot"], a["mscale"], a["n_pos"], a["table"], None)


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=7), dict(rot=514), dict(n_pos=0), dict(n_pos=(1 << 24) + 1), dict(table=None),
                                dict(table=AT[0] + 8), dict(freqs=None), dict(mscale=float("nan"))])
def test_rope_table_refusals(kw):
    assert _table(**kw) == EINVAL


def test_rope_table_takes_finite_frequencies():
    import ctypes
    f = (ctypes.c_double * 32)(*[1.0] * 31 + [float("inf")])
    assert _table(freqs=f) == EINVAL


def _rope(**kw):
    a = dict(x=AT[0], dtype=0, n=4, heads=2, hd=64, ldx=128, ldhx=64, pos=AT[1], table=AT[2], n_pos=128, rot=64, layout=0, back=0,
             out=AT[3], ldo=128, ldho=64)
    a.update(kw)
    return B.lib().lmgc_op_rope(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(n=-1), dict(n=(1 << 24) + 1), dict(heads=0), dict(hd=1), dict(hd=513, ldx=2000, ldhx=513), dict(rot=66), dict(rot=63),
    dict(layout=2), dict(n_pos=0), dict(table=None), dict(table=AT[2] + 4), dict(x=None), dict(out=None), dict(pos=None), dict(x=AT[0] + 2),
    dict(pos=AT[1] + 1), dict(ldhx=63), dict(ldx=127, ldhx=64), dict(ldx=1 << 41), dict(ldhx=1 << 41),
    dict(out=AT[0] + 4), dict(out=AT[0], ldo=192), dict(out=AT[1] - 64), dict(out=AT[2] + 64),
    dict(ldx=64, ldhx=4 * 64 - 1)])
def test_rope_refusals(kw):
    assert _rope(**kw) == EINVAL


def test_rope_of_no_rows_is_fine():
    assert _rope(n=0, x=None, out=None, pos=None) == 0


def _append(**kw):
    a = dict(k=AT[0], v=AT[1], dtype=1, ldk=128, ldv=128, n=8, B=2, Hkv=2, hd=64, kc=AT[2], vc=AT[3], n_pages=4, page=64, pages=AT[4],
             most=2, starts=AT[5], lens=AT[6], table=AT[7], n_pos=128, rot=64, layout=0, q=AT[8], ldq=256, Hq=4, qo=AT[9], ldqo=256)
    a.update(kw)
    return B.lib().lmgc_op_paged_append(*a.values(), None)


POOL = 4 * 2 * 64 * 64 * 2  # bytes of the pools of these calls


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(n=-1), dict(n=(1 << 24) + 1), dict(B=0), dict(B=65536), dict(Hkv=0), dict(Hkv=4097), dict(Hq=3), dict(Hq=0),
    dict(n_pages=0), dict(most=0), dict(most=1 << 19), dict(kc=None), dict(vc=None), dict(pages=None), dict(starts=None), dict(lens=None),
    dict(k=None), dict(v=None), dict(q=None), dict(qo=None), dict(table=None), dict(kc=AT[2] + 8), dict(vc=AT[3] + 2), dict(pages=AT[4] + 2),
    dict(k=AT[0] + 1), dict(dtype=0, v=AT[1] + 2), dict(ldk=127), dict(ldv=1 << 41), dict(ldq=255), dict(ldqo=255), dict(rot=66), dict(rot=1),
    dict(layout=2), dict(n_pos=0), dict(table=AT[7] + 8), dict(vc=AT[2] + POOL - 16), dict(k=AT[2] + 16), dict(v=AT[3] + POOL - 2),
    dict(q=AT[2]), dict(qo=AT[3] + 32), dict(table=AT[2] + 16), dict(lens=AT[2] + 4), dict(starts=AT[3]), dict(pages=AT[9] + 4), dict(qo=AT[8]),
    dict(qo=AT[0]), dict(qo=AT[7] + 2)])
def test_append_refusals(kw):
    assert _append(**kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(hd=96), dict(hd=32), dict(page=16), dict(page=48), dict(page=512)])
def test_append_unsupported(kw):
    assert _append(**kw) == EUNSUPPORTED


def test_append_of_no_rows_is_fine():
    assert _append(n=0, k=None, v=None) == 0


def _attention(**kw):
    a = dict(q=AT[0], ldq=256, n=8, B=2, Hq=4, Hkv=2, hd=64, kc=AT[2], vc=AT[3], n_pages=4, page=64, pages=AT[4], most=2, starts=AT[5],
             lens=AT[6], max_new=8, window=0, sinks=0, shared=0, scale=0.125, out=AT[7], ws=AT[8], bytes=1 << 30)
    a.update(kw)
    return B.lib().lmgc_op_attention_paged(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(B=0), dict(Hq=3), dict(Hkv=0), dict(n_pages=0), dict(most=0), dict(max_new=0), dict(max_new=(1 << 24) + 1), dict(window=-1),
    dict(sinks=-1), dict(shared=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
    dict(out=None), dict(kc=None), dict(lens=None), dict(q=AT[0] + 2), dict(ldq=255), dict(ldq=260), dict(out=AT[7] + 8), dict(ws=AT[8] + 8),
    dict(out=AT[0] + 64), dict(out=AT[2]), dict(lens=AT[7]), dict(starts=AT[7] + 16), dict(pages=AT[7] + 8 * 4 * 64 * 2 - 4)])
def test_attention_refusals(kw):
    assert _attention(**kw) == EINVAL


@pytest.mark.parametrize("kw", [dict(hd=80), dict(page=24)])
def test_attention_unsupported(kw):
    assert _attention(**kw) == EUNSUPPORTED


def test_attention_of_more_columns_than_a_launch_has():
    """(of the batch, behind a prefix: rows of no token count too)"""
    rows = dict(n=1 << 24, Hq=1024, Hkv=64, ldq=1 << 16, max_new=1, n_pages=1, page=64, bytes=1 << 62, ws=1 << 58, q=1 << 55, out=1 << 56)
    assert _attention(**rows, shared=64) == EUNSUPPORTED
    rows["max_new"] = 1 << 24
    assert _attention(**rows) == EUNSUPPORTED


def test_attention_counts_only_what_it_launches():
    """65535 sequences of few columns have no use for the form for many, nor have longer ones
    behind a window that is one part of keys: such calls come as far as the workspace."""
    rows = dict(n=65535, B=65535, Hq=32, Hkv=32, ldq=32 * 64, most=512, max_new=1, n_pages=1, page=64, bytes=0, ws=None, q=1 << 55, out=1 << 56)
    assert _attention(**rows) == ESIZE
    rows.update(n=65535 * 16, Hq=128, ldq=128 * 64, max_new=16)
    assert _attention(**rows) == ESIZE
    rows.update(max_new=17)  # 68 columns
    assert _attention(**rows) == EUNSUPPORTED and _attention(**rows, window=64) == ESIZE


def test_attention_scale_in_powers_of_two():
    """log2(e) times the scale, which scores are multiplied by, has to be a number too."""
    assert _attention(scale=3e38) == EINVAL
    assert _attention(scale=2.3e38, most=128, page=256, ws=None) == ESIZE  # (as far as the workspace)


def test_attention_of_no_rows_is_fine():
    assert _attention(n=0, q=None, out=None, ws=None, bytes=0) == 0


def test_attention_workspace():
    """Refused where it is too small or in the way; sizes do not fall with the batch."""
    long = dict(most=128, page=256, n_pages=4)
    need = B.paged_workspace(8, 2, 4, 2, 64, 8, 128 * 256)
    assert need > 0
    assert _attention(**long, bytes=need - 1) == ESIZE and _attention(**long, ws=None, bytes=need) == ESIZE
    for ws in (AT[0] - 16, AT[7] + 16, AT[2] - 16, AT[3] + 16):
        assert _attention(**long, ws=ws, bytes=need) == EINVAL
    for at in ("lens", "starts", "pages"):
        assert _attention(**long, bytes=need, **{at: AT[8] + need - 4}) == EINVAL
    assert B.paged_workspace(0, 1, 4, 2, 64, 8, 4096) == 0
    assert B.paged_workspace(8, 2, 4, 2, 64, 8, 128 * 256, 4096) >= need
    for bad in ((8, 2, 4, 2, 64, 0, 64), (8, 2, 4, 2, 64, 1, 0), (8, 2, 4, 2, 64, 1, 64, -1), (8, 2, 5, 2, 64, 1, 64)):
        with pytest.raises(B.LMGCError):
            B.paged_workspace(*bad)


def test_attention_workspace_is_what_rows_fill():
    """A chunk beside single tokens: the partial results of its rows, not those of a chunk for
    each sequence."""
    part = (128 + 2) * 4  # bytes of a partial result
    for singles in (63, 255):
        rows = 64 + singles
        # 64 parts of 512 tokens for each row and head
        assert B.paged_workspace(rows, singles + 1, 32, 32, 128, 64, 32768) <= rows * 32 * 64 * part
        assert B.paged_workspace(rows, singles + 1, 32, 8, 128, 16, 32768) <= rows * 32 * 64 * part
    # nor those of each row of a long prompt, where few sequences have few columns
    assert B.paged_workspace(6000, 2, 32, 32, 128, 6000, 32768) <= 2 * 32 * 64 * 64 * part
    # single tokens: a column of each
    assert B.paged_workspace(64, 64, 32, 8, 128, 1, 32768) == 64 * 32 * 64 * part


# ------------------------------------------------------------------- binding
def _batch(n=4, Bn=2, most=2):
    import torch
    return torch.zeros(Bn, most, dtype=torch.int32), torch.zeros(Bn + 1, dtype=torch.int32), torch.zeros(Bn, dtype=torch.int32)


def test_binding_refuses_wrong_tensors():
    import torch
    cache = B.paged_cache(4, 2, 64, 64, device="cpu")
    pages, starts, lens = _batch()
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    q = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    bad = [dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)), dict(v=k.float()), dict(pages=pages.long()), dict(starts=starts[:2]),
           dict(lens=lens.repeat(2)[::2]), dict(cache=(cache[0], cache[1].float())), dict(cache=(cache[0], cache[1][:3])), dict(q=q.float()),
           dict(rope=torch.zeros(8, 32, 3)), dict(q_out=q)]
    for kw in bad:
        a = dict(cache=cache, k=k, v=k, pages=pages, starts=starts, lens=lens)
        a.update(kw)
        with pytest.raises(AssertionError):
            B.op_paged_append(**a)
    for kw in (dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(out=torch.zeros(4, 256)), dict(ws=torch.zeros(64, dtype=torch.uint8)[::2]),
               dict(pages=pages.t()), dict(starts=starts[1:])):
        a = dict(q=q, cache=cache, pages=pages, starts=starts, lens=lens, max_new=1)
        a.update(kw)
        with pytest.raises(AssertionError):
            B.op_attention_paged(**a)
    x, pos, table = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(8, 32, 2)
    for kw in (dict(x=x.transpose(1, 2)), dict(positions=pos.long()), dict(positions=pos[:2]), dict(table=table.double()), dict(table=table[::2]),
               dict(out=x.bfloat16()), dict(x=x.half())):
        a = dict(x=x, positions=pos, table=table)
        a.update(kw)
        with pytest.raises((AssertionError, RuntimeError)):
            B.op_rope(**a)


class _Library:
    """Takes the place of the library: keeps the arguments of the attention call."""

    def __init__(self, real):
        self.real, self.args = real, None

    def __getattr__(self, name):
        return getattr(self.real, name)

    def lmgc_op_attention_paged(self, *args):
        self.args = args
        return 0


@pytest.mark.parametrize("given,taken", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 32 + 16, 2 ** 31 - 1), (-1, -1), (-2 ** 32 + 5, -1)])
def test_windows_past_32_bits(monkeypatch, given, taken):
    import torch
    fake = _Library(B.lib())
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(B, "_on", lambda stream, *tensors: (0, [0] * len(tensors)))
    cache = B.paged_cache(4, 2, 64, 64, device="cpu")
    ws = torch.zeros(1 << 12, dtype=torch.float32)
    args = (torch.zeros(4, 4, 64, dtype=torch.bfloat16), cache, *_batch(), 1)
    for i, name in enumerate(("window", "sinks", "shared")):
        B.op_attention_paged(*args, ws=ws, **{name: given})
        assert fake.args[-8 + i] == taken
    assert fake.args[-2] == 4 * (1 << 12)  # bytes of the workspace


@pytest.mark.parametrize("at", range(8))
@pytest.mark.parametrize("past", [1 << 32, -(1 << 32)])
def test_sizes_past_32_bits(at, past):
    """They are refused, not taken for what their low 32 bits hold."""
    sizes = [8, 2, 4, 2, 64, 8, 4096, 0]
    assert B.paged_workspace(*sizes) > 0
    if at == 7 and past > 0:  # (more in common than there is: all of it)
        assert B.paged_workspace(*sizes[:7], past) == B.paged_workspace(*sizes[:7], 4096)
        return
    sizes[at] += past
    with pytest.raises(B.LMGCError):
        B.paged_workspace(*sizes)
    with pytest.raises(B.LMGCError) as e:
        B.rope_frequencies(64 + past)
    assert e.value.code == EINVAL
