"""Calls of the operators in fewer bits that have to be refused, or whose
arguments have to be brought into range, before anything is launched."""
import pytest

from paper_2409_17836_amd import binding as B

EINVAL = -1
SRC, CODES, SCALES, OUT = 1 << 44, 1 << 45, 1 << 46, 1 << 47  # addresses that are never read


def test_attention_workspace_is_plain_bytes():
    """A workspace whose elements do not lie one behind the other has less memory
    behind its address than it has elements; refused like every other tensor
    that is not contiguous (so without a GPU too)."""
    import torch
    B_, Hq, Hkv, T, hd, cap = 1, 4, 2, 1, 64, 4096
    need = B.kv8_workspace(B_, Hq, Hkv, T, hd, cap)
    assert need > 0
    cache = B.kv8_cache(B_, Hkv, cap, hd, device="cpu")
    q = torch.zeros((B_, Hq, T, hd), dtype=torch.bfloat16)
    lens = torch.zeros(B_, dtype=torch.int32)
    one = torch.zeros(1, dtype=torch.uint8)
    for ws in (one.expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2], one.expand(2, need)):
        with pytest.raises(AssertionError):
            B.op_attention_kv8(q, cache, lens, ws=ws)


class _Library:
    """Takes the place of the library: keeps the arguments of the attention call."""

    def __init__(self, real):
        self.real, self.args = real, None

    def __getattr__(self, name):
        return getattr(self.real, name)

    def lmgc_op_attention_kv8(self, *args):
        self.args = args
        return 0


def _attention_args(monkeypatch, **kw):
    import torch
    fake = _Library(B.lib())
    monkeypatch.setattr(B, "lib", lambda: fake)
    monkeypatch.setattr(B, "_on", lambda stream, *tensors: (0, [0] * len(tensors)))
    cache = B.kv8_cache(1, 2, 4096, 64, device="cpu")
    B.op_attention_kv8(torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16), cache, torch.zeros(1, dtype=torch.int32), **kw)
    return fake.args


def test_attention_workspace_counts_bytes(monkeypatch):
    """The size that the library is told is in bytes, whatever the tensor's elements are."""
    import torch
    need = B.kv8_workspace(1, 4, 2, 1, 64, 4096)
    assert _attention_args(monkeypatch, ws=torch.zeros(need // 4, dtype=torch.float32))[-2] == need


def test_strides_past_the_address_space_are_refused():
    """Rows that lie so far apart that the matrix's extent in bytes passes 64
    bits: its overlap with the other buffers cannot be told from a wrapped
    extent, and no such matrix exists.  (2^24 rows 2^40 elements apart: 2^66 and
    2^65 bytes, zero in 64 bits.)"""
    rows = (1 << 24) + 1
    for dtype in (0, 1):
        for r, ld in ((rows, 1 << 40), ((1 << 31) - 1, 1 << 40), (rows, (1 << 39) + 1), (1 << 30, 1 << 20)):
            assert B.lib().lmgc_op_mx_quantize(SRC, dtype, r, 1, ld, 0, SRC + (1 << 20), SCALES, None) == EINVAL
            assert B.lib().lmgc_op_mx_dequantize(CODES, SCALES, 0, r, 1, CODES + (r << 8), dtype, ld, None) == EINVAL


@pytest.mark.parametrize("given,taken", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32 + 16, 2 ** 31 - 1),
                                         (10 ** 30, 2 ** 31 - 1), (-1, -1), (-2 ** 32 + 5, -1)])
def test_attention_windows_and_sinks_past_32_bits(monkeypatch, given, taken):
    """Positions end at 2^24, so more than 2^31 - 1 is the same as that, and is
    not cut to its low bits; what is negative stays so (and is refused)."""
    assert _attention_args(monkeypatch, window=given)[-6:-4] == (taken, 0)
    assert _attention_args(monkeypatch, sinks=given)[-6:-4] == (0, taken)


def test_lengths_inside_what_a_call_writes_are_refused():
    """lens and counts are read while the call runs: not in its output, its
    workspace or (for an append) the cache."""
    lib, at = B.lib(), [0x10000000 + (i << 24) for i in range(12)]
    kc, ks, vc, vs, q, out, ws, k, v = at[1:10]
    Bn, Hq, Hkv, T, hd, cap = 4, 4, 2, 1, 64, 4096
    need = B.kv8_workspace(Bn, Hq, Hkv, T, hd, cap)

    def attention(lens, counts=None):
        return lib.lmgc_op_attention_kv8(q, Bn, Hq, Hkv, T, hd, cap, lens, counts, kc, ks, vc, vs, 0, 0, out, ws, need, None)

    def append(lens, counts=None):
        return lib.lmgc_op_kv8_append(k, v, Bn, Hkv, T, hd, cap, lens, counts, kc, ks, vc, vs, None)
    for buffer in (out, out + Bn * T * Hq * hd * 2 - 4, ws, ws + need - 4):
        assert attention(buffer) == EINVAL and attention(at[0], buffer) == EINVAL
    for buffer in (kc, kc - 12, ks, vc + 256, vs + 4 * Bn * Hkv * (cap // 64) - 4):
        assert append(buffer) == EINVAL and append(at[0], buffer) == EINVAL


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_binding_sizes_are_the_library_s(fmt):
    for rows, cols in ((1, 1), (3, 127), (5, 128), (7, 129), (2, 512), (9, 513), (4, 11008), (1, 1 << 20)):
        nc, ns = B._mx_sizes(rows, cols, fmt)
        assert rows * nc == B.lib().lmgc_mx_code_bytes(B.MX_FORMATS[fmt], rows, cols)
        assert rows * ns == B.lib().lmgc_mx_scale_bytes(rows, cols)
