"""The operators in fewer bits without a GPU: their sizes, and the calls they
refuse before anything is launched."""
import ctypes

import pytest

from paper_2409_17836_amd import binding as B

EINVAL, ESIZE, EUNSUPPORTED = -1, -4, -6
# addresses that are never read: every call here is refused on its arguments
A = [0x10000000 + (i << 24) for i in range(12)]


def rc(name, *args):
    return getattr(B.lib(), name)(*args)


@pytest.mark.parametrize("rows,cols", [(0, 1), (1, 1), (3, 31), (5, 128), (17, 129), (16, 512), (33, 513), (2, 11008)])
def test_sizes(rows, cols):
    kp, ns = -(-cols // 128) * 128, 16 * -(-cols // 512)
    n16 = -(-rows // 16) * 16
    assert rc("lmgc_mx_code_bytes", 0, rows, cols) == rows * kp
    assert rc("lmgc_mx_code_bytes", 1, rows, cols) == rows * kp // 2
    assert rc("lmgc_mx_scale_bytes", rows, cols) == rows * ns
    assert rc("lmgc_mx_block_code_bytes", rows, cols) == n16 * kp // 2
    assert rc("lmgc_mx_block_scale_bytes", rows, cols) == n16 * ns


def test_sizes_refuse():
    for fmt, rows, cols in ((2, 1, 1), (-1, 1, 1), (0, -1, 1), (0, 1 << 31, 1), (0, 1, 0), (0, 1, (1 << 20) + 1)):
        assert rc("lmgc_mx_code_bytes", fmt, rows, cols) == EINVAL
    assert rc("lmgc_mx_scale_bytes", 1, 0) == EINVAL
    assert rc("lmgc_mx_block_code_bytes", -1, 8) == EINVAL
    assert rc("lmgc_mx_block_scale_bytes", 1, 1 << 21) == EINVAL
    # large matrices pass 32 bits without wrapping
    assert rc("lmgc_mx_code_bytes", 0, (1 << 31) - 1, 1 << 20) == ((1 << 31) - 1) << 20


def test_quantize_refuses():
    def q(src=A[0], dtype=0, rows=4, cols=64, ld=64, fmt=0, codes=A[1], scales=A[2]):
        return rc("lmgc_op_mx_quantize", src, dtype, rows, cols, ld, fmt, codes, scales, None)
    assert q(rows=0) == 0 and q(rows=0, src=None, codes=None, scales=None) == 0
    for bad in (dict(src=None), dict(codes=None), dict(scales=None), dict(dtype=2), dict(fmt=2), dict(rows=-1),
                dict(cols=0), dict(ld=63), dict(src=A[0] + 2), dict(src=A[0] + 1, dtype=1), dict(codes=A[1] + 8),
                dict(scales=A[2] + 4), dict(codes=A[0]), dict(scales=A[0] + 16), dict(scales=A[1])):
        assert q(**bad) == EINVAL, bad


def test_dequantize_and_block_refuse():
    def d(codes=A[0], scales=A[1], fmt=1, rows=4, cols=64, out=A[2], dtype=0, ld=64):
        return rc("lmgc_op_mx_dequantize", codes, scales, fmt, rows, cols, out, dtype, ld, None)
    assert d(rows=0) == 0
    for bad in (dict(codes=None), dict(scales=None), dict(out=None), dict(fmt=7), dict(dtype=5), dict(cols=0),
                dict(ld=10), dict(out=A[2] + 2), dict(codes=A[0] + 1), dict(out=A[0]), dict(out=A[1])):
        assert d(**bad) == EINVAL, bad

    def b(codes=A[0], scales=A[1], n=20, k=64, bc=A[2], bs=A[3]):
        return rc("lmgc_op_mx_block", codes, scales, n, k, bc, bs, None)
    assert b(n=0) == 0
    for bad in (dict(codes=None), dict(bs=None), dict(n=-1), dict(k=0), dict(bc=A[0]), dict(bs=A[1]), dict(bs=A[2]),
                dict(bc=A[2] + 4)):
        assert b(**bad) == EINVAL, bad


def test_add_norm_refuses():
    def n(h=A[0], hd=0, x=A[1], xd=1, g=A[2], gd=1, eps=1e-5, M=4, d=64, fmt=0, out=A[3], codes=A[4], scales=A[5]):
        return rc("lmgc_op_add_norm_mx", h, hd, x, xd, g, gd, eps, M, d, fmt, out, codes, scales, None)
    assert n(M=0) == 0
    for bad in (dict(h=None), dict(g=None), dict(codes=None), dict(scales=None), dict(hd=2), dict(xd=2), dict(gd=-1),
                dict(fmt=2), dict(eps=-1.0), dict(eps=float("nan")), dict(M=-1), dict(d=0), dict(h=A[0] + 4),
                dict(x=A[1] + 8), dict(g=A[2] + 2), dict(out=A[3] + 4), dict(out=A[0] + 16), dict(out=A[1]),
                dict(out=A[2]), dict(codes=A[0]), dict(codes=A[3]), dict(scales=A[4]), dict(scales=A[1]),
                dict(out=A[0], x=A[0])):
        assert n(**bad) == EINVAL, bad
    for d in (16, 33, 16416):
        assert n(d=d) == EUNSUPPORTED


def test_gemm_refuses():
    def g(a=A[0], asc=A[1], fmt=0, b=A[2], bsc=A[3], add=None, out=A[4], M=4, N=32, K=128, kind=0):
        return rc("lmgc_op_gemm_mx", a, asc, fmt, b, bsc, add, out, M, N, K, kind, None)

    def t(fmt, tile):
        return rc("lmgc_op_gemm_mx_tile", A[0], A[1], fmt, A[2], A[3], None, A[4], 0, 32, 128, 0, tile, None)
    assert g(M=0) == 0
    assert [t(0, i) for i in (-1, 0, 7, 8)] == [0, 0, 0, EINVAL] and [t(1, i) for i in (6, 7)] == [0, EINVAL]
    for bad in (dict(a=None), dict(asc=None), dict(b=None), dict(bsc=None), dict(out=None), dict(fmt=2), dict(kind=1),
                dict(kind=2), dict(kind=4), dict(M=-1), dict(M=(1 << 26) + 1), dict(N=0), dict(K=0), dict(K=(1 << 20) + 1),
                dict(out=A[0]), dict(out=A[1]), dict(out=A[2]), dict(out=A[3]), dict(a=A[0] + 8), dict(out=A[4] + 4),
                dict(add=A[4] + 16), dict(add=A[4], kind=3), dict(add=A[5] + 4)):
        assert g(**bad) == EINVAL, bad


def _cache_args(**kw):
    a = dict(B=2, Hkv=2, T=3, hd=64, cap=128, lens=A[0], counts=None, kc=A[1], ks=A[2], vc=A[3], vs=A[4])
    a.update(kw)
    return a


CACHE_BAD = [dict(B=0), dict(Hkv=0), dict(T=0), dict(cap=0), dict(cap=100), dict(B=16384), dict(cap=(1 << 24) + 64),
             dict(lens=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(kc=A[1] + 8),
             dict(ks=A[2] + 4), dict(lens=A[0] + 2), dict(counts=A[5] + 1), dict(vc=A[1]), dict(vs=A[2]),
             dict(ks=A[1] + 16), dict(vs=A[3] + 64), dict(ks=A[3])]


def test_append_refuses():
    def ap(k=A[6], v=A[7], **kw):
        a = _cache_args(**kw)
        return rc("lmgc_op_kv8_append", k, v, a["B"], a["Hkv"], a["T"], a["hd"], a["cap"], a["lens"], a["counts"],
                  a["kc"], a["ks"], a["vc"], a["vs"], None)
    for bad in CACHE_BAD + [dict(k=None), dict(v=None), dict(k=A[6] + 8), dict(k=A[1] + 64), dict(v=A[3]), dict(v=A[2]),
                            dict(k=A[4])]:
        assert ap(**bad) == EINVAL, bad
    for hd in (32, 96, 256):
        assert ap(hd=hd) == EUNSUPPORTED


def test_attention_refuses():
    def at(q=A[6], Hq=4, window=0, sinks=0, out=A[7], ws=A[8], nws=1 << 20, **kw):
        a = _cache_args(**kw)
        return rc("lmgc_op_attention_kv8", q, a["B"], Hq, a["Hkv"], a["T"], a["hd"], a["cap"], a["lens"], a["counts"],
                  a["kc"], a["ks"], a["vc"], a["vs"], window, sinks, out, ws, nws, None)
    for bad in CACHE_BAD + [dict(q=None), dict(out=None), dict(Hq=3), dict(Hq=0), dict(window=-1), dict(sinks=-1),
                            dict(out=A[6]), dict(q=A[6] + 8), dict(ws=A[8] + 8), dict(cap=4096, ws=A[6]),
                            dict(cap=4096, ws=A[7]), dict(out=A[1] + 64), dict(out=A[4]), dict(cap=4096, ws=A[3])]:
        assert at(**bad) == EINVAL, bad
    assert at(hd=80) == EUNSUPPORTED
    # over 2^32 threads in one launch (far apart: the buffers of such a call do not overlap)
    far = dict(kc=1 << 50, ks=1 << 51, vc=1 << 52, vs=1 << 53, q=1 << 54, out=1 << 55, cap=1 << 24, T=1 << 24, B=64)
    assert at(**far) == EUNSUPPORTED
    need = rc("lmgc_kv8_workspace", 2, 4, 2, 3, 64, 4096)
    assert need > 0
    assert at(cap=4096, nws=need - 1) == ESIZE and at(cap=4096, ws=None) == ESIZE
    assert b"workspace" in B.lib().lmgc_last_error()


def test_workspace():
    for bad in ((0, 4, 2, 1, 64, 128), (1, 3, 2, 1, 64, 128), (1, 4, 2, 0, 64, 128), (1, 4, 2, 1, 64, 100)):
        assert rc("lmgc_kv8_workspace", *bad) == EINVAL
    assert rc("lmgc_kv8_workspace", 1, 4, 2, 1, 96, 128) == EUNSUPPORTED
    assert rc("lmgc_kv8_workspace", 1, 4, 2, 1, 64, 128) >= 0
    # a long cache is split into 64 parts at most, 16 with many columns
    assert rc("lmgc_kv8_workspace", 1, 4, 2, 1, 64, 1 << 24) == 4 * 64 * 66 * 4
    assert rc("lmgc_kv8_workspace", 1, 4, 2, 512, 64, 1 << 24) == 4 * 512 * 16 * 66 * 4
    assert rc("lmgc_kv8_workspace", 1, 4, 2, 1 << 15, 64, 1 << 24) == 0
    assert ctypes.sizeof(ctypes.c_int64) == 8
