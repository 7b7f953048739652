"""Microscaled rows, blocks, the add with RMSNorm and the product against plain
float64 references."""
import numpy as np
import pytest

import lowbit_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _torch(x, dtype="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _host(t):
    import torch
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _values(rows, cols, seed, spread=2.0):
    g = np.random.default_rng(seed)
    return (g.standard_normal((rows, cols)) * np.exp(spread * g.standard_normal((rows, (cols + 31) // 32)).repeat(32, 1)[:, :cols])).astype(np.float32)


# -------------------------------------------------------------- quantisation
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 7), (2, 33), (5, 127), (4, 128), (17, 129), (16, 511), (3, 512),
                                       (2, 520), (7, 1000), (1, 4096), (300, 768), (70000, 40)])
def test_quantize_is_exact(fmt, dtype, rows, cols):
    log(f"quantize {fmt} {dtype} {rows}x{cols}")
    x = _torch(_values(rows, cols, rows + cols), dtype)
    codes, scales = B.op_mx_quantize(x, fmt)
    rc, rb = R.mx_quantize(_host(x), fmt)
    wc, ws = R.rows_layout(rc, rb, fmt, cols)
    assert np.array_equal(codes.cpu().numpy(), wc)
    assert np.array_equal(scales.cpu().numpy(), ws)
    back = B.op_mx_dequantize(codes, scales, fmt, cols)
    assert np.array_equal(_host(back), R.mx_values(rc, rb, fmt, cols).astype(np.float32))
    half = B.op_mx_dequantize(codes, scales, fmt, cols, dtype=__import__("torch").bfloat16)
    assert np.array_equal(_host(half), _host(back.to(half.dtype)))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_quantize_special_values(fmt):
    """Zeros of both signs, subnormals, ties, the largest numbers, amax at and
    around a scale's border; NaN and infinities mark their own block alone."""
    top = R.TOP[fmt]
    grid = R.POSITIVE[fmt]
    ties = (grid[:-1] + grid[1:]) / 2
    rows = [np.concatenate([[top], ties, -ties])[:256], np.concatenate([grid, -grid])[:256], np.full(64, -0.0), np.full(64, 1e-45),
            np.full(64, 3.4e38), [top * 2.0 ** -127, 1e-39, -1e-40], np.nextafter(np.float32(top), np.float32(1e9)) * np.ones(3),
            np.nextafter(np.float32(top), np.float32(0)) * np.ones(3), [np.inf] + [1.0] * 40, [1.0] * 33 + [np.nan], [-np.inf, np.nan],
            np.linspace(-1, 1, 96) * 2.0 ** -130]
    x = np.zeros((len(rows), 256), np.float32)
    for i, r in enumerate(rows):
        x[i, :len(r)] = np.asarray(r, np.float32)
    codes, scales = B.op_mx_quantize(_torch(x), fmt)
    rc, rb = R.mx_quantize(x, fmt)
    wc, ws = R.rows_layout(rc, rb, fmt, 256)
    got_c, got_s = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(got_s, ws)
    assert np.array_equal(got_c, wc)
    back = _host(B.op_mx_dequantize(codes, scales, fmt, 256))
    assert np.array_equal(back, R.mx_values(rc, rb, fmt, 256).astype(np.float32), equal_nan=True)
    assert np.isnan(back[8, :32]).all() and not np.isnan(back[8, 32:]).any() and not np.isnan(back[9, :32]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_strided_rows(dtype):
    """Rows of a wider matrix, at a column offset that leaves them unaligned."""
    import torch
    wide = _torch(_values(9, 400, 5), dtype)
    for off, cols in ((0, 256), (1, 200), (3, 129), (8, 64)):
        x = wide[:, off:off + cols]
        codes, scales = B.op_mx_quantize(x, "fp8")
        c2, s2 = B.op_mx_quantize(x.contiguous(), "fp8")
        assert torch.equal(codes, c2) and torch.equal(scales, s2)
        out = torch.full((9, 400), 7.0, device="cuda")
        B.op_mx_dequantize(codes, scales, "fp8", cols, out=out[:, off:off + cols])
        assert torch.equal(out[:, off:off + cols], B.op_mx_dequantize(codes, scales, "fp8", cols))
        assert (out[:, :off] == 7).all() and (out[:, off + cols:] == 7).all()


@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 130), (40, 700), (48, 1152)])
def test_block_layout(N, K):
    rc, rb = R.mx_quantize(_values(N, K, 3), "fp4")
    codes, scales = R.rows_layout(rc, rb, "fp4", K)
    import torch
    bc, bs = B.op_mx_block(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K)
    wc, ws = R.blocks_layout(rc, rb, K)
    assert np.array_equal(bc.cpu().numpy(), wc) and np.array_equal(bs.cpu().numpy(), ws)


# ----------------------------------------------------------- add and RMSNorm
def _check_norm(codes, scales, fmt, y, delta=2.0 ** -18):
    """Codes and scales of y known to `delta` (2^-18 would do for a float32 sum
    of d squares of at most 64 terms a lane, its root and three products: under
    43 2^-24): the scale is y's, or the neighbour's where amax lies that close
    to its border; the values are within half a step of y, and that."""
    d = y.shape[1]
    nb = R.up(d, 128) // 32
    byte = np.stack([scales[:, 16 * (j // 16) + 4 * (j % 4) + (j % 16) // 4] for j in range(nb)], 1)
    z = np.zeros((y.shape[0], nb * 32))
    z[:, :d] = y
    amax = np.abs(z.reshape(y.shape[0], nb, 32)).max(-1)
    lo = R.power_at_least(amax * (1 - delta) / R.TOP[fmt], -127) + 127
    hi = R.power_at_least(amax * (1 + delta) / R.TOP[fmt], -127) + 127
    assert ((byte == lo) | (byte == hi)).all()
    one = codes if fmt == "fp8" else np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    got = R.mx_values(one, byte, fmt, nb * 32)
    assert (got[:, d:] == 0).all()
    s = np.ldexp(1.0, byte.astype(int) - 127).repeat(32, 1)
    rel, low = (2.0 ** -4, 2.0 ** -6) if fmt == "fp8" else (2.0 ** -2, 1.0)
    assert (np.abs(got - z) <= rel * np.maximum(np.abs(z) * (1 + delta), low * s) + delta * np.abs(z)).all()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("h,x,g", [("f32", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("bf16", None, "bf16")])
@pytest.mark.parametrize("M,d", [(1, 32), (2, 64), (3, 160), (5, 768), (17, 2048), (9, 4096), (4, 8192), (2, 16384)])
def test_add_norm(fmt, h, x, g, M, d):
    import torch
    log(f"add_norm {fmt} {h} {x} {g} {M}x{d}")
    r = np.random.default_rng(M * d)
    th = _torch(r.standard_normal((M, d)) * 3, h)
    tx = None if x is None else _torch(r.standard_normal((M, d)), x)
    tg = _torch(1 + 0.1 * r.standard_normal(d), g)
    out = torch.empty_like(th)
    codes, scales = B.op_add_norm_mx(th, tx, tg, 1e-5, fmt, out=out)
    t = th if tx is None else (th.float() + tx.float()).to(th.dtype)
    assert torch.equal(out, t)
    v = _host(t).astype(np.float64)
    y = v / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-5) * _host(tg).astype(np.float64)
    _check_norm(codes.cpu().numpy(), scales.cpu().numpy(), fmt, y)
    # in place, and without storing the sum: the same codes
    again = th.clone()
    c2, s2 = B.op_add_norm_mx(again, tx, tg, 1e-5, fmt, out=again)
    c3, s3 = B.op_add_norm_mx(th, tx, tg, 1e-5, fmt)
    assert torch.equal(again, t) and torch.equal(c2, codes) and torch.equal(s2, scales)
    assert torch.equal(c3, codes) and torch.equal(s3, scales)
    # a row alone gives the row's bits
    c1, s1 = B.op_add_norm_mx(th[M - 1:], None if tx is None else tx[M - 1:], tg, 1e-5, fmt)
    assert torch.equal(c1[0], codes[M - 1]) and torch.equal(s1[0], scales[M - 1])


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("h,M,d", [("bf16", 1500, 4096), ("f32", 4003, 768), ("f32", 2001, 1024), ("bf16", 999, 1056)])
def test_add_norm_next_to_a_border(fmt, h, M, d):
    """Some values of millions lie within a float32's rounding of the border
    between two codes; theirs are the nearer codes all the same.  The kernel's y
    before its last step is off by the float32 corrections' own rounding: of
    the root's (2^-48), of the two products' (2^-48 each) and of their sums
    (2 2^-48), under 2^-45, and that step keeps the side of the border."""
    import torch
    log(f"add_norm border {fmt} {h} {M}x{d}")
    r = np.random.default_rng(d)
    th = _torch(r.standard_normal((M, d)) * 3, h)
    tg = _torch(1 + 0.1 * r.standard_normal(d), "f32")
    codes, scales = B.op_add_norm_mx(th, None, tg, 1e-5, fmt)
    v = _host(th).astype(np.float64)
    y = v / np.sqrt((v * v).mean(-1, keepdims=True) + float(np.float32(1e-5))) * _host(tg).astype(np.float64)
    _check_norm(codes.cpu().numpy(), scales.cpu().numpy(), fmt, y, 2.0 ** -44)


def test_add_norm_nonfinite_and_zero_rows():
    import torch
    h = torch.ones(4, 64, device="cuda")
    h[0, 3] = float("nan")
    h[1, 5] = float("inf")
    h[2] = 0
    g = torch.ones(64, device="cuda")
    codes, scales = B.op_add_norm_mx(h, None, g, 1e-5, "fp8")
    y = B.op_mx_dequantize(codes, scales, "fp8", 64).cpu().numpy()
    assert np.isnan(y[0]).all() and np.isnan(y[1, :32]).all()  # inf * 0 in its block
    assert (y[2] == 0).all() and np.allclose(y[3], 1, atol=2.0 ** -4)


# ------------------------------------------------------------------- product
def _operand(rows, cols, fmt, seed):
    rc, rb = R.mx_quantize(_values(rows, cols, seed, 0.5), fmt)
    return rc, rb, R.mx_values(rc, rb, fmt, cols)


def _device(rc, rb, fmt, cols):
    import torch
    c, s = R.rows_layout(rc, rb, fmt, cols)
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


def _product_tol(a, b, fmt, kind, ref, add):
    """Float32 accumulation: a step (128 columns) adds its products and the sum
    so far with an error of at most 2^-23 of their magnitudes, over ceil(K /
    128) steps.  With e4m3 operands the instruction also drops what lies 2^-18
    and more below the largest product of a step, from each of its 128
    products.  Then the add's rounding and bf16's."""
    K = a.shape[1]
    nk = -(-K // 128)
    mag = np.abs(a) @ np.abs(b).T
    tol = (nk + 1) * 2.0 ** -23 * mag
    if fmt == "fp8":
        for k in range(nk):
            pa, pb = np.abs(a[:, 128 * k:128 * k + 128]).max(1), np.abs(b[:, 128 * k:128 * k + 128]).max(1)
            tol += 128 * 2.0 ** -18 * np.outer(pa, pb)
    tol += 2.0 ** -24 * np.abs(ref)
    if kind == "bf16":
        tol += 2.0 ** -8 * (np.abs(ref) + tol)
    return tol


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(1, 16, 32), (1, 256, 4096), (2, 17, 128), (5, 33, 129), (8, 300, 1000), (16, 64, 512), (31, 48, 640),
                                   (33, 129, 257), (64, 128, 384), (100, 250, 1100), (128, 256, 2048), (257, 513, 900), (300, 520, 5632)])
def test_product(fmt, M, N, K):
    import torch
    log(f"gemm_mx {fmt} {M}x{N}x{K}")
    ac, ab, a = _operand(M, K, fmt, 1)
    bc, bb, b = _operand(N, K, "fp4", 2)
    da, dsa = _device(ac, ab, fmt, K)
    db, dsb = B.op_mx_block(*_device(bc, bb, "fp4", K), K)
    add = np.random.default_rng(3).standard_normal((M, N)).astype(np.float32)
    tadd = torch.from_numpy(add).cuda()
    ref = a @ b.T
    for kind in ("store", "bf16"):
        for ta, r in ((None, ref), (tadd, ref + add)):
            out = B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, kind, add=ta)
            err = np.abs(_host(out).astype(np.float64) - r)
            assert (err <= _product_tol(a, b, fmt, kind, r, ta)).all(), (kind, ta is not None, err.max())
    inplace = tadd.clone()
    B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, "store", add=inplace, out=inplace)
    assert torch.equal(inplace, B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, "store", add=tadd))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("tile", B.MX_TILES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (3, 50, 129), (40, 264, 385), (300, 130, 640), (517, 777, 897), (260, 600, 2200)])
def test_product_tiles(fmt, tile, M, N, K):
    """Every tile, with odd numbers of steps and of pieces past the ends: within
    the bound, and bit for bit the tile that the library takes."""
    import torch
    log(f"gemm_mx {fmt} tile {tile} {M}x{N}x{K}")
    ac, ab, a = _operand(M, K, fmt, 1)
    bc, bb, b = _operand(N, K, "fp4", 2)
    da, dsa = _device(ac, ab, fmt, K)
    db, dsb = B.op_mx_block(*_device(bc, bb, "fp4", K), K)
    if fmt == "fp4" and tile == "256x256":
        with pytest.raises(B.LMGCError):
            B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, tile=tile)
        return
    out = B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, tile=tile)
    ref = a @ b.T
    err = np.abs(_host(out).astype(np.float64) - ref)
    assert (err <= _product_tol(a, b, fmt, "store", ref, None)).all(), err.max()
    assert torch.equal(out, B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K))
    add = torch.randn(M, N, device="cuda")
    for kind, dt in (("store", torch.float32), ("bf16", torch.bfloat16)):
        room = torch.full((M * N + 512,), 7.0, dtype=dt, device="cuda")
        got = B.op_gemm_mx(da, dsa, fmt, db, dsb, N, K, kind, add=add, out=room[256:256 + M * N].view(M, N), tile=tile)
        assert torch.equal(got, (out + add).to(dt))
        assert (room[:256] == 7).all() and (room[256 + M * N:] == 7).all()


@pytest.mark.parametrize("fmt,M,N,K", [("fp8", 2000, 2050, 900), ("fp8", 4100, 4100, 1200), ("fp8", 9000, 4600, 700),
                                       ("fp8", 600000, 24, 130), ("fp4", 1030, 2050, 1200), ("fp4", 4100, 4100, 600), ("fp4", 20, 13001, 700)])
def test_product_large(fmt, M, N, K):
    """Sizes at which the library takes its large tiles, against float64 on the
    device; the bound is _product_tol's, with the largest products of all steps
    in the place of each step's."""
    import torch
    log(f"gemm_mx {fmt} {M}x{N}x{K}")
    g = torch.Generator(device="cuda").manual_seed(M)
    a, sa = B.op_mx_quantize(torch.randn(M, K, generator=g, device="cuda"), fmt)
    w, sw = B.op_mx_quantize(0.02 * torch.randn(N, K, generator=g, device="cuda"), "fp4")
    b, sb = B.op_mx_block(w, sw, K)
    va, vb = B.op_mx_dequantize(a, sa, fmt, K).double(), B.op_mx_dequantize(w, sw, "fp4", K).double()
    out = B.op_gemm_mx(a, sa, fmt, b, sb, N, K)
    nk = -(-K // 128)
    tol = (nk + 1) * 2.0 ** -23 * (va.abs() @ vb.abs().T)
    if fmt == "fp8":
        tol += nk * 128 * 2.0 ** -18 * torch.outer(va.abs().amax(1), vb.abs().amax(1))
    assert ((out.double() - va @ vb.T).abs() <= tol).all()


def test_norm_and_product_in_graphs():
    """Add + norm, product and quantisation captured once and replayed over new
    inputs, with eager work between; two graphs, one after the other, on the
    same buffers."""
    import torch
    M, d, N = 37, 768, 640
    g = torch.Generator(device="cuda").manual_seed(3)
    h, x, gain = (torch.zeros(M, d, device="cuda"), torch.zeros(M, d, dtype=torch.bfloat16, device="cuda"),
                  torch.ones(d, device="cuda"))
    b, sb = B.op_mx_block(*B.op_mx_quantize(0.02 * torch.randn(N, d, generator=g, device="cuda"), "fp4"), d)
    codes, scales = B.op_mx_quantize(h, "fp8")
    y, yc, ys = torch.empty(M, N, device="cuda"), *B.op_mx_quantize(torch.zeros(M, N, device="cuda"), "fp4")

    def step(h, x, y, codes, scales, yc, ys):
        B.op_add_norm_mx(h, x, gain, 1e-5, "fp8", out=h, codes=codes, scales=scales)
        B.op_gemm_mx(codes, scales, "fp8", b, sb, N, d, out=y)
        B.op_mx_quantize(y, "fp4", codes=yc, scales=ys)

    bufs = (h, x, y, codes, scales, yc, ys)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*bufs)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*bufs)
        graphs.append(graph)
    for i in range(6):
        nh, nx = torch.randn(M, d, generator=g, device="cuda"), torch.randn(M, d, generator=g, device="cuda").to(torch.bfloat16)
        h.copy_(nh), x.copy_(nx)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        mine = (nh, nx) + tuple(t.clone().zero_() for t in bufs[2:])
        step(*mine)
        assert all(torch.equal(p, q) for p, q in zip(bufs, mine)), i


def test_calls_on_a_stream():
    """Results and workspaces that the call allocates belong to its stream: long
    work on the current stream does not touch them."""
    import torch
    x = torch.randn(300, 768, device="cuda")
    h, g = torch.randn(300, 768, device="cuda"), torch.ones(768, device="cuda")
    want = B.op_mx_quantize(x, "fp4")
    b, sb = B.op_mx_block(*want, 768)
    norm = B.op_add_norm_mx(h, x, g, 1e-5, "fp8")
    prod = B.op_gemm_mx(*norm, "fp8", b, sb, 300, 768)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        junk = [torch.full((300, 768), 3.0, device="cuda") for _ in range(20)]
        del junk  # their memory is the current stream's to give out
        c, sc = B.op_mx_quantize(x, "fp4", stream=s)
        bb, sbb = B.op_mx_block(c, sc, 768, stream=s)
        n, ns = B.op_add_norm_mx(h, x, g, 1e-5, "fp8", stream=s)
        p = B.op_gemm_mx(n, ns, "fp8", bb, sbb, 300, 768, stream=s)
        y = B.op_mx_dequantize(c, sc, "fp4", 768, stream=s)
        s.synchronize()
        assert torch.equal(c, want[0]) and torch.equal(sc, want[1]) and torch.equal(bb, b) and torch.equal(sbb, sb)
        assert torch.equal(n, norm[0]) and torch.equal(ns, norm[1]) and torch.equal(p, prod)
        assert torch.equal(y, B.op_mx_dequantize(*want, "fp4", 768))


def test_tensors_on_another_device_are_refused():
    import torch
    h, g = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    codes, scales = B.op_mx_quantize(h, "fp4")
    b, sb = B.op_mx_block(codes, scales, 64)
    for call in (lambda: B.op_mx_quantize(h.cpu(), "fp8"), lambda: B.op_mx_dequantize(codes, scales.cpu(), "fp4", 64),
                 lambda: B.op_mx_block(codes.cpu(), scales, 64), lambda: B.op_add_norm_mx(h, h.cpu(), g, 1e-5, "fp8"),
                 lambda: B.op_add_norm_mx(h, None, g.cpu(), 1e-5, "fp8"),
                 lambda: B.op_gemm_mx(codes, scales, "fp4", b.cpu(), sb, 4, 64),
                 lambda: B.op_gemm_mx(codes, scales, "fp4", b, sb, 4, 64, add=torch.zeros(4, 4))):
        with pytest.raises(ValueError):
            call()


def test_rows_past_32_bits():
    """Rows 2^31 elements apart, and more rows than one launch takes."""
    import torch
    ld = (1 << 31) + 64
    big = torch.empty(ld + 96, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((2, 96), (ld, 1))
    x.copy_(torch.randn(2, 96, device="cuda"))
    codes, scales = B.op_mx_quantize(x, "fp8")
    c2, s2 = B.op_mx_quantize(x.contiguous(), "fp8")
    assert torch.equal(codes, c2) and torch.equal(scales, s2)
    back = B.op_mx_dequantize(codes, scales, "fp8", 96, dtype=torch.bfloat16)
    B.op_mx_dequantize(codes, scales, "fp8", 96, out=x)
    assert torch.equal(x, back)
    del big, x
    M, d = (1 << 23) + 5, 32
    h = torch.randn(M, d, device="cuda").to(torch.bfloat16)
    g = torch.ones(d, device="cuda")
    codes, scales = B.op_add_norm_mx(h, None, g, 1e-5, "fp4")
    for lo, hi in ((0, 9), ((1 << 23) - 4, M)):
        c2, s2 = B.op_add_norm_mx(h[lo:hi].contiguous(), None, g, 1e-5, "fp4")
        assert torch.equal(codes[lo:hi], c2) and torch.equal(scales[lo:hi], s2)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("N,K", [(272, 1184), (2048, 640)])
def test_product_rows_do_not_depend_on_m(fmt, N, K):
    """A row's bits are the same alone, in a step's batch and in a prompt."""
    import torch
    M = 700
    g = torch.Generator(device="cuda").manual_seed(4)
    a, sa = B.op_mx_quantize(torch.randn(M, K, generator=g, device="cuda"), fmt)
    b, sb = B.op_mx_block(*B.op_mx_quantize(0.02 * torch.randn(N, K, generator=g, device="cuda"), "fp4"), K)
    whole = B.op_gemm_mx(a, sa, fmt, b, sb, N, K)
    for lo, hi in ((0, 1), (3, 5), (10, 26), (1, 33), (100, 164), (7, 135), (200, 500), (699, 700)):
        part = B.op_gemm_mx(a[lo:hi].clone(), sa[lo:hi].clone(), fmt, b, sb, N, K)
        assert torch.equal(part, whole[lo:hi]), (lo, hi)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_product_nan_blocks_stay_in_their_row_and_column(M):
    import torch
    N, K = 96, 384
    x, w = torch.randn(M, K, device="cuda"), torch.randn(N, K, device="cuda")
    x[1, 200] = float("nan")
    w[5, 300] = float("inf")
    a, sa = B.op_mx_quantize(x, "fp8")
    b, sb = B.op_mx_block(*B.op_mx_quantize(w, "fp4"), K)
    out = B.op_gemm_mx(a, sa, "fp8", b, sb, N, K).cpu().numpy()
    bad = np.zeros((M, N), bool)
    bad[1], bad[:, 5] = True, True
    assert np.array_equal(np.isnan(out), bad)


def test_product_writes_only_its_output():
    """Rows behind the last and memory around the output keep what they held."""
    import torch
    for M, N in ((1, 48), (5, 40), (37, 130), (130, 200), (260, 300)):
        K = 256
        a, sa = B.op_mx_quantize(torch.randn(M, K, device="cuda"), "fp4")
        b, sb = B.op_mx_block(*B.op_mx_quantize(torch.randn(N, K, device="cuda"), "fp4"), K)
        for kind, dt in (("store", torch.float32), ("bf16", torch.bfloat16)):
            room = torch.full((M * N + 512,), 7.0, dtype=dt, device="cuda")
            out = room[256:256 + M * N].view(M, N)
            B.op_gemm_mx(a, sa, "fp4", b, sb, N, K, kind, out=out)
            assert (room[:256] == 7).all() and (room[256 + M * N:] == 7).all()
            assert torch.equal(out, B.op_gemm_mx(a, sa, "fp4", b, sb, N, K, kind))
