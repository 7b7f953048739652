"""Add and RMSNorm with a microscaled output: the bytes behind a row, and rows at
the ends of float32."""
import numpy as np
import pytest

import lowbit_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("d", [32, 96, 544, 1056, 4128, 8224])
def test_bytes_behind_the_last_block_are_zero(fmt, d):
    """Also of rows that are NaN, hold an infinity, or are zero with eps 0: such
    a row's blocks have the scale byte 255 and codes of zero, the bytes behind
    its last block are zero as in every row."""
    import torch
    log(f"bytes behind {fmt} d={d}")
    h = torch.ones(5, d, device="cuda")
    h[0, 3] = float("nan")
    h[1, d - 1] = float("inf")
    h[2] = 0
    h[3, 0] = -float("inf")
    gain = torch.ones(d, device="cuda")
    nb = d // 32
    behind = [16 * (j // 16) + 4 * (j % 4) + (j % 16) // 4 for j in range(nb, 16 * -(-d // 512))]
    codes, scales = B.op_add_norm_mx(h, None, gain, 0.0, fmt)
    scales = scales.cpu().numpy()
    assert not codes[:, d // (1 if fmt == "fp8" else 2):].any() and not scales[:, behind].any()
    y = B.op_mx_dequantize(codes, torch.from_numpy(scales).cuda(), fmt, d).cpu().numpy()
    assert np.isnan(y[0]).all() and np.isnan(y[2]).all()
    assert np.isnan(y[1, d - 32:]).all() and (y[1, :d - 32] == 0).all()
    assert np.isnan(y[3, :32]).all() and (y[3, 32:] == 0).all()
    assert np.abs(y[4] - 1).max() <= (2.0 ** -4 if fmt == "fp8" else 2.0 ** -2)


def _check(codes, scales, fmt, y):
    """Scales and codes of y, known to 2^-44: those of the float64 value, or of
    one off by that, or (below 2^-126, where float32 has steps of 2^-149) by
    half a step."""
    one = codes if fmt == "fp8" else np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    ok_c = ok_s = False
    for z in (y, y * (1 - 2.0 ** -44), y * (1 + 2.0 ** -44), y - 2.0 ** -150 * (np.abs(y) < 2.0 ** -126), y + 2.0 ** -150 * (np.abs(y) < 2.0 ** -126)):
        rc, rb = R.mx_quantize(z, fmt)
        ok_c = ok_c | (one == rc)
        ok_s = ok_s | (scales == R.rows_layout(rc, rb, fmt, y.shape[1])[1])
    assert ok_s.all() and ok_c.all(), (~ok_s).sum() + (~ok_c).sum()


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("exponent,eps", [(-146, 0.0), (-140, 0.0), (-128, 0.0), (-126, 0.0), (-100, 0.0), (-60, 1e-37), (0, 0.0), (70, 1e-5),
                                          (104, 1e-5), (118, 1e-5), (122, 1e-5), (123, 1e-5)])
def test_rows_at_the_ends_of_float32(fmt, exponent, eps):
    """Rows of 2^exponent: subnormal ones normalised with eps 0, and ones whose
    reciprocal root is subnormal; the codes are the nearest ones as they are for
    ordinary rows.  (float64: the squares, their sum and its root are off by d
    2^-53 at most, which is 2^-43.)"""
    import torch
    log(f"rows of 2^{exponent} {fmt} eps {eps}")
    M, d = 300, 1024
    g = np.random.default_rng(exponent + 200)
    h = np.ldexp(np.clip(g.standard_normal((M, d)), -15, 15), exponent).astype(np.float32)
    gain = (1 + 0.1 * g.standard_normal(d)).astype(np.float32)
    codes, scales = B.op_add_norm_mx(torch.from_numpy(h).cuda(), None, torch.from_numpy(gain).cuda(), eps, fmt)
    v = h.astype(np.float64)
    y = v / np.sqrt((v * v).mean(-1, keepdims=True) + float(np.float32(eps))) * gain.astype(np.float64)
    _check(codes.cpu().numpy(), scales.cpu().numpy(), fmt, y)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_gains_of_any_size(fmt):
    """Gains down to 2^-120 and up to 2^120, and values that are small beside
    their row: the codes of the float64 product."""
    import torch
    M, d = 64, 768
    g = np.random.default_rng(7)
    h = (g.standard_normal((M, d)) * np.exp2(g.integers(-60, 2, (M, d)))).astype(np.float32)
    gain = np.ldexp(1 + 0.1 * g.standard_normal(d), np.repeat(g.integers(-120, 120, d // 32), 32)).astype(np.float32)
    codes, scales = B.op_add_norm_mx(torch.from_numpy(h).cuda(), None, torch.from_numpy(gain).cuda(), 1e-5, fmt)
    v = h.astype(np.float64)
    y = v / np.sqrt((v * v).mean(-1, keepdims=True) + float(np.float32(1e-5))) * gain.astype(np.float64)
    _check(codes.cpu().numpy(), scales.cpu().numpy(), fmt, y)
