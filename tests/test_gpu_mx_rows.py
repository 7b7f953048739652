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
