"""The rotary table and the rotation of rows against plain float64 references."""
import numpy as np
import pytest

import paged_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _table(n_pos, rot, seed=None):
    """A table on the GPU and its numbers; seeded: any numbers, not of length one."""
    if seed is None:
        t = B.rope_table(n_pos, rot)
    else:
        t = _torch().from_numpy(np.random.default_rng(seed).standard_normal((n_pos, rot // 2, 2)).astype(np.float32)).cuda()
    return t, t.cpu().numpy().astype(np.float64)


# --------------------------------------------------------------------- table
@pytest.mark.parametrize("n_pos,rot,theta,scaling,kw", [
    (1, 2, 1e4, "none", {}), (7, 6, 1e4, "none", {}), (300, 128, 1e4, "none", {}), (131073, 64, 5e5, "none", {}),
    (5000, 96, 1e4, "linear", dict(factor=4.0)), (70000, 128, 1e4, "ntk", dict(factor=16.0)),
    (70000, 128, 1e4, "yarn", dict(factor=16.0, orig=4096)), (100, 512, 1e4, "yarn", dict(factor=2.0, orig=64, mscale=1.5))])
def test_table(n_pos, rot, theta, scaling, kw):
    log(f"table {n_pos} {rot} {scaling}")
    got = B.rope_table(n_pos, rot, theta, scaling, **kw).cpu().numpy().astype(np.float64)
    mscale = kw.pop("mscale", 0.1 * np.log(kw["factor"]) + 1.0 if scaling == "yarn" else 1.0)
    f = B.rope_frequencies(rot, theta, scaling, **kw)
    a = np.arange(n_pos)[:, None] * f[None, :]
    want = mscale * np.stack([np.cos(a), np.sin(a)], -1)
    # one rounding to float32; the angles' product is off by 2^-53 of 2^17 at most, as is the reference's
    assert (abs(got - want) <= 2.0 ** -24 * abs(want) + 2.0 ** -34 * mscale).all()


def test_table_into_a_buffer_on_a_stream():
    torch = _torch()
    s = torch.cuda.Stream()
    out = torch.full((64, 32, 2), 7.0, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    assert B.rope_table(64, 64, out=out, stream=s) is out
    s.synchronize()
    assert torch.equal(out, B.rope_table(64, 64))
    other = B.rope_table(64, 64, stream=s)
    s.synchronize()
    assert torch.equal(out, other)


# ------------------------------------------------------------------ rotation
def _check(x, pos, table, tab, layout, backward, out):
    torch = _torch()
    ok = (pos >= 0) & (pos < tab.shape[0])
    want, mag = R.rotate(x.double().cpu().numpy(), tab[np.clip(pos, 0, tab.shape[0] - 1)][:, None], layout, backward)
    # two products and a sum, each off by half a step at most; then one rounding to bf16
    tol = 2.0 ** -23 * mag + (2.0 ** -8 * abs(want) * (1 + 2.0 ** -8) if out.dtype == torch.bfloat16 else 0.0) + 1e-38
    tol[..., 2 * tab.shape[1]:] = 0
    got = out.double().cpu().numpy()
    assert (abs(got - want) <= tol)[ok].all(), abs(got - want)[ok].max()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n,heads,hd,rot", [(1, 1, 2, 2), (3, 5, 64, 64), (33, 2, 128, 128), (17, 3, 128, 32), (70, 1, 80, 80), (9, 4, 96, 16),
                                            (5, 2, 64, 10), (11, 3, 33, 6), (300, 36, 64, 64), (2, 2, 512, 512), (4, 1, 256, 100), (1030, 7, 128, 128)])
def test_rope(n, heads, hd, rot, layout, dtype):
    log(f"rope {n} {heads} {hd} {rot} {layout} {dtype}")
    torch = _torch()
    g = np.random.default_rng(n + hd)
    x = torch.from_numpy(g.standard_normal((n, heads, hd)).astype(np.float32)).cuda().to(getattr(torch, dtype))
    table, tab = _table(200, rot, n)
    pos = g.integers(0, 200, n)
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    keep = x.clone()
    for backward in (False, True):
        out = B.op_rope(x, p, table, layout, backward)
        _check(x, pos, table, tab, layout, backward, out)
        assert torch.equal(x, keep)
        place = x.clone()
        assert B.op_rope(place, p, table, layout, backward, out=place) is place
        assert torch.equal(place, out)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gap,shift", [(0, 0), (64, 0), (6, 0), (3, 1), (64, 1)])
def test_rope_inside_wider_rows(gap, shift, dtype):
    """Strided rows of any alignment; what lies between them stays."""
    torch = _torch()
    n, heads, hd = 37, 3, 64
    wide = torch.randn(n, heads * hd + gap + 8, device="cuda").to(getattr(torch, dtype))
    into = torch.full_like(wide, 5.0)
    x = wide[:, shift:shift + heads * hd].unflatten(1, (heads, hd))
    out = into[:, shift:shift + heads * hd].unflatten(1, (heads, hd))
    table, tab = _table(40, hd, 3)
    pos = np.arange(n) + 2
    B.op_rope(x, torch.from_numpy(pos.astype(np.int32)).cuda(), table, "half", out=out)
    _check(x, pos, table, tab, "half", False, out)
    assert (into[:, :shift] == 5).all() and (into[:, shift + heads * hd:] == 5).all()


def test_rope_of_heads_that_lie_apart():
    """The attention kernels' order [B, H, T, hd], every window at the same positions."""
    torch = _torch()
    Bn, H, T, hd = 2, 3, 50, 128
    q = torch.randn(Bn, H, T, hd, device="cuda").to(torch.bfloat16)
    x = q.view(Bn * H, T, hd).transpose(0, 1)
    table, tab = _table(64, hd)
    pos = np.arange(T) + 5
    out = torch.empty_like(q)
    B.op_rope(x, torch.from_numpy(pos.astype(np.int32)).cuda(), table, "half", out=out.view(Bn * H, T, hd).transpose(0, 1))
    _check(x, pos, table, tab, "half", False, out.view(Bn * H, T, hd).transpose(0, 1))


@pytest.mark.parametrize("rot", [64, 10])
def test_rope_leaves_rows_outside_the_table(rot):
    torch = _torch()
    x = torch.randn(6, 2, 64, device="cuda")
    table, tab = _table(16, rot, 1)
    pos = np.array([0, -1, 15, 16, 2 ** 31 - 1, -2 ** 31])
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    out = torch.full_like(x, 9.0)
    B.op_rope(x, p, table, "interleaved", out=out)
    _check(x, pos, table, tab, "interleaved", False, out)
    assert (out[[1, 3, 4, 5]] == 9).all()
    place = x.clone()
    B.op_rope(place, p, table, "interleaved", out=place)
    assert torch.equal(place[[1, 3, 4, 5]], x[[1, 3, 4, 5]])


def test_rope_special_values():
    """NaN and infinities stay in their pairs, and come through unrotated dims as they are."""
    torch = _torch()
    x = torch.ones(1, 1, 64, device="cuda").to(torch.bfloat16)
    x[0, 0, 3], x[0, 0, 40] = float("nan"), float("-inf")
    table = torch.full((4, 16, 2), 0.5, device="cuda")
    out = B.op_rope(x, torch.ones(1, dtype=torch.int32, device="cuda"), table, "half")[0, 0]
    assert torch.isnan(out[[3, 19]]).all() and out[40] == float("-inf")
    assert torch.isfinite(out[[i for i in range(64) if i not in (3, 19, 40)]]).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_backward_is_the_gradient(layout):
    """Against differences of the forward (linear, so one step of one is exact up to
    rounding), and the rotation undone where the table's pairs have length one."""
    torch = _torch()
    n, H, hd, rot = 5, 2, 64, 48
    table, _ = _table(32, rot, 8)
    p = torch.tensor([0, 3, 31, 7, 7], dtype=torch.int32, device="cuda")
    g = torch.randn(n, H, hd, device="cuda")
    zero = torch.zeros(n, H, hd, device="cuda")
    grad = B.op_rope(g, p, table, layout, backward=True).double()
    for d in list(range(0, hd, 5)) + [hd - 1]:
        e = zero.clone()
        e[..., d] = 1.0
        want = (B.op_rope(e, p, table, layout).double() * g.double()).sum(-1)  # two products of float32 numbers
        # each product and the sum off by 2^-24: table entries and gradients of up to 5
        assert (abs(grad[..., d] - want) <= 2.0 ** -22 * 25).all()
    table, _ = _table(32, rot)
    back = B.op_rope(B.op_rope(g, p, table, layout), p, table, layout, backward=True)
    # c^2 + s^2 = 1 within 2^-23, and two roundings of each of two terms
    assert (abs(back - g) <= 2.0 ** -21 * abs(g).max()).all()


def test_rope_past_32_bits():
    """Rows whose offset passes 2^32 bytes and 2^31 numbers."""
    torch = _torch()
    n, H, hd = 70000, 256, 128  # 2.3e9 numbers
    x = torch.empty(n, H, hd, dtype=torch.bfloat16, device="cuda")
    x[:4], x[-4:] = 1.0, 2.0
    table, tab = _table(8, hd, 4)
    pos = np.full(n, -1)
    pos[:4], pos[-4:] = [0, 1, 2, 3], [4, 5, 6, 7]
    out = B.op_rope(x, torch.from_numpy(pos.astype(np.int32)).cuda(), table)
    for i in (slice(0, 4), slice(n - 4, n)):
        _check(x[i], pos[i], table, tab, "half", False, out[i])


def test_rope_in_a_graph_and_on_a_stream():
    torch = _torch()
    x = torch.randn(100, 4, 64, device="cuda")
    table, _ = _table(128, 64)
    p = torch.arange(100, dtype=torch.int32, device="cuda")
    out, want = torch.empty_like(x), []
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.op_rope(x, p, table, out=out, stream=s)
    with torch.cuda.stream(s):
        want.append(out.clone())
    s.synchronize()
    assert torch.equal(want[0], B.op_rope(x, p, table))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.op_rope(x, p, table, out=out)
    for i in range(3):
        x.normal_()
        p.copy_((p + 3) % 128)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.op_rope(x, p, table))
