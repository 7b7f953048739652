"""The paged key/value cache and attention over it, with and without a prefix in
common, against plain float64 references."""
import numpy as np
import pytest

import paged_ref as R
from gpu_util import log
from paper_2409_17836_amd import binding as B

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _ints(v):
    torch = _torch()
    return torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device="cuda")


def _np(t):
    return t.double().cpu().numpy()


class Setup:
    """A batch of (new tokens, tokens before) over a pool of shuffled pages, whose every
    place holds something."""

    def __init__(self, seqs, page=64, Hkv=2, hd=64, seed=0, pad=0, shared=0, spare=2, extra_pages=0, stale=None):
        torch = _torch()
        g = np.random.default_rng(seed)
        self.seqs, self.page, self.Hkv, self.hd = seqs, page, Hkv, hd
        starts = np.concatenate([[0], np.cumsum([t for t, _ in seqs])])
        self.n = int(starts[-1]) + pad
        most = max(-(-(t + n) // page) for t, n in seqs) + extra_pages
        lead = shared // page
        n_pages = lead + sum(most - lead for _ in seqs) + spare
        order = g.permutation(n_pages)
        pages = np.array([np.concatenate([order[:lead], order[lead + i * (most - lead):lead + (i + 1) * (most - lead)]]) for i in range(len(seqs))])
        self.n_pages = n_pages
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed + 1)
        self.cache = tuple(torch.randn(n_pages, Hkv, page, hd, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
        self.gen = gen
        self.set(pages, starts, [n for _, n in seqs])
        if stale is not None:  # what lies behind the tokens and on pages of no sequence
            t = np.arange(page)
            for i, pool in enumerate(self.cache):
                plain = R.in_pool(np.arange(pool.numel()).reshape(pool.shape), bool(i))  # where each number is
                hold = np.zeros((n_pages, page), bool)
                for b, (T, n) in enumerate(seqs):
                    for k in range(-(-(T + n) // page)):
                        hold[pages[b, k]] |= t + k * page < T + n
                at = plain.transpose(0, 2, 1, 3)[~hold].reshape(-1)
                pool.view(-1)[torch.from_numpy(at).cuda()] = stale

    def set(self, pages, starts, lens):
        self.pages_h, self.starts_h, self.lens_h = np.asarray(pages), np.asarray(starts), np.asarray(lens)
        self.pages, self.starts, self.lens = _ints(pages), _ints(starts), _ints(lens)
        self.batch = R.Batch(self.pages_h, self.starts_h, self.lens_h, self.n, self.n_pages, self.page)
        return self

    def rows(self, heads, dtype="bfloat16"):
        torch = _torch()
        return torch.randn(self.n, heads, self.hd, device="cuda", generator=self.gen).to(getattr(torch, dtype))

    def plain(self):
        return [R.in_pool(_np(x), bool(i)) for i, x in enumerate(self.cache)]

    @property
    def max_new(self):
        return max(t for t, _ in self.seqs)


# -------------------------------------------------------------------- append
def _append_check(s, k, v, q, table, layout, rot):
    torch = _torch()
    before = [x.clone() for x in s.cache]
    q_out = torch.full((s.n, q.shape[1], s.hd), 3.0, dtype=torch.bfloat16, device="cuda") if q is not None else None
    B.op_paged_append(s.cache, k, v, s.pages, s.starts, s.lens, rope=table, layout=layout, q=q, q_out=q_out)
    want = [R.in_pool(_np(x), bool(i)) for i, x in enumerate(before)]
    tol = [np.zeros_like(x) for x in want]
    tab = _np(table) if table is not None else None
    wq, tq = np.full((s.n, q.shape[1], s.hd), 3.0) if q is not None else None, None
    tq = np.zeros_like(wq) if q is not None else None
    kn, vn, qn = _np(k), _np(v), _np(q) if q is not None else None

    def turned(x, pos):
        if tab is None:
            return x, 2.0 ** -8 * abs(x)
        y, mag = R.rotate(x, tab[pos][None], layout)
        return y, 2.0 ** -23 * mag + 2.0 ** -8 * abs(y) * (1 + 2.0 ** -8)  # float32, then one rounding to bf16
    for b, row, pos in s.batch.rows():
        if tab is not None and pos >= tab.shape[0]:
            continue
        page = s.pages_h[b, pos // s.page]
        ky, kt = turned(kn[row], pos)
        if 0 <= page < s.n_pages:
            want[0][page, :, pos % s.page], tol[0][page, :, pos % s.page] = ky, kt
            want[1][page, :, pos % s.page], tol[1][page, :, pos % s.page] = vn[row], 2.0 ** -8 * abs(vn[row])
        if q is not None:
            wq[row], tq[row] = turned(qn[row], pos)
    for got, w, t, name in zip(s.plain(), want, tol, ("keys", "values")):
        assert (abs(got - w) <= t).all(), name
    if q is not None:
        assert (abs(_np(q_out) - wq) <= tq).all()
    return q_out


BATCHES = [
    [(1, 0)], [(1, 31)], [(1, 32), (1, 63)], [(5, 0), (1, 200), (70, 30), (3, 61)], [(64, 64)], [(33, 31)], [(130, 1), (1, 130)],
    [(1, i) for i in range(0, 140, 7)], [(0, 5), (2, 0), (0, 0), (31, 1)], [(300, 17)]]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("hd,page,layout,rot", [(64, 32, "half", 64), (64, 64, "interleaved", 32), (128, 128, "half", 128), (128, 32, "interleaved", 128),
                                                (128, 64, "half", 16), (64, 256, "half", 10), (128, 64, "interleaved", 50), (64, 64, "none", 0)])
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_append(batch, hd, page, layout, rot, dtype):
    log(f"append {BATCHES[batch][:4]} hd={hd} page={page} {layout} {rot} {dtype}")
    s = Setup(BATCHES[batch], page, 2, hd, batch, pad=batch % 3)
    table = B.rope_table(512, rot) if layout != "none" else None
    k, v, q = s.rows(2, dtype), s.rows(2, dtype), s.rows(6, dtype)
    _append_check(s, k, v, q if layout != "none" else None, table, layout if layout != "none" else "half", rot)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_append_from_a_product_s_rows(dtype, shift):
    """k, v and q inside the rows of one QKV product, aligned or not; one head of keys."""
    torch = _torch()
    s = Setup([(40, 3), (1, 77)], 64, 1, 64)
    wide = torch.randn(s.n, 10 * 64 + 8, device="cuda").to(getattr(torch, dtype))[:, shift:shift + 640].unflatten(1, (10, 64))
    _append_check(s, wide[:, 8:9], wide[:, 9:], wide[:, :8], B.rope_table(128, 64), "half", 64)


def test_append_leaves_what_is_out_of_range():
    """Pages outside the pool, lengths and rows outside theirs, positions behind the table."""
    s = Setup([(20, 35), (1, 70), (1, 3), (1, 4), (1, 20)], 32, 2, 64, extra_pages=1, pad=4)
    pages = s.pages_h.copy()
    pages[0, 1], pages[3, 0], pages[4, 0] = -1, s.n_pages, 2 ** 31 - 1
    s.set(pages, s.starts_h, [35, 70, -1, 4, 20])
    _append_check(s, s.rows(2), s.rows(2), s.rows(4), B.rope_table(64, 64), "half", 64)
    s.set(s.pages_h, [0, 20, 10, 500, -4, 6], [30, 2, 4 * 32, 5, 6])
    _append_check(s, s.rows(2), s.rows(2), s.rows(4), B.rope_table(64, 64), "half", 64)
    s.set(s.pages_h, [-4, 20, 21, 22, 23, 24], [126, 127, 128, 1 << 30, 100])
    _append_check(s, s.rows(2), s.rows(2), s.rows(4), B.rope_table(200, 64), "half", 64)


def test_append_special_values():
    """NaN and infinities arrive as they are, unrotated; large numbers round to infinity."""
    torch = _torch()
    s = Setup([(3, 62)], 64, 1, 64)
    k = torch.zeros(3, 1, 64, device="cuda")
    k[0, 0, 5], k[1, 0, 6], k[2, 0, 7] = float("nan"), float("-inf"), 3.4e38
    B.op_paged_append(s.cache, k, k, s.pages, s.starts, s.lens)
    for pool in s.plain():
        got = [pool[s.pages_h[0, p // 64], 0, p % 64] for p in (62, 63, 64)]
        assert np.isnan(got[0][5]) and got[1][6] == -np.inf and got[2][7] == np.inf
        assert np.isfinite(np.delete(got[0], 5)).all()


# ----------------------------------------------------------------- attention
def _attend(s, q, **kw):
    torch = _torch()
    out = torch.full((s.n, q.shape[1] * s.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    B.op_attention_paged(q, s.cache, s.pages, s.starts, s.lens, kw.pop("max_new", s.max_new), out=out, **kw)
    return out


def _attend_check(s, q, **kw):
    out = _attend(s, q, **kw)
    kw.pop("shared", None)
    kw.pop("ws", None)
    want, tol, token = R.attention(_np(q), *s.plain(), s.batch, kw.pop("max_new", s.max_new), **kw)
    got = _np(out).reshape(want.shape)
    bad = ~(abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want)) & ~(np.isinf(want) & (got == want))
    assert not bad[token].any(), (np.argwhere(bad & token[:, None, None])[:5], abs(got - want)[token].max())
    assert (got[~token] == 7.0).all()
    return out


ATTEND = [
    [(1, 0)], [(1, 1), (2, 0)], [(1, 30), (1, 31), (1, 32), (1, 33)], [(1, 63), (1, 64), (1, 65), (0, 9)], [(1, 500), (1, 3), (1, 1111)],
    [(5, 0), (1, 200), (70, 30), (3, 61)], [(17, 300)], [(33, 31), (32, 0), (31, 1)], [(200, 0)], [(150, 333), (1, 700), (20, 5)],
    [(1, 2500)], [(3, 5000), (1, 4000)]]


@pytest.mark.parametrize("hd,page,Hkv,G", [(64, 32, 2, 1), (64, 64, 1, 8), (128, 128, 2, 4), (128, 32, 1, 3), (64, 256, 3, 2), (128, 64, 1, 20)])
@pytest.mark.parametrize("batch", range(len(ATTEND)))
def test_attention(batch, hd, page, Hkv, G):
    log(f"attention {ATTEND[batch][:4]} hd={hd} page={page} {Hkv} x {G}")
    s = Setup(ATTEND[batch], page, Hkv, hd, batch, pad=batch % 3, stale=float("nan"))
    _attend_check(s, s.rows(Hkv * G))


@pytest.mark.parametrize("hd,page", [(64, 32), (128, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (32, 4), (33, 32), (64, 40), (100, 0), (100, 65), (500, 7), (2 ** 31 - 1, 0), (7, 2 ** 31 - 1)])
def test_attention_windows(window, sinks, hd, page):
    log(f"windows {window} {sinks} {hd}")
    s = Setup([(1, 0), (1, 99), (40, 300), (3, 64), (1, 1500), (90, 0)], page, 2, hd, 5, stale=float("inf"))
    _attend_check(s, s.rows(4), window=window, sinks=sinks)


@pytest.mark.parametrize("n0", [0, 27, 31, 32, 61, 63, 64])
def test_attention_every_border(n0):
    """Token by token over the borders of groups, pages and windows."""
    s = Setup([(4, n0 + i) for i in range(0, 40)], 32, 1, 64, n0, stale=float("nan"))
    _attend_check(s, s.rows(2), window=34, sinks=2)
    _attend_check(s, s.rows(2))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("T", [3, 45, 300])
def test_attention_masked_numbers_count_for_nothing(T, hd):
    """NaN and infinities in keys and values of later tokens, of tokens before the
    window and behind the last: a query that does not see them is as without them, to
    the bit; one that does is what the formula says."""
    torch = _torch()
    s = Setup([(T, 100), (1, 60)], 32, 2, hd, T, extra_pages=1)
    q = s.rows(4)
    clean = _attend(s, q, window=90, sinks=2)
    at = [2 + 9, 100 + T // 2, 100 + T - 1, 100 + T]  # outside the window, between the queries, the last, behind it
    plain = [R.in_pool(np.arange(x.numel()).reshape(x.shape), bool(i)) for i, x in enumerate(s.cache)]
    for j, value in zip(at, (float("nan"), float("inf"), float("-inf"), float("nan"))):
        for x, p in zip(s.cache, plain):
            where = p[s.pages_h[0, j // 32], :, j % 32, 1::7].reshape(-1)
            x.view(-1)[torch.from_numpy(where).cuda()] = value
    out = _attend(s, q, window=90, sinks=2)
    first = 100 + T // 2 - 100  # rows before it see none of them
    lo = 11 + 90 - 100  # rows up to 11 + 90 - 1 see the first
    same = [r for r in range(max(0, lo), first)]
    assert torch.equal(out[same], clean[same]) and torch.equal(out[T:], clean[T:])
    if first < T:
        assert not torch.isfinite(out[first].float()).all()


@pytest.mark.parametrize("T", [2, 40])
def test_attention_visible_infinities_of_values(T):
    torch = _torch()
    s = Setup([(T, 30)], 32, 1, 64, 3)
    plain = R.in_pool(np.arange(s.cache[1].numel()).reshape(s.cache[1].shape), True)
    for j, d, value in ((30, 5, float("inf")), (31, 9, float("-inf")), (30, 60, float("nan")), (29, 17, float("inf"))):
        s.cache[1].view(-1)[int(plain[s.pages_h[0, j // 32], 0, j % 32, d])] = value
    _attend_check(s, s.rows(2))


def _set_keys(s, tokens, value, dim=slice(None)):
    """The keys of the first sequence's tokens, or one dim of them."""
    torch = _torch()
    plain = R.in_pool(np.arange(s.cache[0].numel()).reshape(s.cache[0].shape), False)
    for j in tokens:
        at = np.atleast_1d(plain[s.pages_h[0, j // s.page], :, j % s.page, dim]).reshape(-1)
        s.cache[0].view(-1)[torch.from_numpy(at).cuda()] = value


@pytest.mark.parametrize("T", [1, 30])
@pytest.mark.parametrize("tokens", [range(3), range(4500), range(5000)])
def test_attention_keys_that_are_no_numbers(T, tokens):
    """A NaN among the keys that a query sees is one in its result, in whichever of its parts."""
    s = Setup([(T, 5000), (1, 40)], 64, 1, 128, 3)
    _set_keys(s, tokens, float("nan"))
    out = _attend_check(s, s.rows(4))
    assert bool(out[:T].isnan().all()) and bool(out[T:].isfinite().all())


@pytest.mark.parametrize("T", [1, 30])
def test_attention_scores_of_minus_infinity(T):
    """They weigh nothing beside others; where there are no others the result is zeros."""
    s = Setup([(T, 5000), (1, 40)], 64, 1, 128, 3)
    q = s.rows(4)
    q[:, :, 0] = 1.0
    older = 4700
    _set_keys(s, range(older), 0.0)
    want, tol, _ = R.attention(_np(q)[T - 1:T], *s.plain(), R.Batch(s.pages_h[:1], np.array([0, 1]), np.array([5000 + T - 1]), 1, s.n_pages, s.page), 1,
                               window=5000 + T - older)
    _set_keys(s, range(older), float("-inf"), 0)
    got = _np(_attend(s, q)).reshape(s.n, 4, 128)
    assert (abs(got[T - 1] - want[0]) <= tol[0]).all()
    _set_keys(s, range(older, 5000 + T), float("-inf"), 0)
    assert (_np(_attend(s, q))[:T] == 0).all()


def test_attention_pages_outside_the_pool():
    """Their tokens count as masked; a query that sees no other gets zeros."""
    s = Setup([(40, 100), (1, 20), (2, 90), (1, 64)], 32, 2, 64, 4, stale=float("nan"))
    pages = s.pages_h.copy()
    pages[0, 1], pages[1, 0], pages[2, 2], pages[3, :] = -1, s.n_pages, 2 ** 31 - 1, -7
    s.set(pages, s.starts_h, s.lens_h)
    out = _attend_check(s, s.rows(4))
    assert (out[40] == 0).all() and (out[43] == 0).all()


def test_attention_leaves_what_is_out_of_range():
    """Lengths and rows outside theirs, more new tokens than max_new."""
    s = Setup([(20, 35), (1, 70), (1, 3), (5, 4), (1, 20)], 32, 2, 64, pad=3)
    _attend_check(s, s.rows(4), max_new=4)
    s.set(s.pages_h, s.starts_h, [35, -1, 96, 1 << 30, 95])
    _attend_check(s, s.rows(4))
    s.set(s.pages_h, [0, 20, 10, 500, -4, 6], [35, 2, 3, 5, 6])
    _attend_check(s, s.rows(4))
    s.set(s.pages_h, [0, 20, 21, 22, 27, 28], [90, 95, 94, 93, 92])
    _attend_check(s, s.rows(4))


def test_attention_scale_and_large_scores():
    s = Setup([(9, 100), (1, 1000)], 64, 2, 128, 6)
    _attend_check(s, s.rows(4), scale=0.5)
    _attend_check(s, s.rows(4) * 8, scale=1.0)  # most probabilities vanish


def test_attention_does_not_depend_on_the_batch():
    """A sequence's bits are its own: alone, beside others, with wider page tables, in
    another order, behind rows of other lengths."""
    torch = _torch()
    for seqs in ([(1, 3000), (1, 10), (1, 700)], [(90, 3000), (1, 10), (30, 700), (260, 5)]):
        s = Setup(seqs, 64, 2, 64, 8)
        q = s.rows(8)
        whole = _attend(s, q)
        pages, starts, lens = s.pages_h, s.starts_h, s.lens_h
        wide = np.concatenate([pages, np.full((len(seqs), 300), -1)], 1)
        assert torch.equal(_attend(s.set(wide, starts, lens), q), whole)
        order = list(range(len(seqs)))[::-1]
        new = np.concatenate([[0], np.cumsum([seqs[b][0] for b in order])])
        rows = np.concatenate([np.arange(starts[b], starts[b + 1]) for b in order])
        r = torch.from_numpy(rows).cuda()
        assert torch.equal(_attend(s.set(pages[order], new, lens[order]), q[r]), whole[r])
        for b in range(len(seqs)):
            one = Setup([seqs[b]], 64, 2, 64)
            one.cache, one.n_pages = s.cache, s.n_pages
            one.set(pages[b:b + 1], [0, seqs[b][0]], lens[b:b + 1])
            sl = slice(starts[b], starts[b + 1])
            assert torch.equal(_attend(one, q[sl].contiguous(), max_new=s.max_new), whole[sl]), b


def test_attention_splits_do_not_follow_the_number_of_rows():
    """max_new decides how a long sequence is split, not the rows that a batch has."""
    torch = _torch()
    for new in (1, 30):
        s = Setup([(new, 3000), (2000, 5)], 64, 2, 64, 8)
        q = s.rows(8)
        for most in (2000, 9000):
            whole = _attend(s, q, max_new=most)
            one = Setup([(new, 3000)], 64, 2, 64)
            one.cache, one.n_pages = s.cache, s.n_pages
            one.set(s.pages_h[:1], [0, new], s.lens_h[:1])
            assert torch.equal(_attend(one, q[:new].contiguous(), max_new=most), whole[:new]), (new, most)


# Around the borders between the forms: 64 columns of any sequence, 512 of one of at
# most 512 keys of 128 (1024 of 64) where max_new allows no more.
@pytest.mark.parametrize("new,old", [(16, 100), (17, 100), (17, 495), (17, 496), (128, 384), (128, 385), (17, 1007), (17, 1008), (128, 896),
                                     (128, 897), (127, 0), (129, 100), (128, 2000)])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_borders_of_the_forms(new, old, hd):
    s = Setup([(new, old), (1, 2000), (3, 0)], 64, 2, hd, new)
    _attend_check(s, s.rows(8))
    _attend_check(s, s.rows(8), window=200, sinks=3)


@pytest.mark.parametrize("new,old", [(16, 1200), (17, 1200), (17, 1900), (128, 1200), (128, 1900), (129, 1200), (300, 1200)])
def test_attention_shared_borders_of_the_forms(new, old):
    s = Setup([(new, old), (1, 1500), (3, 1155)], 64, 2, 64, new, shared=1152)
    _attend_check(s, s.rows(8), shared=1152)


# ------------------------------------------------------------------- shared
@pytest.mark.parametrize("hd,page,Hkv,G", [(64, 32, 2, 1), (64, 64, 1, 8), (128, 128, 2, 4), (128, 64, 2, 2)])
@pytest.mark.parametrize("shared,seqs", [
    (64, [(1, 64), (1, 70)]), (640, [(1, 700), (1, 641), (1, 640)]), (1000, [(3, 1000), (1, 1200), (2, 1001), (20, 1100)]),
    (2048, [(1, 2050 + 9 * i) for i in range(40)]), (300, [(100, 300), (70, 301)]), (63, [(1, 70), (1, 63)])])
def test_shared(shared, seqs, hd, page, Hkv, G):
    log(f"shared {shared} {seqs[:3]} hd={hd} page={page} {Hkv} x {G}")
    torch = _torch()
    s = Setup(seqs, page, Hkv, hd, shared, pad=2, shared=shared)
    # the rest of the prefix, on a page of each sequence's own, is the same too
    if shared % page:
        k = shared // page
        for i, x in enumerate(s.cache):
            at = R.in_pool(np.arange(x[0].numel()).reshape((1,) + tuple(x.shape[1:])), bool(i))[0][:, :shared % page].reshape(-1)
            for b in range(1, len(seqs)):
                x[int(s.pages_h[b, k])].view(-1)[torch.from_numpy(at).cuda()] = x[int(s.pages_h[0, k])].view(-1)[torch.from_numpy(at).cuda()]
    q = s.rows(Hkv * G)
    _attend_check(s, q, shared=shared)
    _attend_check(s, q, shared=shared, window=200, sinks=3)
    _attend_check(s, q, shared=shared, window=shared + 20)


def test_shared_tokens_inside_the_prefix():
    """Sequences whose new tokens lie inside what is called shared see no later token of it."""
    s = Setup([(3, 10), (1, 63), (2, 100), (4, 126), (1, 300)], 64, 2, 64, 3, shared=256, stale=None)
    _attend_check(s, s.rows(4), shared=256)
    _attend_check(s, s.rows(4), shared=256, window=40, sinks=70)


@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("B_", [65, 150])
def test_shared_by_more_sequences_than_lanes(B_, G):
    """(some of them without rows)"""
    s = Setup([(0 if b % 9 == 4 else 2 if b % 9 == 5 else 1, 128 + b % 70) for b in range(B_)], 64, 1, 64, B_, pad=2, shared=128)
    q = s.rows(G)
    _attend_check(s, q, shared=128)
    _attend_check(s, q, shared=128, window=90, sinks=3)


def test_shared_of_one_sequence_and_of_none():
    torch = _torch()
    s = Setup([(2, 300)], 64, 2, 64, 3)
    q = s.rows(4)
    assert torch.equal(_attend(s, q, shared=256), _attend(s, q))
    s = Setup([(2, 300), (1, 400)], 64, 2, 64, 3, shared=256)
    q = s.rows(4)
    assert torch.equal(_attend(s, q, shared=40), _attend(s, q))  # less than is worth it


def test_shared_reads_the_first_sequence_s_pages():
    """(and masked numbers on them count for nothing, whatever they are)"""
    s = Setup([(1, 100), (1, 70), (1, 64)], 64, 1, 64, 3, shared=64, stale=float("nan"))
    _attend_check(s, s.rows(4), shared=64)
    pages = s.pages_h.copy()
    pages[:, 0] = -1
    s.set(pages, s.starts_h, s.lens_h)
    _attend_check(s, s.rows(4), shared=64)


# ------------------------------------------------------------ ways of calling
def test_strided_queries_and_defaults():
    torch = _torch()
    s = Setup([(3, 100), (1, 20)], 64, 2, 64, 1)
    wide = torch.randn(s.n, 640, device="cuda").to(torch.bfloat16)
    q = wide[:, 64:64 + 256].unflatten(1, (4, 64))
    got = B.op_attention_paged(q, s.cache, s.pages, s.starts, s.lens, 3)
    assert torch.equal(got, _attend(s, q.contiguous()))


def test_on_another_stream():
    torch = _torch()
    s = Setup([(30, 400), (1, 2000)], 64, 2, 64, 1)
    q, k, v = s.rows(8), s.rows(2), s.rows(2)
    table = B.rope_table(2048, 64)
    saved = [x.clone() for x in s.cache]
    q1 = B.op_paged_append(s.cache, k, v, s.pages, s.starts, s.lens, rope=table, q=q)
    want = _attend(s, q1)
    after = [x.clone() for x in s.cache]
    for x, y in zip(s.cache, saved):
        x.copy_(y)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q2 = B.op_paged_append(s.cache, k, v, s.pages, s.starts, s.lens, rope=table, q=q, stream=st)
    got = B.op_attention_paged(q2, s.cache, s.pages, s.starts, s.lens, s.max_new, stream=st)
    st.synchronize()
    assert torch.equal(got, want) and torch.equal(q1, q2) and all(torch.equal(x, y) for x, y in zip(s.cache, after))


def test_steps_in_graphs_that_share_a_workspace():
    """Two captured steps (one with a shared prefix) on one workspace, replayed by turns
    with other lengths, pages and rows each time, with eager work in between."""
    torch = _torch()
    s = Setup([(1, 1100 + 13 * i) for i in range(6)], 64, 2, 64, 9, shared=1024, extra_pages=2)
    q, k, v = s.rows(8), s.rows(2), s.rows(2)
    table = B.rope_table(2048, 64)
    q_out, out = torch.zeros_like(q), [torch.zeros(s.n, 8 * 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tokens = s.pages.shape[1] * 64
    ws = torch.empty(max(B.paged_workspace(s.n, 6, 8, 2, 64, 1, tokens, sh) for sh in (0, 1024)), dtype=torch.uint8, device="cuda")

    def step(i):
        B.op_paged_append(s.cache, k, v, s.pages, s.starts, s.lens, rope=table, q=q, q_out=q_out)
        B.op_attention_paged(q_out, s.cache, s.pages, s.starts, s.lens, 1, shared=1024 * i, out=out[i], ws=ws)
    step(0), step(1)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i)
        graphs.append(g)
    for turn in range(3):
        s.lens += 1
        q.normal_(), k.normal_(), v.normal_()
        for i in (0, 1):
            graphs[i].replay()
            torch.cuda.synchronize()
            got = out[i].clone()
            want = B.op_attention_paged(q_out, s.cache, s.pages, s.starts, s.lens, 1, shared=1024 * i)
            assert torch.equal(got, want), (turn, i)
            ws.fill_(255)
    s.set(s.pages_h, s.starts_h, s.lens.cpu().numpy())
    _attend_check(s, q_out, max_new=1, shared=1024)


def test_pools_past_32_bits():
    """Pages behind 2^32 bytes and 2^31 numbers of a pool."""
    torch = _torch()
    page, Hkv, hd = 256, 32, 128
    n_pages = 2200  # 2.3e9 numbers each
    cache = tuple(torch.empty(n_pages, Hkv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = tuple(torch.zeros(4, Hkv, page, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v, q = (torch.randn(300, h, hd, device="cuda").to(torch.bfloat16) for h in (Hkv, Hkv, Hkv))
    starts, lens = _ints([0, 299, 300]), _ints([0, 0])
    got = []
    for c, pages in ((cache, [[2199, 1], [2198, 5]]), (small, [[0, 1], [2, 3]])):
        B.op_paged_append(c, k, v, _ints(pages), starts, lens, rope=B.rope_table(512, hd))
        got.append(B.op_attention_paged(q, c, _ints(pages), starts, lens, 299))
    assert torch.equal(got[0], got[1])
    assert all(torch.equal(a[2199], b[0]) for a, b in zip(cache, small))


def test_whole_windows_as_the_dense_attention():
    """A batch of whole windows, appended and attended in pages, beside the decoder's own
    kernel on dense K and V; then the last tokens again, one at a time."""
    torch = _torch()
    Bn, Hq, Hkv, W, hd = 3, 8, 2, 200, 64
    s = Setup([(W, 0)] * Bn, 64, Hkv, hd, 2)
    q, k, v = s.rows(Hq), s.rows(Hkv), s.rows(Hkv)
    table = B.rope_table(256, hd)
    qr = B.op_paged_append(s.cache, k, v, s.pages, s.starts, s.lens, rope=table, q=q)
    out = _attend_check(s, qr)
    pos = torch.arange(W, dtype=torch.int32, device="cuda").repeat(Bn)
    kr = B.op_rope(k, pos, table)
    assert torch.equal(B.op_rope(q, pos, table), qr)

    def dense(x):
        return x.view(Bn, W, -1, hd).transpose(1, 2).contiguous()
    ref = B.op_attention_bf16(dense(qr), dense(kr), dense(v).transpose(2, 3).contiguous())
    # both round their probabilities to bf16 (2^-8 each at most) and their result; values of up to 5
    assert (abs(out.float() - ref.float()) <= 2 * 5 * 2.0 ** -8 + 2.0 ** -7 * abs(ref.float())).all()
    # the last five tokens again, step by step
    for t in range(W - 5, W):
        rows = torch.arange(Bn, device="cuda") * W + t
        one = Setup([(1, t)] * Bn, 64, Hkv, hd)
        one.cache, one.n_pages = s.cache, s.n_pages
        one.set(s.pages_h, [0, 1, 2, 3], [t] * Bn)
        q1 = B.op_paged_append(one.cache, k[rows], v[rows], one.pages, one.starts, one.lens, rope=table, q=q[rows])
        assert torch.equal(q1, qr[rows])
        got = _attend(one, q1)
        assert (abs(got.float() - out[rows].float()) <= 2 * 5 * 2.0 ** -8 + 2.0 ** -7 * abs(out[rows].float())).all()


# ----------------------------------------------------- values that are no numbers
def _places(s, i, b, tokens, dims):
    """Where the numbers of a sequence's tokens lie in the pool of keys (i = 0) or values."""
    plain = R.in_pool(np.arange(s.cache[i].numel()).reshape(s.cache[i].shape), bool(i))
    j = np.asarray(list(tokens))
    return _torch().from_numpy(plain[s.pages_h[b, j // s.page], :, j % s.page][..., dims].reshape(-1)).cuda()


def _set(s, i, b, tokens, dims, value):
    s.cache[i].view(-1)[_places(s, i, b, tokens, dims)] = value


@pytest.mark.parametrize("at", [3, 600, 1030])
@pytest.mark.parametrize("seqs,G,hd,shared", [([(1, 1100)], 1, 128, 0), ([(70, 1100)], 1, 128, 0), ([(1, 1100), (1, 1040)], 2, 64, 1024),
                                              ([(20, 1024), (17, 1040)], 8, 64, 1024)])
def test_attention_visible_nan_in_a_part_of_no_weight(seqs, G, hd, shared, at):
    """A NaN among visible values is one in the result, whichever part of the keys holds it,
    and if all probabilities of that part are zero."""
    s = Setup(seqs, 64, 1, hd, 3, shared=shared)
    q = s.rows(G)
    q.zero_()
    q[:, :, 0] = hd ** 0.5
    for b, (T, n) in enumerate(seqs):
        _set(s, 0, b, range(T + n), slice(None), 0.0)
        _set(s, 0, b, range(512), [0], -160.0)
        _set(s, 0, b, range(512, T + n), [0], 160.0)
    _set(s, 1, 0, [at], [5], float("nan"))
    out = _attend_check(s, q, shared=shared).view(s.n, G, hd)
    sees = [row for b, row, pos in s.batch.rows() if pos >= at and (b == 0 or at < shared)]
    assert sees and bool(out[sees][:, :, 5].isnan().all())


@pytest.mark.parametrize("seqs,G,shared,most", [([(1, 40)], 1, 0, 1), ([(1, 1100)], 2, 0, 1), ([(20, 70)], 4, 0, 1000), ([(20, 1100)], 4, 0, 20),
                                                ([(1, 70), (2, 70)], 1, 64, 2), ([(20, 70), (18, 70)], 8, 64, 20)])
def test_attention_scores_of_minus_infinity_beside_nan(seqs, G, shared, most):
    """Queries whose scores are all -infinity get zeros, whatever the values are."""
    s = Setup(seqs, 32, 1, 64, 3, shared=shared)
    q = s.rows(G)
    q[:, :, 0] = 1.0
    for b, (T, n) in enumerate(seqs):
        _set(s, 0, b, range(T + n), [0], float("-inf"))
        _set(s, 1, b, [3, n], [5, 6], float("nan"))
    assert (_np(_attend(s, q, shared=shared, max_new=most)) == 0).all()


@pytest.mark.parametrize("rising", [0.0, 0.2])
@pytest.mark.parametrize("seqs,G,hd,shared,kw", [
    ([(1, 40)], 1, 64, 0, {}), ([(1, 1500)], 2, 128, 0, {}), ([(20, 170)], 4, 64, 0, dict(max_new=1000)),
    ([(20, 170)], 4, 64, 0, dict(max_new=1000, window=60, sinks=3)), ([(20, 1100), (1, 5000)], 4, 128, 0, {}),
    ([(1, 700), (2, 650)], 1, 64, 640, {}), ([(20, 700), (18, 650)], 8, 64, 640, {})])
def test_attention_values_near_the_largest(seqs, G, hd, shared, kw, rising):
    """Their mean is a number where their sum is none; with scores around zero and with such
    that rise from key to key."""
    torch = _torch()
    s = Setup(seqs, 64, 1, hd, 3, shared=shared)
    q = s.rows(G)
    v = torch.full((s.n_pages, 1, 64, hd), 3.3e38, device="cuda") - 1e37 * torch.randint(0, 7, (s.n_pages, 1, 64, hd), device="cuda")
    s.cache[1].copy_(v.to(torch.bfloat16))
    if rising:
        q[:, :, 0] = 1.0
        for b, (T, n) in enumerate(seqs):
            _set(s, 0, b, range(T + n), [0], rising * hd ** 0.5 * (torch.arange(T + n, device="cuda") % 1024).to(torch.bfloat16))
    _attend_check(s, q, shared=shared, **kw)


def test_attention_of_single_tokens_of_as_many_sequences_as_there_may_be():
    """65535 on 32 heads: some of them beside float64, all of them by a smaller call's bits."""
    torch = _torch()
    s = Setup([(1, 63)], 64, 32, 64, 3)
    some, n = 40, 65535
    lens = np.arange(n) % 64
    s.n = n
    q = s.rows(32)
    pages = np.repeat(s.pages_h, n, 0)
    whole = B.op_attention_paged(q, s.cache, _ints(pages), _ints(np.arange(n + 1)), _ints(lens), 1)
    s.n = some
    s.set(pages[:some], np.arange(some + 1), lens[:some])
    assert torch.equal(_attend_check(s, q[:some], max_new=1), whole[:some])
    for first in range(some, n, 16384):
        s.n = min(16384, n - first)
        s.set(pages[:s.n], np.arange(s.n + 1), lens[first:first + s.n])
        assert torch.equal(_attend(s, q[first:first + s.n], max_new=1), whole[first:first + s.n])


@pytest.mark.parametrize("G", [1, 8])
def test_shared_rows_of_no_token_may_hold_anything(G):
    torch = _torch()
    s = Setup([(3, 640), (40, 700)], 64, 1, 64, 3, shared=640, pad=30)
    q = s.rows(G)
    clean = _attend_check(s, q, shared=640)
    q[43:, :, ::9] = float("nan")
    q[50:60] = float("inf")
    assert torch.equal(_attend(s, q, shared=640), clean)


@pytest.mark.parametrize("at", [1, 95, 100, 105, 119, 150])
@pytest.mark.parametrize("keys,value", [(False, float("nan")), (False, float("-inf")), (True, float("nan")), (True, float("inf"))])
@pytest.mark.parametrize("G,hd,sinks", [(2, 64, 0), (2, 128, 3), (12, 64, 3), (12, 128, 0)])
def test_shared_masked_numbers_count_for_nothing(G, hd, sinks, keys, value, at):
    """NaN and infinities on a prefix that a window hides from some columns of a wave and not
    from others, 46 columns or 276: who does not see them is as without, to the bit."""
    torch = _torch()
    s = Setup([(12, 200), (1, 220), (9, 192), (1, 300)], 64, 1, hd, 3, shared=192)
    q = s.rows(G)
    clean = _attend_check(s, q, shared=192, window=101, sinks=sinks)
    _set(s, 0 if keys else 1, 0, [at], [5], value)
    out = _attend_check(s, q, shared=192, window=101, sinks=sinks)
    blind = [row for b, row, pos in s.batch.rows() if at <= pos - 101 and at >= sinks]
    assert blind and torch.equal(out[blind], clean[blind]) if at >= sinks else not blind
    sees = [row for row in range(s.n) if row not in blind]
    if not keys and sees:
        assert not bool(out[sees].view(len(sees), G, hd)[:, :, 5].isfinite().any())


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 70)])
@pytest.mark.parametrize("hd,page", [(64, 64), (128, 256)])
@pytest.mark.parametrize("new,old", [(70, 3000), (300, 4500), (70, 9000)])
def test_attention_long_prompts_in_one_part(new, old, hd, page, window, sinks, odd):
    """As a large max_new has it: more steps than the 32 whose pages are looked up at once;
    walked twice where a value that some queries do not see is no number."""
    log(f"long prompts {new} {old} {hd} {window} {odd}")
    s = Setup([(new, old), (1, 2300), (65, 2100)], page, 1, hd, new, stale=float("nan"))
    if odd:
        _set(s, 1, 0, [old + new // 2], [3], float("nan"))
        _set(s, 1, 0, [old - 2470], [4], float("inf"))
    _attend_check(s, s.rows(1), max_new=1 << 20, window=window, sinks=sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (2700, 70)])
@pytest.mark.parametrize("hd", [64, 128])
def test_shared_long_prefix_in_one_part(hd, window, sinks):
    """128 heads by two tiles of columns fill the chip, so the prefix is one part of 40 steps; beside
    float64 for some of the heads."""
    s = Setup([(150, 2560), (151, 2600)], 64, 128, hd, 3, shared=2560)
    q = s.rows(128)
    out = _attend(s, q, shared=2560, window=window, sinks=sinks)
    heads = [0, 77, 127]
    want, tol, token = R.attention(_np(q[:, heads]), *(R.in_pool(_np(x[:, heads]), bool(i)) for i, x in enumerate(s.cache)), s.batch, s.max_new,
                                   window=window, sinks=sinks)
    assert token.all() and (abs(_np(out).reshape(s.n, 128, hd)[:, heads] - want) <= tol).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_a_row_between_masked_numbers(hd, keys, value):
    """Of three new tokens the first sees a number that is none before the others' windows, the last
    one at its own place; the second, in the same wave, is as without them, to the bit."""
    torch = _torch()
    s = Setup([(3, 100), (1, 60)], 32, 2, hd, 3)
    q = s.rows(4)
    clean = _attend_check(s, q, window=90)
    _set(s, 0 if keys else 1, 0, [11, 102], [6], value)
    out = _attend_check(s, q, window=90)
    assert torch.equal(out[[1, 3]], clean[[1, 3]])
    if not keys:
        assert not bool(out[[0, 2]].view(2, 4, hd)[:, :, 6].isfinite().any())


@pytest.mark.parametrize("seqs,G,hd,shared", [([(1, 1500)], 2, 128, 0), ([(20, 1100), (1, 5000)], 4, 128, 0), ([(1, 700), (2, 650)], 1, 64, 640),
                                              ([(20, 700), (18, 650)], 8, 64, 640)])
def test_attention_small_values_keep_their_digits(seqs, G, hd, shared):
    """Values 2^115 times smaller give results as much smaller, to a step of bf16."""
    torch = _torch()
    s = Setup(seqs, 64, 1, hd, 3, shared=shared)
    q = s.rows(G)
    s.cache[1].copy_((1 + s.cache[1].float().abs().clamp(max=2)).to(torch.bfloat16))
    whole = _attend(s, q, shared=shared)
    s.cache[1].mul_(2.0 ** -115)
    small = _attend(s, q, shared=shared)
    # half a step of bf16 (2^-8) each; float32 sums weighted 2^-11 of values past 2^-115 keep 2^-20
    assert (abs(small.double() * 2.0 ** 115 - whole.double()) <= 2.0 ** -7 * whole.double()).all()
