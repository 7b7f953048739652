"""Plain NumPy references (float64) of rotary positions, the paged key/value cache
and attention over it, written from the definitions in include/lmgc.h."""
import numpy as np


def key_at(t, d, hd):
    return ((t // 16) * (hd // 32) + d // 32) * 512 + ((t % 16) + 16 * ((d % 32) // 8)) * 8 + d % 8


def value_at(t, d):
    return (d // 16) * 512 + ((d % 16) + 16 * ((t % 16) // 4)) * 8 + 4 * (t // 16) + t % 4


def rotate(x, angles, layout, backward=False):
    """x [..., hd] float64, angles [..., rot / 2, 2] (cos, sin), broadcast over the heads -> (rotated, sum of |products|)."""
    y, mag = x.copy(), np.zeros_like(x)
    rot = 2 * angles.shape[-2]
    c, s = angles[..., 0], angles[..., 1] * (-1 if backward else 1)
    i = np.arange(rot // 2)
    p, q = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = x[..., p], x[..., q]
    y[..., p], y[..., q] = a * c - b * s, a * s + b * c
    mag[..., p], mag[..., q] = abs(a * c) + abs(b * s), abs(a * s) + abs(b * c)
    return y, mag


class Batch:
    """Ragged rows over pages: what counts of it."""

    def __init__(self, pages, starts, lens, n, n_pages, page):
        self.pages, self.starts, self.lens = np.asarray(pages), list(starts), list(lens)
        self.n, self.n_pages, self.page = n, n_pages, page
        self.tokens = self.pages.shape[1] * page

    def rows(self, limit=1 << 30):
        """(sequence, row, position) of every new token."""
        for b, n in enumerate(self.lens):
            r0, r1 = self.starts[b], self.starts[b + 1]
            if not (0 <= r0 <= r1 <= self.n and 0 <= n < self.tokens):
                continue
            for t in range(min(r1 - r0, limit, self.tokens - n)):
                yield b, r0 + t, n + t

    def places(self, b, upto):
        """(page, token of the page) of positions 0 .. upto - 1; page -1: none."""
        p = np.arange(upto)
        page = self.pages[b][p // self.page]
        return np.where((page >= 0) & (page < self.n_pages), page, -1), p % self.page


def in_pool(pool, values):
    """The pool [n_pages, Hkv, page, hd] in plain order (page, head, token, dim)."""
    n, H, P, hd = pool.shape
    t, d = np.arange(32)[:, None], np.arange(hd)[None, :]
    at = value_at(t, d) + 0 * d if values else key_at(t, d, hd)
    return pool.reshape(n, H, P // 32, 32 * hd)[..., at].reshape(n, H, P, hd)


def attention(q, kp, vp, batch, max_new, window=0, sinks=0, scale=None):
    """q [n, Hq, hd], pools in plain order, all float64 -> (o [n, Hq, hd], bound of what
    rounding the probabilities and the result to bf16 and the scores to float32 changes,
    which rows are tokens)."""
    n, Hq, hd = q.shape
    Hkv = kp.shape[1]
    G = Hq // Hkv
    scale = hd ** -0.5 if scale is None else scale
    o, tol, token = np.zeros((n, Hq, hd)), np.zeros((n, Hq, hd)), np.zeros(n, bool)
    seqs = {}
    for b, row, pos in batch.rows(max_new):
        seqs.setdefault(b, []).append((row, pos))
    for b, rows in seqs.items():
        L = rows[-1][1] + 1
        page, at = batch.places(b, L)
        k = kp[np.maximum(page, 0), :, at]  # [L, Hkv, hd]
        v = vp[np.maximum(page, 0), :, at]
        r = np.array([x for x, _ in rows])
        pos = np.array([p for _, p in rows])[:, None]
        j = np.arange(L)[None, :]
        see = (j <= pos) & (page >= 0)[None, :]
        if window:
            see &= (j > pos - window) | (j < sinks)
        token[r] = True
        for h in range(Hkv):
            qs = q[r, h * G:(h + 1) * G]
            hid = ~see.any(0)
            kk, vv = np.where(hid[:, None], 0.0, k[:, h]), np.where(hid[:, None], 0.0, v[:, h])
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(see[:, None], scale * np.einsum("rgd,jd->rgj", qs, kk), -np.inf)
                size = scale * np.max(np.where(see[:, None], np.einsum("rgd,jd->rgj", abs(qs), abs(kk)), 0.0), axis=-1)
                m = s.max(-1, keepdims=True)
                p = np.where(see[:, None], np.exp(s - np.where(np.isneginf(m), 0.0, m)), 0.0)
                l = p.sum(-1, keepdims=True)
                p = np.divide(p, l, out=np.zeros_like(p), where=l != 0)
                # (a masked value counts for nothing, whatever it is)
                if np.isfinite(vv).all():
                    w = np.einsum("rgj,jd->rgd", p, vv)
                    dev = np.einsum("rgj,jd->rgd", p, abs(vv)) + abs(w)  # >= sum p |v - o|
                else:
                    t = np.where(see[:, None, :, None], p[..., None] * vv[None, None], 0.0)
                    w, dev = t.sum(2), abs(t).sum(2) + abs(t.sum(2))
            # p (1 + e): |e| <= 2^-8 for bf16, and what float32 sums of hd products and an exponential do
            e = 2.0 ** -8 + 2.0 ** -22 + 2.0 ** -24 * (hd + 8) * size[..., None]
            o[r, h * G:(h + 1) * G] = w
            tol[r, h * G:(h + 1) * G] = e * dev * (1 + 2.0 ** -6) + 2.0 ** -8 * abs(w) + 1e-37
    return o, tol, token
