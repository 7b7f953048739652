"""Plain NumPy references (float64) of the operators in fewer bits: microscaled
rows and blocks, the 8-bit key/value cache and attention over it, written from
the definitions in include/lmgc.h."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _e4m3(code):
    s, e, m = code >> 7, (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return np.nan
    v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
    return -v if s else v


E4M3 = np.array([_e4m3(c) for c in range(256)])
TOP = {"fp8": 448.0, "fp4": 6.0}
POSITIVE = {"fp8": E4M3[:127], "fp4": E2M1}


def nearest(x, fmt):
    """Magnitude codes of the nearest number to |x| <= top, half to the even code."""
    grid = POSITIVE[fmt]
    hi = np.clip(np.searchsorted(grid, x), 0, len(grid) - 1)  # grid[hi] >= x
    lo = np.maximum(hi - 1, 0)
    dl, dh = x - grid[lo], grid[hi] - x
    return np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))


def power_at_least(x, low):
    """Exponent e >= low of the smallest 2^e >= x (x >= 0)."""
    m, e = np.frexp(x)
    e = np.where(m == 0.5, e - 1, e)
    return np.maximum(np.where(m == 0, low, e), low)


def up(n, m):
    return -(-n // m) * m


def mx_quantize(x, fmt):
    """x [rows, cols] (any float type) -> (codes uint8 [rows, Kp], one to a byte; scale bytes [rows, Kp / 32])."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    z = np.zeros((rows, up(cols, 128)))
    z[:, :cols] = x
    z = z.reshape(rows, -1, 32)
    bad = ~np.isfinite(z).all(-1)
    z = np.where(bad[..., None], 0.0, z)
    e = power_at_least(np.abs(z).max(-1) / TOP[fmt], -127)
    v = z / np.ldexp(1.0, e)[..., None]
    codes = nearest(np.abs(v), fmt) | np.where(np.signbit(v), 128 if fmt == "fp8" else 8, 0)
    return codes.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def mx_values(codes, bytes_, fmt, cols):
    table = E4M3 if fmt == "fp8" else np.concatenate([E2M1, -E2M1])
    s = np.where(bytes_ == 255, np.nan, np.ldexp(1.0, bytes_.astype(int) - 127))
    return (table[codes].reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape[0], -1)[:, :cols]


def rows_layout(codes, bytes_, fmt, cols):
    """What the buffers of the rows layout hold."""
    if fmt == "fp4":
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    out = np.zeros((codes.shape[0], 16 * -(-cols // 512)), np.uint8)
    for j in range(bytes_.shape[1]):
        out[:, 16 * (j // 16) + 4 * (j % 4) + (j % 16) // 4] = bytes_[:, j]
    return codes, out


def blocks_layout(codes, bytes_, cols):
    N, kp = codes.shape
    packed = codes[:, 0::2] | (codes[:, 1::2] << 4)
    nk, ns, ng = kp // 128, -(-cols // 512), -(-N // 16)
    bc, bs = np.zeros(ng * nk * 1024, np.uint8), np.zeros(ng * ns * 256, np.uint8)
    for n in range(N):
        for j in range(kp // 32):
            k, g = j // 4, j % 4
            at = 1024 * ((n // 16) * nk + k) + 16 * (n % 16 + 16 * g)
            bc[at:at + 16] = packed[n, 16 * j:16 * j + 16]
            bs[256 * ((n // 16) * ns + k // 4) + 4 * (n % 16 + 16 * g) + k % 4] = bytes_[n, j]
    return bc, bs


# ------------------------------------------------------------ 8-bit cache --
def key_index(hd):
    t, d = np.arange(64)[:, None], np.arange(hd)[None, :]
    return ((t // 16) * (hd // 64) + d // 64) * 1024 + ((t % 16) + 16 * ((d % 64) // 16)) * 16 + d % 16


def value_index(hd):
    t, d = np.arange(64)[:, None], np.arange(hd)[None, :]
    return (d // 16) * 1024 + ((d % 16) + 16 * ((t % 16) // 4)) * 16 + 4 * (t // 16) + t % 4


class Cache:
    """The documented cache, codes and scales of keys and values."""

    def __init__(self, B, Hkv, cap, hd):
        self.shape = (B, Hkv, cap, hd)
        self.codes = [np.zeros((B, Hkv, cap, hd), np.uint8) for _ in range(2)]
        self.scales = [np.ones((B, Hkv, cap // 64)) for _ in range(2)]

    def append(self, k, v, lens, counts=None):
        B, Hkv, cap, hd = self.shape
        for which, x in enumerate((k, v)):
            T = x.shape[2]
            for b in range(B):
                n0 = int(lens[b])
                n = min(T, cap - n0) if 0 <= n0 < cap else 0
                if counts is not None:
                    n = min(n, int(counts[b]))
                if n <= 0:
                    continue
                for h in range(Hkv):
                    for blk in range(n0 // 64, (n0 + n - 1) // 64 + 1):
                        self._block(which, b, h, blk, x[b, h].astype(np.float64), n0, n)

    def _block(self, which, b, h, blk, x, n0, n):
        codes, scales = self.codes[which][b, h], self.scales[which][b, h]
        lo, hi = max(n0, blk * 64), min(n0 + n, blk * 64 + 64)
        new = x[lo - n0:hi - n0]
        fresh = lo == blk * 64
        if fresh:
            codes[blk * 64:blk * 64 + 64] = 0
        if not np.isfinite(new).all() or (not fresh and np.isnan(scales[blk])):
            scales[blk] = np.nan
            codes[lo:hi] = 0
            return
        s = 2.0 ** power_at_least(np.abs(new).max() / 448.0, -64)
        if not fresh:
            s = max(s, scales[blk])
            if s != scales[blk]:
                codes[blk * 64:lo] = self._codes(E4M3[codes[blk * 64:lo]] * (scales[blk] / s))
        scales[blk] = s
        codes[lo:hi] = self._codes(new / s)

    @staticmethod
    def _codes(v):
        return (nearest(np.abs(v), "fp8") | np.where(np.signbit(v), 128, 0)).astype(np.uint8)

    def buffers(self):
        """(key codes, key scales, value codes, value scales) as the device buffers hold them."""
        B, Hkv, cap, hd = self.shape
        out = []
        for which, index in enumerate((key_index(hd), value_index(hd))):
            c = np.zeros((B, Hkv, cap // 64, 64 * hd), np.uint8)
            c[..., index.reshape(-1)] = self.codes[which].reshape(B, Hkv, cap // 64, 64 * hd)
            out += [c, self.scales[which].astype(np.float32)]
        return out

    def values(self):
        return [E4M3[c] * np.repeat(s, 64, axis=2)[..., None] for c, s in zip(self.codes, self.scales)]


def attention(q, kv, lens, counts=None, window=0, sinks=0):
    """float64 [B, T, Hq, hd] and the rows that hold a token [B, T]; also the
    scale of the rounding of the probabilities: sqrt(sum (p v)^2) per output."""
    k, v = kv
    B, Hq, T, hd = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    out, spread = np.full((B, T, Hq, hd), np.nan), np.zeros((B, T, Hq, hd))
    there = np.zeros((B, T), bool)
    for b in range(B):
        for t in range(T):
            pos = int(lens[b]) + t
            if not 0 <= int(lens[b]) < cap or pos >= cap or (counts is not None and t >= counts[b]):
                continue
            there[b, t] = True
            j = np.arange(pos + 1)
            if window:
                j = j[(j > pos - window) | (j < sinks)]
            for h in range(Hq):
                kh = h * Hkv // Hq
                z = k[b, kh, j] @ q[b, h, t].astype(np.float64) / np.sqrt(hd)
                p = np.exp(z - z.max())
                p /= p.sum()
                out[b, t, h] = p @ v[b, kh, j]
                spread[b, t, h] = p @ np.abs(v[b, kh, j])
    return out, spread, there
