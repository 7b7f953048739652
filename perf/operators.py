"""The operators of a decoder step held in fewer bits, as cases that can be timed
and checked: the residual add with RMSNorm and a microscaled output, microscaled
quantisation, the product with 4-bit weights, and the key/value cache in 8 bits
(appending to it, and attention over it, with a sliding window and first tokens
that stay visible).

Every case has a plain form in elementary torch operations on the layouts that
include/lmgc.h documents, and the call that a user makes.  Shapes are those of
the decoders this repository is built for (GPT-2 small, TinyLlama 1.1B, LLaMA-2
7B): d_model 768, 2048 and 4096, head dims 64 and 128, with and without grouped
key/value heads, windows of up to 4096 tokens.

Activations are normal with a few large channels, as a decoder's residual stream
has them; weights are N(0, 0.02); keys and values are normal with a magnitude of
their own for each head.
"""
import math

import torch

own = False
DEV = "cuda"
FP8_MAX, FP4_MAX = 448.0, 6.0
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------- cases --
def listed():
    return [
        # one token of one window in a TinyLlama step: the add and norm before a product
        dict(name="norm_step_1x2048", kind="norm", M=1, d=2048, h="f32", x="bf16", fmt="fp8"),
        # the same over a batch of 8 windows of 4096 tokens of a 7B layer
        dict(name="norm_prompt_32768x4096", kind="norm", M=32768, d=4096, h="f32", x="bf16", fmt="fp8"),
        # attention's output of a step of 8 windows before the O product (7B)
        dict(name="quantize_step_8x4096", kind="quantize", rows=8, cols=4096, src="bf16", fmt="fp8"),
        # a gate/up weight matrix of the 7B shape cast to 4 bits and read back
        dict(name="quantize_weights_22016x4096", kind="quantize", rows=22016, cols=4096, src="bf16", fmt="fp4"),
        # a decoding step of 8 windows: gate/up of the 7B shape, bound by the weights
        dict(name="gemm_step_8x22016x4096", kind="gemm", M=8, N=22016, K=4096, a="fp8", out="bf16"),
        # a short ragged prompt: TinyLlama's down product with the residual added
        dict(name="gemm_1000x2048x5632_add", kind="gemm", M=1000, N=2048, K=5632, a="fp4", out="add"),
        # a batch of 4 windows of 4096 tokens: QKV of the 7B shape, bound by the matrix cores
        dict(name="gemm_prompt_16384x12288x4096", kind="gemm", M=16384, N=12288, K=4096, a="fp8", out="bf16"),
        # one token for each of 32 windows of TinyLlama, into blocks partly filled
        dict(name="append_step_32", kind="append", B=32, Hkv=4, hd=64, T=1, len=2000, cap=2048),
        # whole windows of the 7B shape into an empty cache
        dict(name="append_prompt_4x4096", kind="append", B=4, Hkv=32, hd=128, T=4096, len=0, cap=4096),
        # a decoding step of 8 windows near the end of the 7B context
        dict(name="attn_step_8x4095", kind="attn", B=8, Hq=32, Hkv=32, hd=128, T=1, len=4095, cap=4096, window=0, sinks=0),
        # a step of one TinyLlama window, grouped heads, behind a sliding window with four sinks
        dict(name="attn_step_window", kind="attn", B=1, Hq=32, Hkv=4, hd=64, T=1, len=1500, cap=2048, window=512, sinks=4),
        # a prompt of 2 ragged windows behind tokens already in the cache, grouped heads
        dict(name="attn_prompt_2x3001", kind="attn", B=2, Hq=32, Hkv=8, hd=128, T=3001, len=1000, cap=4096, window=0, sinks=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "quantize", "gemm", "gemm", "append", "attn", "attn", "attn"])
    if kind == "norm":
        d = 32 * _log_int(rng, 2, 256)
        return dict(kind=kind, M=_log_int(rng, 1, min(32768, (1 << 27) // d)), d=d, h=rng.choice(["f32", "f32", "bf16"]),
                    x=rng.choice(["f32", "bf16"]), fmt=rng.choice(["fp8", "fp8", "fp4"]))
    if kind == "quantize":
        cols = _log_int(rng, 32, 11008)
        return dict(kind=kind, rows=_log_int(rng, 1, min(32768, 90_000_000 // cols)), cols=cols, src=rng.choice(["f32", "bf16"]),
                    fmt=rng.choice(["fp8", "fp4"]))
    if kind == "gemm":
        # widths and depths between a small decoder's and the 7B shape's, any multiple of 16
        N, K = 16 * _log_int(rng, 16, 2000), 32 * _log_int(rng, 4, 344)
        M = _log_int(rng, 1, max(2, min(32768, 800_000_000_000 // (N * K))))
        a = rng.choice(["fp8", "fp4"])
        return dict(kind=kind, M=M, N=N, K=K, a=a, out="bf16" if a == "fp8" else rng.choice(["bf16", "f32", "add"]))
    hd = rng.choice([64, 128])
    Hkv = rng.choice([4, 8, 12, 32])
    cap = 64 * _log_int(rng, 2, 64)
    if kind == "append":
        T = 1 if rng.random() < 0.5 else _log_int(rng, 1, cap)
        return dict(kind=kind, B=_log_int(rng, 1, max(1, min(32, (1 << 26) // (cap * Hkv * hd)))), Hkv=Hkv, hd=hd, T=T,
                    len=rng.randrange(0, cap - T + 1), cap=cap)
    G = rng.choice([1, 1, 2, 8])
    Hq = Hkv * G if Hkv * G <= 64 else Hkv
    T = 1 if rng.random() < 0.5 else _log_int(rng, 2, min(cap, 2048))
    most = max(1, min(32, (1 << 26) // (cap * Hkv * hd), (1 << 28) // (T * Hq * cap)))
    win = rng.choice([0, 0, _log_int(rng, 16, cap)])
    return dict(kind=kind, B=_log_int(rng, 1, most), Hq=Hq, Hkv=Hkv, hd=hd, T=T, len=rng.randrange(0, cap - T + 1), cap=cap,
                window=win, sinks=rng.choice([0, 4, 4]) if win else 0)


def _lens(case):
    """Tokens in the cache before the call, for each sequence: some shorter than the longest."""
    return [max(0, case["len"] - (37 * b) % (case["len"] // 4 + 1)) for b in range(case["B"])]


# --------------------------------------------------------- layouts (lmgc.h) --
def _up(n, m):
    return -(-n // m) * m


def _place_scales(sc, cols):
    """[rows, blocks of 32] -> [rows, 16 ceil(cols / 512)]: block j at byte 16 (j / 16) + 4 (j % 4) + (j % 16) / 4."""
    n = 16 * (-(-cols // 512))
    sc = torch.nn.functional.pad(sc, (0, n - sc.shape[1]))
    return sc.reshape(-1, n // 16, 4, 4).transpose(2, 3).reshape(-1, n).contiguous()


def _take_scales(sc, nblocks):
    return sc.reshape(sc.shape[0], -1, 4, 4).transpose(2, 3).reshape(sc.shape[0], -1)[:, :nblocks]


def _pack4(codes):
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def _block4(packed, scales):
    """Row-major 4-bit codes and scales -> blocks of 16 rows x 128 columns."""
    N = packed.shape[0]
    p = torch.nn.functional.pad(packed, (0, 0, 0, _up(N, 16) - N))
    s = torch.nn.functional.pad(scales, (0, 0, 0, _up(N, 16) - N))
    p = p.reshape(p.shape[0] // 16, 16, -1, 4, 16).permute(0, 2, 3, 1, 4).contiguous()
    s = s.reshape(s.shape[0] // 16, 16, -1, 4, 4).permute(0, 2, 3, 1, 4).contiguous()
    return p.reshape(-1), s.reshape(-1)


def _unblock4(p, s, N, K):
    Kp, n16 = _up(K, 128), _up(N, 16)
    p = p.reshape(n16 // 16, Kp // 128, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(n16, Kp // 2)
    s = s.reshape(n16 // 16, -1, 4, 16, 4).permute(0, 3, 1, 2, 4).reshape(n16, -1)
    return p[:N], s[:N]


def _place_k(k):
    """[B, Hkv, cap, hd] -> the cache's order of keys: 64 tokens, blocks of 16 tokens x 64 dims."""
    B, H, cap, hd = k.shape
    return k.reshape(B, H, cap // 64, 4, 16, hd // 64, 4, 16).permute(0, 1, 2, 3, 5, 6, 4, 7).contiguous().reshape(B, H, cap // 64, 64 * hd)


def _take_k(k, hd):
    B, H, n, _ = k.shape
    return k.reshape(B, H, n, 4, hd // 64, 4, 16, 16).permute(0, 1, 2, 3, 6, 4, 5, 7).reshape(B, H, n * 64, hd)


def _place_v(v):
    B, H, cap, hd = v.shape
    return v.reshape(B, H, cap // 64, 4, 4, 4, hd // 16, 16).permute(0, 1, 2, 6, 4, 7, 3, 5).contiguous().reshape(B, H, cap // 64, 64 * hd)


def _take_v(v, hd):
    B, H, n, _ = v.shape
    return v.reshape(B, H, n, hd // 16, 4, 16, 4, 4).permute(0, 1, 2, 6, 4, 7, 3, 5).reshape(B, H, n * 64, hd)


# -------------------------------------------------- microscaling, plain form --
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _scale_byte(amax, fmt):
    """Biased exponent of the smallest power of two s with amax <= max * s."""
    u = amax.contiguous().view(torch.int32)
    e, m = u >> 23, u & 0x7FFFFF
    big = (m > (0x600000 if fmt == "fp8" else 0x400000)).to(torch.int32)
    return (e - (8 if fmt == "fp8" else 2) + big).clamp_(min=0)


def _power(byte):
    """2^(byte - 127) in 32 bits."""
    return torch.where(byte > 0, byte << 23, torch.full_like(byte, 1 << 22)).view(torch.float32)


def _quantize(x, fmt):
    """float32 [rows, cols] -> (codes uint8 [rows, Kp(/ 2)], scale bytes uint8, both as lmgc.h places them)."""
    rows, cols = x.shape
    kp = _up(cols, 128)
    x = torch.nn.functional.pad(x, (0, kp - cols)).reshape(rows, kp // 32, 32)
    byte = _scale_byte(x.abs().amax(-1), fmt)
    v = (x * _power(254 - byte)[..., None]).reshape(rows, kp)
    if fmt == "fp8":
        codes = v.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        a = v.abs()
        c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
        codes = _pack4(c | (torch.signbit(v).to(torch.uint8) << 3))
    return codes, _place_scales(byte.to(torch.uint8), cols)


def _values(codes, scales, fmt, cols):
    """The values that codes and scales stand for, float32 [rows, cols]."""
    kp = _up(cols, 128)
    if fmt == "fp8":
        v = codes.view(torch.float8_e4m3fn).to(torch.float32)
    else:
        t = torch.tensor(_E2M1 + tuple(-e for e in _E2M1), device=codes.device)
        v = torch.stack([t[(codes & 15).long()], t[(codes >> 4).long()]], -1).reshape(codes.shape[0], kp)
    s = _power(_take_scales(scales, kp // 32).to(torch.int32))
    return (v.reshape(-1, kp // 32, 32) * s[..., None]).reshape(-1, kp)[:, :cols]


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _acts(rows, cols, g):
    x = torch.randn(rows, cols, generator=g, device=DEV)
    return x.mul_(1.0 + 4.0 * (torch.rand(cols, generator=g, device=DEV) < 0.02))


def _heads(case, T, g):
    """Keys or values of T tokens, bf16 [B, Hkv, T, hd]."""
    x = torch.randn(case["B"], case["Hkv"], T, case["hd"], generator=g, device=DEV)
    return x.mul_(torch.exp(0.5 * torch.randn(case["Hkv"], generator=g, device=DEV))[:, None, None]).to(torch.bfloat16)


def _kv_scale(amax):
    """The cache's block scale: the smallest power of two (2^-64 at least) with amax <= 448 * scale."""
    return _power(_scale_byte(amax, "fp8").clamp_(min=63))


def _full_cache(case, g):
    """A cache that holds len tokens of every sequence: codes and scales of keys and values."""
    B, H, hd, cap = case["B"], case["Hkv"], case["hd"], case["cap"]
    lens = torch.tensor(_lens(case), device=DEV)
    held = lens + (case["T"] if case["kind"] == "attn" else 0)
    there = torch.arange(cap, device=DEV)[None, :] < held[:, None]
    out = []
    for place in (_place_k, _place_v):
        x = _heads(case, cap, g).float() * there[:, None, :, None]
        s = _kv_scale(x.reshape(B, H, cap // 64, 64 * hd).abs().amax(-1))
        c = (x.reshape(B, H, cap // 64, 64 * hd) / s[..., None]).reshape(x.shape).to(torch.float8_e4m3fn).view(torch.uint8)
        out += [place(c), s]
    return out, lens.to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)
    kind = case["kind"]
    if kind == "norm":
        M, d = case["M"], case["d"]
        st["hin"] = _acts(M, d, g).to(DTYPES[case["h"]])
        st["xin"] = (0.3 * torch.randn(M, d, generator=g, device=DEV)).to(DTYPES[case["x"]])
        st["gain"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        st["sum"] = torch.empty_like(st["hin"])
    elif kind == "quantize":
        x = _acts(case["rows"], case["cols"], g)
        st["xin"] = (x if case["fmt"] == "fp8" else 0.02 * x).to(DTYPES[case["src"]])
    elif kind == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        st["ac"], st["as"] = _quantize(_acts(M, K, g), case["a"])
        st["bc"], st["bs"] = _block4(*_quantize(0.02 * torch.randn(N, K, generator=g, device=DEV), "fp4"))
        if case["out"] == "add":
            st["add"] = torch.randn(M, N, generator=g, device=DEV)
    else:
        st["cache"], st["lens"] = _full_cache(case, g)
        if kind == "append":
            st["kin"], st["vin"] = _heads(case, case["T"], g), _heads(case, case["T"], g)
        else:
            q = torch.randn(case["B"], case["Hq"], case["T"], case["hd"], generator=g, device=DEV)
            st["q"] = q.to(torch.bfloat16)
            st["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------- plain form --
def _plain_append(st):
    """Tokens lens[b] .. lens[b] + T - 1 of each sequence into the cache; a block's scale never falls."""
    B, H, hd, cap, T = st["B"], st["Hkv"], st["hd"], st["cap"], st["T"]
    kc, ks, vc, vs = st["cache"]
    lens = st["lens"].long()
    # every block that a new token falls into, of each sequence
    nb = (T + 62) // 64 + 1
    blk = (lens // 64)[:, None] + torch.arange(nb, device=DEV)[None, :]
    ok = (blk * 64 < (lens + T)[:, None]) & (blk < cap // 64)
    b, j = ok.nonzero(as_tuple=True)
    blk = blk[b, j]
    pos = blk[:, None] * 64 + torch.arange(64, device=DEV)[None, :]
    src = pos - lens[b][:, None]
    new, old = (src >= 0) & (src < T), src < 0
    fresh = blk * 64 >= lens[b]
    for new_x, codes, scales, place, take in ((st["kin"], kc, ks, _place_k, _take_k), (st["vin"], vc, vs, _place_v, _take_v)):
        x = new_x[b[:, None], :, src.clamp(0, T - 1)].transpose(1, 2).float() * new[:, None, :, None]
        n = x.shape[0]
        s_new = _kv_scale(x.reshape(n, H, -1).abs().amax(-1))
        s_old = scales[b, :, blk]
        s = torch.where(fresh[:, None], s_new, torch.maximum(s_new, s_old))
        # earlier tokens follow a grown scale; behind the new ones a new block is cleared, an old one left
        was = take(codes[b, :, blk].reshape(n, H, 1, 64 * hd), hd).contiguous().view(torch.float8_e4m3fn).float()
        was = torch.where(old[:, None, :, None], was * (s_old / s)[..., None, None], was) * ~fresh[:, None, None, None]
        c = torch.where(new[:, None, :, None], x / s[..., None, None], was).to(torch.float8_e4m3fn).view(torch.uint8)
        codes[b, :, blk] = place(c).reshape(n, H, 64 * hd)
        scales[b, :, blk] = s
    return _cache_out(st)


def _cache_out(st):
    kc, ks, vc, vs = st["cache"]
    return kc.view(torch.float8_e4m3fn), ks, vc.view(torch.float8_e4m3fn), vs


def _visible(case, lens):
    """[B, T, cap]: whether the query of new token t sees key j."""
    pos = (lens.long()[:, None] + torch.arange(case["T"], device=DEV)[None, :])[..., None]
    j = torch.arange(case["cap"], device=DEV)
    see = j <= pos
    if case["window"]:
        see = see & ((j > pos - case["window"]) | (j < case["sinks"]))
    return see


def _plain_attention(st):
    B, Hq, H, hd, T, cap = st["B"], st["Hq"], st["Hkv"], st["hd"], st["T"], st["cap"]
    kc, ks, vc, vs = st["cache"]
    k = _take_k(kc, hd).contiguous().view(torch.float8_e4m3fn).float().reshape(B, H, cap // 64, 64 * hd).mul_(ks[..., None])
    v = _take_v(vc, hd).contiguous().view(torch.float8_e4m3fn).float().reshape(B, H, cap // 64, 64 * hd).mul_(vs[..., None])
    k, v = k.reshape(B, H, cap, hd), v.reshape(B, H, cap, hd)
    G = Hq // H
    q = st["q"].float().reshape(B, H, G * T, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd)).reshape(B, H, G, T, cap)
    s.masked_fill_(~_visible(st, st["lens"])[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    s = s.div_(s.sum(-1, keepdim=True))
    o = torch.matmul(s.reshape(B, H, G * T, cap), v).reshape(B, Hq, T, hd)
    return o.permute(0, 2, 1, 3).reshape(B * T, Hq * hd).to(torch.bfloat16)


def _plain(st):
    kind = st["kind"]
    if kind == "norm":
        t = (st["hin"].float() + st["xin"].float()).to(st["hin"].dtype)
        x = t.float()
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * st["gain"].float()
        codes, scales = _quantize(y, st["fmt"])
        return _mx_out(t, codes, scales, st["fmt"], st["d"])
    if kind == "quantize":
        codes, scales = _quantize(st["xin"].float(), st["fmt"])
        return _mx_out(None, codes, scales, st["fmt"], st["cols"])
    if kind == "gemm":
        a = _values(st["ac"], st["as"], st["a"], st["K"])
        b = _values(*_unblock4(st["bc"], st["bs"], st["N"], st["K"]), "fp4", st["K"])
        c = torch.matmul(a, b.T)
        if st["out"] == "add":
            c += st["add"]
        return c.to(torch.bfloat16) if st["out"] == "bf16" else c
    if kind == "append":
        return _plain_append(st)
    return _plain_attention(st)


def _mx_out(t, codes, scales, fmt, cols):
    """8-bit codes as the numbers they are, with their scales; 4-bit ones as the values they stand for, in bf16."""
    if fmt == "fp8":
        out = [codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)]
    else:
        out = [_values(codes, scales, fmt, cols).to(torch.bfloat16)]
    return out if t is None else [t] + out


# --------------------------------------------------------------------- calls --
def _call(st):
    from paper_2409_17836_amd import binding as B

    kind = st["kind"]
    if kind in ("norm", "quantize"):
        t = None
        if kind == "norm":
            t = st["sum"]
            codes, scales = B.op_add_norm_mx(st["hin"], st["xin"], st["gain"], 1e-5, st["fmt"], out=t)
        else:
            codes, scales = B.op_mx_quantize(st["xin"], st["fmt"])
        if st["fmt"] == "fp8":
            out = [codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)]
        else:
            cols = st["d"] if kind == "norm" else st["cols"]
            out = [B.op_mx_dequantize(codes, scales, "fp4", cols, dtype=torch.bfloat16)]
        return out if t is None else [t] + out
    if kind == "gemm":
        return B.op_gemm_mx(st["ac"], st["as"], st["a"], st["bc"], st["bs"], st["N"], st["K"],
                            "bf16" if st["out"] == "bf16" else "store", add=st.get("add"))
    if kind == "append":
        B.op_kv8_append(st["cache"], st["kin"], st["vin"], st["lens"])
        return _cache_out(st)
    return B.op_attention_kv8(st["q"], st["cache"], st["lens"], window=st["window"], sinks=st["sinks"], ws=st["ws"])


def run(st):
    if own:
        return _call(st)
    return _plain(st)


# -------------------------------------------------------------------- work --
def _mx_bytes(rows, cols, fmt):
    return rows * cols * ((1.0 if fmt == "fp8" else 0.5) + 1.0 / 32)


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, size = case["M"] * case["d"], {"f32": 4, "bf16": 2}
        out = _mx_bytes(case["M"], case["d"], "fp8") if case["fmt"] == "fp8" else 2.0 * n
        return {"bytes": n * (2.0 * size[case["h"]] + size[case["x"]]) + 2.0 * case["d"] + out, "flops": 6.0 * n}
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        out = _mx_bytes(case["rows"], case["cols"], "fp8") if case["fmt"] == "fp8" else 2.0 * n
        return {"bytes": n * (4.0 if case["src"] == "f32" else 2.0) + out, "flops": 3.0 * n}
    if kind == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        out = {"bf16": 2.0, "f32": 4.0, "add": 8.0}[case["out"]]
        return {"bytes": _mx_bytes(M, K, case["a"]) + _mx_bytes(N, K, "fp4") + out * M * N, "flops": 2.0 * M * N * K}
    lens, T, hd, H = _lens(case), case["T"], case["hd"], case["Hkv"]
    if kind == "append":
        return {"bytes": len(lens) * H * T * hd * 2 * 3.0, "flops": 2.0 * len(lens) * H * T * hd * 2}
    pairs = keys = 0
    for n in lens:
        w, s = case["window"], case["sinks"]
        if not w:
            pairs += T * n + T * (T + 1) // 2
            keys += n + T
            continue
        for t in range(T):
            p = n + t
            lo = max(0, p - w + 1)
            pairs += p + 1 - lo + min(s, lo)
        lo = max(0, n - w + 1)
        keys += n + T - lo + min(s, lo)
    return {"bytes": keys * H * hd * 2.0 + 4.0 * len(lens) * case["Hq"] * T * hd, "flops": 4.0 * hd * case["Hq"] * pairs}


# ------------------------------------------------------------------- exact --
def _two64(e):
    """2^e in float64, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _grid64(x, top, low, bits):
    """float64 values rounded to the nearest number with `bits` fraction bits and exponents from `low`, half to even."""
    e = torch.frexp(x)[1] - 1
    step = _two64(e.clamp(min=low) - bits)
    return (torch.round(x / step) * step).clamp(-top, top)


def _mx64(x, fmt):
    """(numbers on the format's grid [rows, Kp], scales [rows, Kp / 32]) of float64 [rows, cols]."""
    top, low, bits = (FP8_MAX, -6, 3) if fmt == "fp8" else (FP4_MAX, 0, 1)
    rows, cols = x.shape
    kp = -(-cols // 128) * 128
    z = torch.zeros(rows, kp, dtype=torch.float64, device=DEV)
    z[:, :cols] = x
    z = z.view(rows, -1, 32)
    m, e = torch.frexp(z.abs().max(-1).values / top)  # in [1/2, 1) x 2^e: the power of two at or above it
    e = torch.where(m == 0.5, e - 1, e)
    s = _two64(torch.where(m == 0, -127, e).clamp(min=-127))
    return _grid64(z / s[..., None], top, low, bits).reshape(rows, kp), s


def _mx64_out(x, fmt):
    cols = x.shape[1]
    n, s = _mx64(x, fmt)
    if fmt == "fp8":
        # scales where the bytes are: 16 to 512 columns, the others 2^-127
        out = torch.full((x.shape[0], 16 * (-(-cols // 512))), 2.0 ** -127, dtype=torch.float64, device=DEV)
        j = torch.arange(s.shape[1], device=DEV)
        out[:, 16 * (j // 16) + 4 * (j % 4) + (j % 16) // 4] = s
        return [n, out]
    return [(n.view(n.shape[0], -1, 32) * s[..., None]).reshape(n.shape)[:, :cols]]


def _cache64(st):
    """The cache's numbers in float64, and where key and value (t, d) of a block of 64 tokens are."""
    hd = st["hd"]
    t, d = torch.arange(64, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    at_k = ((t // 16) * (hd // 64) + d // 64) * 1024 + ((t % 16) + 16 * ((d % 64) // 16)) * 16 + d % 16
    at_v = (d // 16) * 1024 + ((d % 16) + 16 * ((t % 16) // 4)) * 16 + (t // 16) * 4 + t % 4
    return [c.double() if c.dtype != torch.uint8 else c.view(torch.float8_e4m3fn).double() for c in st["cache"]], at_k, at_v


def _append64(st):
    """Sequence by sequence, in float64."""
    (kc, ks, vc, vs), at_k, at_v = _cache64(st)
    for codes, scales, at, x in ((kc, ks, at_k, st["kin"]), (vc, vs, at_v, st["vin"])):
        for b, n in enumerate(_lens(st)):
            first, last = n // 64, (n + st["T"] - 1) // 64
            was = codes[b, :, first:last + 1][:, :, at].flatten(1, 2)  # [Hkv, tokens, hd]
            s0 = scales[b, :, first:last + 1].clone()
            val = torch.zeros_like(was)
            val[:, :n % 64] = was[:, :n % 64] * s0[:, :1, None]
            val[:, n % 64:n % 64 + st["T"]] = x[b].double()
            top = val.clone()
            top[:, :n % 64] = 0
            m, e = torch.frexp(top.unflatten(1, (-1, 64)).abs().amax((2, 3)) / FP8_MAX)
            s = _two64(torch.where(m == 0, -64, torch.where(m == 0.5, e - 1, e)).clamp(min=-64))
            if n % 64:
                s[:, 0] = torch.maximum(s[:, 0], s0[:, 0])
            num = _grid64(val.unflatten(1, (-1, 64)) / s[..., None, None], FP8_MAX, -6, 3)
            if n % 64 and n % 64 + st["T"] < 64:
                num[:, 0, n % 64 + st["T"]:] = was[:, n % 64 + st["T"]:]
            part = codes[b, :, first:last + 1]
            part[:, :, at.flatten()] = num.flatten(2)
            scales[b, :, first:last + 1] = s
    return kc, ks, vc, vs


def _attention64(st):
    """Head by head, in float64."""
    B, Hq, H, hd, T, cap = st["B"], st["Hq"], st["Hkv"], st["hd"], st["T"], st["cap"]
    (kc, ks, vc, vs), at_k, at_v = _cache64(st)
    out = torch.empty(B, T, Hq, hd, dtype=torch.float64, device=DEV)
    j = torch.arange(cap, device=DEV)
    for b, n in enumerate(_lens(st)):
        pos = (n + torch.arange(T, device=DEV))[:, None]
        hid = j[None, :] > pos
        if st["window"]:
            hid |= (j[None, :] <= pos - st["window"]) & (j[None, :] >= st["sinks"])
        for h in range(Hq):
            i = h * H // Hq
            k = (kc[b, i][:, at_k] * ks[b, i][:, None, None]).reshape(cap, hd)
            v = (vc[b, i][:, at_v] * vs[b, i][:, None, None]).reshape(cap, hd)
            z = (st["q"][b, h].double() @ k.T) / math.sqrt(hd)
            out[b, :, h] = torch.softmax(z.masked_fill(hid, -math.inf), -1) @ v
    return out.reshape(B * T, Hq * hd)


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    if kind == "append":
        return _append64(st)
    if kind == "norm":
        t = st["hin"].double() + st["xin"].double()
        x = t.to(st["hin"].dtype).double()
        r = 1.0 / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + 1e-5)
        return [t] + _mx64_out(x * r * st["gain"].double(), case["fmt"])
    if kind == "quantize":
        return _mx64_out(st["xin"].double(), case["fmt"])
    if kind == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        if 2.0 * M * N * K > 4e12:
            return None
        num = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)

        def nibbles(c):
            c = torch.stack([c % 16, c // 16], -1).flatten(-2).long()
            return num[c % 8] * (1.0 - 2.0 * (c // 8))

        kb, ns = -(-K // 128), -(-K // 512)
        k = torch.arange(K, device=DEV)
        # where the scale of column k sits in a row of scales
        at = 16 * (k // 512) + 4 * ((k // 32) % 4) + (k % 512) // 128
        a = st["ac"].view(torch.float8_e4m3fn).double() if case["a"] == "fp8" else nibbles(st["ac"])
        a = a[:, :K] * _two64(st["as"].long() - 127)[:, at]
        n = torch.arange(N, device=DEV)[:, None]
        w = nibbles(st["bc"].view(-1, 16))  # pieces of 32 columns of a row
        piece = ((n // 16) * kb + torch.arange(kb * 4, device=DEV) // 4) * 64 + n % 16 + 16 * (torch.arange(kb * 4, device=DEV) % 4)
        w = w[piece].reshape(N, kb * 128)[:, :K]
        ws = _two64(st["bs"].long() - 127)
        w *= ws[((n // 16) * ns + k // 512) * 256 + (n % 16 + 16 * ((k // 32) % 4)) * 4 + (k % 512) // 128]
        c = a @ w.T
        return c + st["add"].double() if case["out"] == "add" else c
    return _attention64(st)
