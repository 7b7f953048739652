"""The operators around a paged key/value cache, as cases that can be timed and
checked: the table of rotary angles, rotary positions, appending to the cache with
the rotation on the way, attention over it for ragged batches of prompts and single
tokens, and the same where the batch shares a long prefix.

Every case has a plain form in elementary torch operations on the layouts that
include/lmgc.h documents, and the call that a user makes.  Shapes are those of the
decoders this repository is built for (GPT-2 small, TinyLlama 1.1B, LLaMA-2 7B):
heads of 64 and 128 dims, with and without grouped key/value heads, windows of up to
4096 tokens, and generic longer ones.

Queries, keys and values are normal, keys and values with a magnitude of their own
for each head; pages lie in the pool in no order, and the places behind a sequence's
last token hold other sequences' stale numbers.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32  # tokens of a page whose keys (and values) lie in one piece


# ------------------------------------------------------------------- cases --
def listed():
    return [
        # a server's start: the angles of a 4096-token window, heads of 128
        dict(name="table_4096x128", kind="table", n=4096, rot=128, theta=1e4, scaling="none", factor=1.0, orig=4096),
        # the angles of a context stretched from 4096 to 131072 tokens
        dict(name="table_131072x128_yarn", kind="table", n=131072, rot=128, theta=1e4, scaling="yarn", factor=32.0, orig=4096),
        # one token of 8 windows (7B): queries and keys inside the QKV product's rows
        dict(name="rope_step_8x64x128", kind="rope", n=8, heads=64, hd=128, rot=128, dtype="bf16", layout="half",
             backward=False, gap=4096, table=4096),
        # a ragged batch of TinyLlama heads in float32, part of the head, neighbours paired, the gradient's direction
        dict(name="rope_8191x36x64_back", kind="rope", n=8191, heads=36, hd=64, rot=32, dtype="f32", layout="interleaved",
             backward=True, gap=0, table=8192),
        # a token for each of 32 windows of TinyLlama, into pages partly filled
        dict(name="append_step_32", kind="append", B=32, T=1, mix="all", len=2000, Hq=32, Hkv=4, hd=64, page=64, dtype="bf16",
             layout="half", rot=64, pad=0),
        # whole windows of the 7B shape into empty pages
        dict(name="append_prompt_4x4096", kind="append", B=4, T=4096, mix="all", len=0, Hq=32, Hkv=32, hd=128, page=128,
             dtype="bf16", layout="half", rot=128, pad=0),
        # a decoding step of 8 windows near the end of the 7B context
        dict(name="attn_step_8x4095", kind="attn", B=8, T=1, mix="all", len=4095, Hq=32, Hkv=32, hd=128, page=128, window=0,
             sinks=0, shared=0, pad=0),
        # a step of one TinyLlama window, grouped heads, behind a sliding window with four sinks
        dict(name="attn_step_window", kind="attn", B=1, T=1, mix="all", len=1500, Hq=32, Hkv=4, hd=64, page=32, window=512,
             sinks=4, shared=0, pad=0),
        # a served batch: a chunk of a prompt beside 15 windows at single tokens, rows left over behind them
        dict(name="attn_mixed_16x6000", kind="attn", B=16, T=509, mix="one", len=6000, Hq=32, Hkv=8, hd=128, page=64, window=0,
             sinks=0, shared=0, pad=3),
        # 2 ragged prompts behind tokens already in the cache, grouped heads
        dict(name="attn_prompt_2x3001", kind="attn", B=2, T=3001, mix="all", len=1000, Hq=32, Hkv=8, hd=128, page=128, window=0,
             sinks=0, shared=0, pad=0),
        # a decoding step of 32 windows behind one long instruction, a few hundred tokens of their own
        dict(name="shared_step_32x8192", kind="attn", B=32, T=1, mix="all", len=8700, Hq=32, Hkv=8, hd=128, page=64, window=0,
             sinks=0, shared=8192, pad=0),
        # short ragged prompts of 8 windows behind one instruction, a head of keys to each of queries
        dict(name="shared_prompt_8x150", kind="attn", B=8, T=150, mix="all", len=2011, Hq=12, Hkv=12, hd=64, page=32, window=0,
             sinks=0, shared=2000, pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["table", "rope", "rope", "append", "append", "attn", "attn", "attn", "shared", "shared"])
    if kind == "table":
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return dict(kind=kind, n=_log_int(rng, 16, 131072), rot=2 * _log_int(rng, 8, 64), theta=rng.choice([1e4, 5e5, 1e6]),
                    scaling=scaling, factor=1.0 if scaling == "none" else rng.uniform(1.5, 40.0), orig=_log_int(rng, 512, 8192))
    if kind == "rope":
        hd = rng.choice([32, 64, 80, 96, 128, 128, 256])
        heads = rng.choice([1, 4, 12, 24, 36, 64])
        n = _log_int(rng, 1, min(32768, (1 << 25) // (heads * hd)))
        return dict(kind=kind, n=n, heads=heads, hd=hd, rot=rng.choice([hd, hd, hd // 2, 2 * rng.randrange(1, hd // 2 + 1)]),
                    dtype=rng.choice(["f32", "bf16"]), layout=rng.choice(["half", "interleaved"]),
                    backward=rng.random() < 0.3, gap=rng.choice([0, 0, hd, 8 * hd, 6]), table=_log_int(rng, 64, 32768))
    hd = rng.choice([64, 128])
    page = rng.choice([32, 64, 128, 256])
    if kind == "append":
        Hkv = rng.choice([1, 4, 8, 12, 32])
        Hq = Hkv * rng.choice([1, 2, 4, 8]) if Hkv <= 8 else Hkv
        B = _log_int(rng, 1, 64)
        T = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, min(4096, (1 << 20) // (B * (Hq + 2 * Hkv)) * 64 // hd)))
        ln = rng.choice([0, _log_int(rng, 1, 4096)])
        return dict(kind=kind, B=B, T=T, mix=rng.choice(["all", "all", "one"]), len=ln, Hq=Hq, Hkv=Hkv, hd=hd, page=page,
                    dtype=rng.choice(["f32", "bf16", "bf16"]), layout=rng.choice(["half", "interleaved", "none"]),
                    rot=rng.choice([hd, hd, hd // 2, 2 * rng.randrange(1, hd // 2 + 1)]), pad=rng.choice([0, 0, 5]))
    Hkv = rng.choice([1, 4, 8, 12, 32])
    G = rng.choice([1, 2, 4, 8]) if Hkv <= 8 else 1
    shared = 0
    if kind == "shared":
        shared = _log_int(rng, 64, min(32768, (1 << 26) // (Hkv * hd)))
        B = _log_int(rng, 2, 64)
    else:
        B = _log_int(rng, 1, 64)
    ln = _log_int(rng, 1, max(2, min(131072, (1 << 26) // (B * Hkv * hd)))) + shared
    T = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, min(3000, (1 << 27) // (B * Hkv * G * (ln + 1000)))))
    window = rng.choice([0, 0, _log_int(rng, 16, ln + T)])
    return dict(kind="attn", B=B, T=T, mix=rng.choice(["all", "one"]) if T > 1 else "all", len=ln, Hq=Hkv * G, Hkv=Hkv, hd=hd,
                page=page, window=window, sinks=rng.choice([0, 4]) if window else 0, shared=shared, pad=rng.choice([0, 0, 7]))


def _seqs(case):
    """(new tokens, tokens there before) of each sequence: ragged, at most T and len."""
    out = []
    for b in range(case["B"]):
        T, n, s = case["T"], case["len"], case.get("shared", 0)
        if case["mix"] == "one":
            T = T if b == 0 else 1
        else:
            T = max(1, T - (53 * b) % (T // 4 + 1))
        out.append((T, max(s, n - (37 * b) % ((n - s) // 4 + 1))))
    return out


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rand(shape, g):
    return torch.randn(shape, generator=g, device=DEV)


def _angles(n, rot, theta=1e4):
    """(cos, sin) of n positions, float32 [n, rot / 2, 2]."""
    f = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _batch(case, st, g):
    """Rows, lengths and pages of a ragged batch, and a pool whose every place holds some number."""
    seqs, page = _seqs(case), case["page"]
    Hkv, hd, shared = case["Hkv"], case["hd"], case.get("shared", 0)
    st["seqs"] = seqs
    starts = [0]
    for T, _ in seqs:
        starts.append(starts[-1] + T)
    st["n"] = starts[-1] + case["pad"]
    st["starts"], st["lens"] = _ints(starts), _ints([n for _, n in seqs])
    st["max_new"] = max(T for T, _ in seqs)
    most = max(-(-(T + n) // page) for T, n in seqs)
    lead = shared // page  # whole pages that every sequence has in common
    n_pages = lead + sum(max(0, -(-(T + n) // page) - lead) for T, n in seqs) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    common, order = order[:lead], order[lead:]
    table = torch.full((case["B"], most), -1, dtype=torch.int32)
    for b, (T, n) in enumerate(seqs):
        own_pages = max(0, -(-(T + n) // page) - lead)
        mine, order = order[:own_pages], order[own_pages:]
        table[b, :lead + own_pages] = torch.tensor(common + mine, dtype=torch.int32)
    st["pages"] = table.to(DEV)
    mag = torch.exp(0.5 * _rand(Hkv, g))[:, None, None].to(torch.bfloat16)
    cache = []
    for _ in range(2):
        x = torch.empty((n_pages, Hkv, page, hd), dtype=torch.bfloat16, device=DEV)
        x.normal_(generator=g)
        cache.append(x.mul_(mag))
    # a shared prefix that ends inside a page: each sequence has those tokens on a page of its own
    part = shared % page
    if part:
        for x in cache:
            first = st["pages"][:, lead].long()
            src = x[first[0]].clone()
            for b in range(case["B"]):
                _copy_tokens(x, int(first[b]), src, part, x is cache[1])
    st["cache"] = tuple(cache)
    return seqs


def _copy_tokens(pool, page, src, n, values):
    """Tokens 0 .. n - 1 of one page's contents onto another page."""
    H, P, hd = src.shape
    take, place = (_take_v, _place_v) if values else (_take_k, _place_k)
    a, b = take(src[None]).clone(), take(pool[page][None]).clone()
    b[:, :, :n] = a[:, :, :n]
    pool[page] = place(b)[0].reshape(H, P, hd)


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)
    kind = case["kind"]
    if kind == "table":
        # other angles for another seed: the base moves by a little
        st["theta"] = case["theta"] * (1.0 + 1e-3 * (int(seed) % 1009))
    elif kind == "rope":
        n, H, hd = case["n"], case["heads"], case["hd"]
        wide = _rand((n, H * hd + case["gap"]), g).to(DTYPES[case["dtype"]])
        st["x"] = wide[:, :H * hd].unflatten(1, (H, hd))
        st["table"] = _angles(case["table"], case["rot"])
        first = torch.randint(case["table"], (1,), generator=g, device=DEV)
        st["positions"] = ((torch.arange(n, device=DEV) + first) % case["table"]).to(torch.int32)
    elif kind == "append":
        seqs = _batch(case, st, g)
        Hq, Hkv, hd = case["Hq"], case["Hkv"], case["hd"]
        # the QKV product's result
        qkv = _rand((st["n"], (Hq + 2 * Hkv) * hd), g).to(DTYPES[case["dtype"]]).unflatten(1, (Hq + 2 * Hkv, hd))
        st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st["q_out"] = torch.zeros((st["n"], Hq, hd), dtype=torch.bfloat16, device=DEV)
        if case["layout"] != "none":
            st["table"] = _angles(max(T + n for T, n in seqs), case["rot"])
    else:
        _batch(case, st, g)
        st["q"] = _rand((st["n"], case["Hq"], case["hd"]), g).to(torch.bfloat16)
        st["out"] = torch.zeros((st["n"], case["Hq"] * case["hd"]), dtype=torch.bfloat16, device=DEV)
        st["ws"] = torch.empty(512 << 20, dtype=torch.uint8, device=DEV)
    return st


# --------------------------------------------------------- layouts (lmgc.h) --
def _place_k(k):
    """[n, H, P, hd] -> the pool's order: groups of 32 tokens, blocks of 16 tokens x 32 dims."""
    n, H, P, hd = k.shape
    k = k.reshape(n, H, P // GROUP, 2, 16, hd // 32, 4, 8)
    return k.permute(0, 1, 2, 3, 5, 6, 4, 7).contiguous().reshape(n, H, P, hd)


def _take_k(k):
    n, H, P, hd = k.shape
    k = k.reshape(n, H, P // GROUP, 2, hd // 32, 4, 16, 8)
    return k.permute(0, 1, 2, 3, 6, 4, 5, 7).reshape(n, H, P, hd)


def _place_v(v):
    """blocks of 16 dims x 32 tokens; a dim's 8 numbers are tokens 4 g .. + 3 of both halves."""
    n, H, P, hd = v.shape
    v = v.reshape(n, H, P // GROUP, 2, 4, 4, hd // 16, 16)
    return v.permute(0, 1, 2, 6, 4, 7, 3, 5).contiguous().reshape(n, H, P, hd)


def _take_v(v):
    n, H, P, hd = v.shape
    v = v.reshape(n, H, P // GROUP, hd // 16, 4, 16, 2, 4)
    return v.permute(0, 1, 2, 6, 4, 7, 3, 5).reshape(n, H, P, hd)


# ---------------------------------------------------------------- plain form --
def _frequencies(theta, rot, scaling, factor, orig):
    """float64 [rot / 2], and what cos and sin are multiplied by."""
    i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** -i
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        keep = ((f * orig / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _rotate(x, rows, layout, backward=False):
    """x [n, heads, hd] float32, rows of the table [n, rot / 2, 2]."""
    rot = 2 * rows.shape[1]
    c, s = rows[:, None, :, 0], rows[:, None, :, 1]
    if backward:
        s = -s
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(st):
    """Every row at once: a row's sequence and position, then where its numbers are in the pools."""
    P, H, hd = st["page"], st["Hkv"], st["hd"]
    T = (st["starts"][1:] - st["starts"][:-1]).long()
    rows = sum(t for t, _ in st["seqs"])
    seq = torch.repeat_interleave(torch.arange(st["B"], device=DEV), T, output_size=rows)
    pos = torch.arange(rows, device=DEV) - st["starts"].long()[seq] + st["lens"].long()[seq]
    k, v, q = (st[x][:rows].float() for x in "kvq")
    if st["layout"] != "none":
        rot = st["table"][pos]
        k, q = _rotate(k, rot, st["layout"]), _rotate(q, rot, st["layout"])
        st["q_out"][:rows] = q.to(torch.bfloat16)
    first = (st["pages"].long()[seq, pos // P][:, None] * H + torch.arange(H, device=DEV)) * (P * hd)  # of a page's head
    index = torch.arange(P * hd, device=DEV).reshape(1, 1, P, hd)  # each place's own number, brought into the tokens' order
    for pool, x, take in zip(st["cache"], (k, v), (_take_k, _take_v)):
        at = take(index)[0, 0][pos % P]
        pool.view(-1)[first[..., None] + at[:, None]] = x.to(torch.bfloat16)
    return list(st["cache"]) + ([st["q_out"]] if st["layout"] != "none" else [])


def _plain_attention(st):
    Hq, H, hd = st["Hq"], st["Hkv"], st["hd"]
    G, row = Hq // H, 0
    for b, (T, n) in enumerate(st["seqs"]):
        L = n + T
        at = st["pages"][b, :-(-L // st["page"])].long()
        k = _take_k(st["cache"][0][at]).transpose(0, 1).reshape(H, -1, hd)[:, :L].float()
        v = _take_v(st["cache"][1][at]).transpose(0, 1).reshape(H, -1, hd)[:, :L].float()
        q = st["q"][row:row + T].float().reshape(T, H, G, hd).permute(1, 2, 0, 3).reshape(H, G * T, hd)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(hd)).reshape(H, G, T, L)
        pos = n + torch.arange(T, device=DEV)[:, None]
        j = torch.arange(L, device=DEV)
        see = j <= pos
        if st["window"]:
            see = see & ((j > pos - st["window"]) | (j < st["sinks"]))
        s.masked_fill_(~see, -math.inf)
        s = s.sub_(s.amax(-1, keepdim=True)).exp_()
        s = s.div_(s.sum(-1, keepdim=True))
        o = torch.matmul(s.reshape(H, G * T, L), v).reshape(H, G, T, hd)
        st["out"][row:row + T] = o.permute(2, 0, 1, 3).reshape(T, Hq * hd).to(torch.bfloat16)
        row += T
    return st["out"]


def _plain(st):
    kind = st["kind"]
    if kind == "table":
        f, m = _frequencies(st["theta"], st["rot"], st["scaling"], st["factor"], st["orig"])
        a = torch.arange(st["n"], dtype=torch.float64, device=DEV)[:, None] * f
        return (m * torch.stack([a.cos(), a.sin()], -1)).float()
    if kind == "rope":
        rows = st["table"][st["positions"].long()]
        return _rotate(st["x"].float(), rows, st["layout"], st["backward"]).to(st["x"].dtype)
    if kind == "append":
        return _plain_append(st)
    return _plain_attention(st)


# --------------------------------------------------------------------- calls --
def _call(st):
    from paper_2409_17836_amd import binding as B

    kind = st["kind"]
    if kind == "table":
        return B.rope_table(st["n"], st["rot"], st["theta"], st["scaling"], factor=st["factor"], orig=st["orig"])
    if kind == "rope":
        return B.op_rope(st["x"], st["positions"], st["table"], st["layout"], backward=st["backward"])
    if kind == "append":
        if st["layout"] == "none":
            B.op_paged_append(st["cache"], st["k"], st["v"], st["pages"], st["starts"], st["lens"])
            return list(st["cache"])
        B.op_paged_append(st["cache"], st["k"], st["v"], st["pages"], st["starts"], st["lens"], rope=st["table"],
                          layout=st["layout"], q=st["q"], q_out=st["q_out"])
        return list(st["cache"]) + [st["q_out"]]
    return B.op_attention_paged(st["q"], st["cache"], st["pages"], st["starts"], st["lens"], st["max_new"],
                                window=st["window"], sinks=st["sinks"], shared=st["shared"], out=st["out"], ws=st["ws"])


def run(st):
    if own:
        return _call(st)
    return _plain(st)


# -------------------------------------------------------------------- work --
def work(case):
    kind = case["kind"]
    if kind == "table":
        n = case["n"] * (case["rot"] // 2)
        return {"bytes": 8.0 * n, "flops": 60.0 * n}
    if kind == "rope":
        size = 4 if case["dtype"] == "f32" else 2
        n = case["n"] * case["heads"] * case["hd"]
        return {"bytes": 2.0 * size * n + 4.0 * case["n"] + 4.0 * case["rot"] * min(case["n"], case["table"]), "flops": 3.0 * n}
    seqs, hd, Hq, H = _seqs(case), case["hd"], case["Hq"], case["Hkv"]
    rows = sum(T for T, _ in seqs)
    if kind == "append":
        size = 4 if case["dtype"] == "f32" else 2
        heads = 2 * H + (Hq if case["layout"] != "none" else 0)
        return {"bytes": rows * heads * hd * (size + 2.0), "flops": 3.0 * rows * (heads - H) * hd}
    w, s, shared = case["window"], case["sinks"], case["shared"]
    pairs, keys, prefix = 0, 0, set()
    for T, n in seqs:
        if not w:
            pairs += T * n + T * (T + 1) // 2
            keys += n + T - shared
            prefix.add((0, shared))
            continue
        for t in range(T):
            p = n + t
            lo = max(0, p - w + 1)
            pairs += p + 1 - lo + min(s, lo)
        lo = max(0, n - w + 1)
        keys += n + T - max(lo, shared) + max(0, min(s, lo) - shared)
        prefix.add((min(lo, shared), shared))
    first = min(a for a, _ in prefix)
    keys += shared - first + min(s, first)
    return {"bytes": keys * H * hd * 4.0 + 4.0 * rows * Hq * hd, "flops": 4.0 * hd * Hq * pairs}


# ------------------------------------------------------------------- exact --
def _exact_table(case, theta):
    rot, s = case["rot"], case["factor"]
    freqs, m = [], 1.0
    for i in range(rot // 2):
        f = math.pow(theta, -2.0 * i / rot)
        if case["scaling"] == "linear":
            f /= s
        elif case["scaling"] == "ntk":
            f = math.pow(theta * math.pow(s, rot / (rot - 2.0)), -2.0 * i / rot)
        elif case["scaling"] == "yarn":
            turns = case["orig"] * f / (2.0 * math.pi)
            g = 0.0 if turns < 1.0 else 1.0 if turns > 32.0 else (turns - 1.0) / 31.0
            f = (1.0 - g) * f / s + g * f
            m = 0.1 * math.log(s) + 1.0
        freqs.append(f)
    out = torch.empty(case["n"], rot // 2, 2, dtype=torch.float64, device=DEV)
    p = torch.arange(case["n"], dtype=torch.float64, device=DEV)
    for i, f in enumerate(freqs):
        out[:, i, 0] = m * torch.cos(p * f)
        out[:, i, 1] = m * torch.sin(p * f)
    return out


def _exact_rotation(x, table, positions, layout, backward):
    """Pair by pair, in float64, as complex numbers."""
    y = x.double().clone()
    z = torch.view_as_complex(table.double().contiguous())[positions.long()]
    if backward:
        z = z.conj()
    rot = 2 * table.shape[1]
    i = torch.arange(rot // 2, device=DEV)
    re, im = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    w = torch.complex(y[..., re], y[..., im]) * z[:, None]
    y[..., re], y[..., im] = w.real, w.imag
    return y


def _places(P, hd):
    """Where key and value (t, d) of a page of P tokens are, by the formulas of the header."""
    t, d = torch.arange(P, device=DEV)[:, None], torch.arange(hd, device=DEV)[None, :]
    u, base = t % 32, (t // 32) * 32 * hd
    at_k = base + ((u // 16) * (hd // 32) + d // 32) * 512 + ((u % 16) + 16 * ((d % 32) // 8)) * 8 + d % 8
    at_v = base + (d // 16) * 512 + ((d % 16) + 16 * ((u % 16) // 4)) * 8 + 4 * (u // 16) + u % 4
    return at_k, at_v


def _exact_append(st):
    P, hd, H = st["page"], st["hd"], st["Hkv"]
    ats = _places(P, hd)
    out = [x.double() for x in st["cache"]]
    q_out = torch.zeros(st["n"], st["Hq"], hd, dtype=torch.float64, device=DEV)
    row = 0
    for b, (T, n) in enumerate(st["seqs"]):
        pos = n + torch.arange(T, device=DEV)
        k, v, q = (st[x][row:row + T].double() for x in "kvq")
        if st["layout"] != "none":
            k = _exact_rotation(k, st["table"], pos, st["layout"], False)
            q = _exact_rotation(q, st["table"], pos, st["layout"], False)
        q_out[row:row + T] = q
        where = st["pages"][b][pos // P].long()
        for pool, at, x in zip(out, ats, (k, v)):
            flat = pool.view(-1)
            for h in range(H):
                flat[((where * H + h) * (P * hd))[:, None] + at[pos % P]] = x[:, h]
        row += T
    return out + ([q_out] if st["layout"] != "none" else [])


def _exact_attention(st):
    P, hd, H, Hq = st["page"], st["hd"], st["Hkv"], st["Hq"]
    at_k, at_v = _places(P, hd)
    out = torch.zeros(st["n"], Hq, hd, dtype=torch.float64, device=DEV)
    row = 0
    for b, (T, n) in enumerate(st["seqs"]):
        L = n + T
        pages = st["pages"][b, :-(-L // P)].long()
        pos, j = (n + torch.arange(T, device=DEV))[:, None], torch.arange(L, device=DEV)[None, :]
        hid = j > pos
        if st["window"]:
            hid |= (j <= pos - st["window"]) & (j >= st["sinks"])
        for h in range(H):
            k = st["cache"][0][pages, h].reshape(len(pages), P * hd)[:, at_k].reshape(-1, hd)[:L].double()
            v = st["cache"][1][pages, h].reshape(len(pages), P * hd)[:, at_v].reshape(-1, hd)[:L].double()
            kt = k.T.contiguous()
            for i in range(h * Hq // H, (h + 1) * Hq // H):
                z = (st["q"][row:row + T, i].double() @ kt) / math.sqrt(hd)
                out[row:row + T, i] = torch.softmax(z.masked_fill(hid, -math.inf), -1) @ v
        row += T
    return out.reshape(st["n"], Hq * hd)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "table":
        return _exact_table(case, st["theta"])
    if kind == "rope":
        return _exact_rotation(st["x"], st["table"], st["positions"], case["layout"], case["backward"])
    if kind == "append":
        return _exact_append(st)
    return _exact_attention(st)
