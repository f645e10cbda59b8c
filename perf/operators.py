"""What runs between the projections and the attention of a token, as cases that can be timed and compared: rotary
positions, the 8-bit key/value cache, and attention over it.

    rotate   rotary positions of the queries and keys of n tokens
    append   keys and values of n tokens into the 8-bit cache
    decode   one generated token over the prompt's sparse index, keys and values out of the cache
    attend   the n newest tokens over everything the cache holds, causal

The cache keeps blocks of `block` tokens.  A full block has, for each key/value head, one scale that is a power of two
(the least that brings the block's largest magnitude into the range of the type) and codes of 8 bits; the tokens behind
the last full block stay in bf16.  `run` computes each operator in its plain form, or calls the library where `own` is set.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
LEAST_EXPONENT = -100  # of a scale


# -------------------------------------------------------------------------------------------- cases
def listed():
    base = {"hq": 32, "hkv": 8, "block": 64, "type": "e4m3"}
    plain = {"layout": "half", "dim": 128, "scaling": "none", "transposed": False, "packed": False}
    return [
        # the query and key of one generated token, at a long position under a wavelength scaling
        dict(base, name="rotate-1", kind="rotate", n=1, pos=131772, **dict(plain, scaling="wavelength")),
        # several prompts packed into one call (positions start again), half of each head, neighbours paired
        dict(base, name="rotate-10k-packed", kind="rotate", n=10304, pos=0,
             **dict(plain, layout="interleaved", dim=64, scaling="linear", packed=True)),
        # the gradient of a training sequence
        dict(base, name="rotate-16k-transposed", kind="rotate", n=16384, pos=0, **dict(plain, scaling="base", transposed=True)),
        # the longest prompt of the benchmark
        dict(base, name="rotate-128k", kind="rotate", n=131072, pos=0, **dict(plain, scaling="ramp")),
        # a generated token that fills its block, the dearest of a block's steps
        dict(base, name="append-1", kind="append", n=1, pos=32831),
        # a prompt that ends in the middle of a block, wide-range codes
        dict(base, name="append-10k-ragged", kind="append", n=10341, pos=0, block=128, type="e5m2"),
        # the longest prompt
        dict(base, name="append-128k", kind="append", n=131072, pos=0, block=128),
        # a generated token after a short and after the longest prompt
        dict(base, name="decode-4k", kind="decode", hq=8, hkv=2, n=4096, generated=1, keep=0.10),
        dict(base, name="decode-128k", kind="decode", n=131072, generated=700, keep=0.03, block=128),
        # a generated token without an index
        dict(base, name="attend-1-128k", kind="attend", n=1, pos=131771, block=128),
        # drafted tokens checked at once, one key/value head
        dict(base, name="attend-5-10k", kind="attend", hq=8, hkv=1, n=5, pos=10303, type="e5m2"),
        # a further turn of 2K tokens at the end of 64K
        dict(base, name="attend-2k-64k", kind="attend", n=2048, pos=63488),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "decode", "attend", "attend"])
    hq, hkv = rng.choice([(4, 4), (8, 8), (8, 2), (6, 2), (8, 1), (16, 4), (24, 3), (32, 8), (32, 8)])
    block = rng.choice([64, 128])
    c = {"kind": kind, "hq": hq, "hkv": hkv, "block": block, "type": rng.choice(["e4m3", "e4m3", "e5m2"])}
    if kind == "rotate":
        c.update(n=_log_int(rng, 1, 131072), pos=_log_int(rng, 1, 131072) - 1, layout=rng.choice(["half", "interleaved"]),
                 dim=rng.choice([128, 128, 128, 64, 32, 96, 36]), scaling=rng.choice(["none", "linear", "base", "wavelength", "ramp"]),
                 transposed=rng.random() < 0.3, packed=rng.random() < 0.3)
    elif kind == "append":
        n, pos = _log_int(rng, 1, 131072), _log_int(rng, 1, 131072) - 1
        if pos % block + n > block:  # a pass that can be made again: it does not write over the open rows that it reads
            pos -= pos % block
        c.update(n=n, pos=pos)
    elif kind == "decode":
        n = max(8, _log_int(rng, 1024, 131072) // block) * block
        c.update(n=n, generated=_log_int(rng, 1, 2000), keep=round(min(0.5, max(0.01, _log_int(rng, 400, min(4000, n)) / n)), 4))
    else:
        n = _log_int(rng, 1, 2048)
        c.update(n=n, pos=min(_log_int(rng, 1, 131072) - 1, 2048 * 65536 * 32 // (hq * n) - n))
    return c


# ------------------------------------------------------------------------------------------- inputs
def _full(tokens, block):
    """Tokens in full blocks."""
    return tokens // block * block


def _values(gen, *shape):
    """Keys or values as projections give them: N(0,1) with a few dimensions of larger spread."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x[..., 5::32] *= 4.0
    return x.bfloat16()


def _quantise(x, block, kind):
    """Codes [heads, n, 128] and scales [heads, n / block] of full blocks."""
    heads, n = x.shape[:2]
    b = x.float().view(heads, n // block, block * D)
    top = b.abs().amax(-1)
    m, e = torch.frexp(top / LARGEST[kind])  # top / largest = m 2^e with m in [0.5, 1)
    e = torch.where(top > 0, e - (m == 0.5).int(), 0).clamp(min=LEAST_EXPONENT)
    s = (e + 127 << 23).view(torch.float32)  # 2^e
    return (b / s[..., None]).to(CODES[kind]).view(heads, n, D), s


def _cache(case, tokens, capacity, gen):
    """The cache after `tokens` tokens."""
    hkv, block, kind = case["hkv"], case["block"], case["type"]
    c = {"capacity": capacity}
    for name in ("k", "v"):
        x = _values(gen, hkv, max(tokens, 1), D)[:, :tokens]
        codes = torch.zeros((hkv, capacity, D), dtype=torch.uint8, device="cuda")
        scale = torch.zeros((hkv, capacity // block), dtype=torch.float32, device="cuda")
        rows = torch.zeros((hkv, block, D), dtype=torch.bfloat16, device="cuda")
        full = _full(tokens, block)
        if full:
            q, s = _quantise(x[:, :full].contiguous(), block, kind)
            codes[:, :full] = q.view(torch.uint8)
            scale[:, :full // block] = s
        rows[:, :tokens - full] = x[:, full:]
        c.update({name: codes, name + "_scale": scale, name + "_open": rows})
    return c


def _budgets(case):
    """The sizes that the library suggests for a keep fraction."""
    n, nb, keep = case["n"], case["n"] // case["block"], case["keep"]
    blocks = max(nb, int(keep * (nb * (nb + 1) // 2) + 0.5))
    local = max([1] + [x for x in range(1, nb + 1) if x * nb - x * (x - 1) // 2 + (nb - x) <= blocks])
    return {"sink_blocks": 1, "local_blocks": local, "k_blocks": blocks, "k_slash": min(n, max(1, int(keep * n / 128 + 0.5))),
            "k_vertical": min(n, 64 * max(1, int(keep * n / 256 + 0.5)))}


def _kept(case):
    """Per query head: key blocks of the last row block, columns, diagonals."""
    b, nb = _budgets(case), case["n"] // case["block"]
    share = min(nb, -(-2 * b["k_blocks"] // (nb + 1)))
    kinds = [(min(nb, 1 + b["local_blocks"]), 0, 0), (1, b["k_vertical"], b["k_slash"]), (1, b["k_vertical"], b["k_slash"]), (share, 0, 0)]
    return [kinds[h % 4] for h in range(case["hq"])]


def _index(case, gen):
    """An index in the library's layout, with the last row block's keys as the four kinds of heads keep them."""
    b, n, nb, hq = _budgets(case), case["n"], case["n"] // case["block"], case["hq"]
    band = sum(min(1, max(0, r - b["local_blocks"] + 1)) + min(r + 1, b["local_blocks"]) for r in range(nb))
    i32 = {"dtype": torch.int32, "device": "cuda"}
    ix = {"pattern": torch.tensor([[0, 1, 1, 2][h % 4] for h in range(hq)], **i32),
          "n_cols": torch.zeros(hq, **i32), "cols": torch.full((hq, b["k_vertical"]), -1, **i32),
          "n_offs": torch.zeros(hq, **i32), "offs": torch.full((hq, b["k_slash"]), -1, **i32),
          "rowptr": torch.zeros((hq, nb + 1), **i32), "blkcols": torch.full((hq, max(band, b["k_blocks"])), -1, **i32)}

    def some(count, top):
        return torch.sort(torch.randperm(top, generator=gen, device="cuda")[:count])[0].int()

    for h, (blocks, cols, offs) in enumerate(_kept(case)):
        chosen = some(blocks - 1, nb - 1)
        if h % 4 == 0:  # sink and band
            chosen = torch.arange(nb - blocks, nb - 1, **i32)
            chosen[:1] = 0
        ix["blkcols"][h, :blocks - 1] = chosen
        ix["blkcols"][h, blocks - 1] = nb - 1
        ix["rowptr"][h, nb] = blocks
        ix["n_cols"][h], ix["n_offs"][h] = cols, offs
        ix["cols"][h, :cols] = some(cols, n)
        ix["offs"][h, :offs] = some(offs, n)
    return ix


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, n, block, kind = case["hq"], case["hkv"], case["n"], case["block"], case["kind"]
    s = {"case": dict(case)}
    if kind == "rotate":
        s["q"] = torch.randn((hq, n, D), generator=gen, device="cuda").bfloat16()
        s["k"] = torch.randn((hkv, n, D), generator=gen, device="cuda").bfloat16()
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["positions"] = None
        if case["packed"]:
            start = torch.randint(0, 1021, (1,), generator=gen, device="cuda")
            s["positions"] = ((torch.arange(n, device="cuda") + start) % 1021 + case["pos"]).int()
    elif kind == "append":
        s["cache"] = _cache(case, case["pos"], _full(case["pos"] + n + block - 1, block), gen)
        s["k"], s["v"] = _values(gen, hkv, n, D), _values(gen, hkv, n, D)
    else:
        tokens = n + case["generated"] if kind == "decode" else case["pos"] + n
        s["cache"] = _cache(case, tokens, _full(tokens + block - 1, block), gen)
        s["q"] = torch.randn((hq, D) if kind == "decode" else (hq, n, D), generator=gen, device="cuda").bfloat16()
        s["o"] = torch.empty_like(s["q"])
        if kind == "decode":
            s["index"] = _index(case, gen)
    return s


# -------------------------------------------------------------------------------------- plain forms
SCALINGS = {  # base, and what the scaling goes by
    "none": (10000.0, {}),
    "linear": (10000.0, {"factor": 4.0}),
    "base": (10000.0, {"factor": 8.0}),
    "wavelength": (500000.0, {"factor": 8.0, "low": 1.0, "high": 4.0, "original_len": 8192}),
    "ramp": (1000000.0, {"factor": 4.0, "low": 1.0, "high": 32.0, "original_len": 32768}),
}


def _frequencies(case):
    """Radians per token of each pair, in 64 bits, and what sine and cosine are multiplied with."""
    dim, (theta, p) = case["dim"], SCALINGS[case["scaling"]]
    i = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    if case["scaling"] == "base" and dim > 2:
        theta *= p["factor"] ** (dim / (dim - 2))
    w = theta ** (-2 * i / dim)
    if case["scaling"] == "linear":
        return w / p["factor"], 1.0
    if case["scaling"] == "wavelength":
        t = ((p["original_len"] * w / (2 * math.pi) - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        return (1 - t) * w / p["factor"] + t * w, 1.0
    if case["scaling"] == "ramp":
        lo, hi = [dim * math.log(p["original_len"] / (x * 2 * math.pi)) / (2 * math.log(theta)) for x in (p["high"], p["low"])]
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), dim - 1)
        t = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return w * (1 - t) + w / p["factor"] * t, 0.1 * math.log(p["factor"]) + 1.0
    return w, 1.0


def _rotate(state):
    case = state["case"]
    dim, n = case["dim"], case["n"]
    pos = state["positions"] if case["packed"] else torch.arange(case["pos"], case["pos"] + n, device="cuda")
    w, amplitude = _frequencies(case)
    angle = pos.double()[:, None] * w
    c = (torch.cos(angle) * amplitude).float()
    s = (torch.sin(angle) * (-amplitude if case["transposed"] else amplitude)).float()

    def turn(x):
        x = x.float()
        r = x[..., :dim]
        if case["layout"] == "half":
            a, b = r[..., :dim // 2], r[..., dim // 2:]
            y = torch.cat([a * c - b * s, a * s + b * c], -1)
        else:
            a, b = r[..., 0::2], r[..., 1::2]
            y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
        return torch.cat([y, x[..., dim:]], -1).bfloat16()

    return [turn(state["q"]), turn(state["k"])]


def _append(state):
    case, cache = state["case"], state["cache"]
    pos, n, block = case["pos"], case["n"], case["block"]
    first, full = _full(pos, block), _full(pos + n, block)
    for name in ("k", "v"):
        rows = cache[name + "_open"]
        x = torch.cat([rows[:, :pos - first], state[name]], 1)  # from the open block's first token on
        if full > first:
            q, s = _quantise(x[:, :full - first].contiguous(), block, case["type"])
            cache[name][:, first:full] = q.view(torch.uint8)
            cache[name + "_scale"][:, first // block:full // block] = s
        lo = max(full, pos)
        rows[:, lo - full:pos + n - full] = x[:, lo - first:]
    return _contents(state)


def _contents(state):
    """What the cache holds, codes as the values they stand for (before the scale)."""
    c, kind = state["cache"], CODES[state["case"]["type"]]
    return [c["k"].view(kind), c["v"].view(kind), c["k_scale"], c["v_scale"], c["k_open"], c["v_open"]]


def _read(state, name, tokens):
    """Keys or values [hkv, tokens, 128] of the cache in fp32."""
    cache, case = state["cache"], state["case"]
    full, block = _full(tokens, case["block"]), case["block"]
    x = cache[name][:, :full].view(CODES[case["type"]]).float().view(case["hkv"], full // block, block * D)
    x = (x * cache[name + "_scale"][:, :full // block, None]).view(case["hkv"], full, D)
    return torch.cat([x, cache[name + "_open"][:, :tokens - full].float()], 1)


def _attention(state, q, keep, tokens):
    """q [hkv, rows, 128] over the cache, keep broadcast to [hkv, rows, tokens]; a row keeps one key at least."""
    s = torch.matmul(q, _read(state, "k", tokens).transpose(1, 2))
    s.mul_(D ** -0.5).masked_fill_(~keep, -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    return torch.matmul(s, _read(state, "v", tokens)) / s.sum(-1, keepdim=True)


def _decode(state):
    case, ix = state["case"], state["index"]
    n, pos, hq, hkv, block = case["n"], case["n"] + case["generated"] - 1, case["hq"], case["hkv"], case["block"]
    nb, tokens = n // block, pos + 1
    j = torch.arange(tokens, device="cuda")
    # one place more than tokens takes what the padding of the lists points at
    blocks = torch.zeros((hq, nb + 1), dtype=torch.bool, device="cuda")
    e = torch.arange(ix["blkcols"].shape[1], device="cuda")
    inside = (e >= ix["rowptr"][:, nb - 1, None]) & (e < ix["rowptr"][:, nb, None])
    blocks.scatter_(1, torch.where(inside & (ix["blkcols"] >= 0), ix["blkcols"], nb).long(), True)
    blocks[:, nb] = False
    single = torch.zeros((hq, tokens + 1), dtype=torch.bool, device="cuda")
    single.scatter_(1, torch.where(ix["cols"] >= 0, ix["cols"], tokens).long(), True)
    single.scatter_(1, torch.where(ix["offs"] >= 0, pos - ix["offs"], tokens).long(), True)
    keep = (j >= n) | single[:, :tokens] | blocks[:, torch.clamp(j // block, max=nb)]
    o = _attention(state, state["q"].float().view(hkv, hq // hkv, D), keep.view(hkv, hq // hkv, tokens), tokens)
    return o.view(hq, D).bfloat16()


def _attend(state):
    case = state["case"]
    hq, hkv, n, pos = case["hq"], case["hkv"], case["n"], case["pos"]
    keep = torch.arange(pos + n, device="cuda") <= torch.arange(pos, pos + n, device="cuda").repeat(hq // hkv)[:, None]
    o = _attention(state, state["q"].float().view(hkv, hq // hkv * n, D), keep, pos + n)
    return o.view(hq, n, D).bfloat16()


# ------------------------------------------------------------------------------- the library's calls
_sessions = {}


def _session(case):
    """One session per shape, as a serving program keeps it for all its layers."""
    n = case["n"] if case["kind"] == "decode" else 1024
    more = _budgets(case) if case["kind"] == "decode" else {"keep": 0.1}
    key = (case["hq"], case["hkv"], n, case["block"]) + tuple(sorted(more.items()))
    if key not in _sessions:
        import paper_2412_06198_amd as sa

        _sessions[key] = sa.Session(case["hq"], case["hkv"], n, case["block"], 64, **more)
    return _sessions[key]


def _handles(state):
    """The session, and what a program keeps beside it: the rotation's frequencies, the cache, the index."""
    if "handles" not in state:
        import paper_2412_06198_amd as sa

        case = state["case"]
        h = {"session": _session(case)}
        if case["kind"] == "rotate":
            theta, more = SCALINGS[case["scaling"]]
            layout = sa.SA_ROTARY_HALF if case["layout"] == "half" else sa.SA_ROTARY_INTERLEAVED
            scaling = getattr(sa, "SA_SCALING_" + case["scaling"].upper())
            h["rotary"] = sa.Rotary(rotary_dim=case["dim"], layout=layout, scaling=scaling, theta=theta,
                                    transposed=int(case["transposed"]), **more)
        else:
            c = state["cache"]
            h["cache"] = sa.Cache(c["k"], c["v"], c["k_scale"], c["v_scale"], c["k_open"], c["v_open"],
                                  sa.SA_CACHE_E4M3 if case["type"] == "e4m3" else sa.SA_CACHE_E5M2)
        if case["kind"] == "decode":
            names = ("pattern", "n_cols", "cols", "n_offs", "offs", "rowptr", "blkcols")
            h["index"] = sa.SaIndex(*[state["index"][x].data_ptr() for x in names])
            h["decode"] = sa.sa_cache_decode
        state["handles"] = h
    return state["handles"]


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"rotate": _rotate, "append": _append, "decode": _decode, "attend": _attend}[kind](state)
    h = _handles(state)
    ses = h["session"]
    if kind == "rotate":
        ses.rotate(h["rotary"], state["q"], state["k"], state["q_out"], state["k_out"], pos=case["pos"], positions=state["positions"])
        return [state["q_out"], state["k_out"]]
    if kind == "append":
        ses.append(h["cache"], state["k"], state["v"], case["pos"])
        return _contents(state)
    if kind == "decode":
        h["decode"](ses.ctx, h["cache"], state["q"], h["index"], case["n"] + case["generated"] - 1, state["o"], ses.stream())
    else:
        ses.attend(h["cache"], state["q"], case["pos"], state["o"])
    return state["o"]


# --------------------------------------------------------------------------------------------- work
def work(case):
    hq, hkv, n, block = case["hq"], case["hkv"], case["n"], case["block"]
    if case["kind"] == "rotate":
        return {"bytes": (hq + hkv) * n * D * 4 + 4 * n * case["packed"], "flops": (hq + hkv) * n * case["dim"] * 3}
    if case["kind"] == "append":
        new, full = case["pos"] + n, _full(case["pos"] + n, block) - _full(case["pos"], block)
        before = case["pos"] % block if full else 0
        return {"bytes": 2 * hkv * ((before + n) * D * 2 + full * D + full // block * 4 + min(n, new % block) * D * 2),
                "flops": 2 * hkv * n * D * 2}
    if case["kind"] == "decode":
        kept = sum(a * block + b + c for a, b, c in _kept(case))
        tokens = case["n"] + case["generated"]
        rest = tokens % block
        return {"bytes": kept * 2 * D + hkv * (case["generated"] - rest) * 2 * D + hkv * rest * 4 * D + hq * D * 4,
                "flops": (kept + hq * case["generated"]) * 4 * D}
    tokens = case["pos"] + n
    full = _full(tokens, block)
    return {"bytes": hkv * (full * 2 * D + full // block * 8 + (tokens - full) * 4 * D) + hq * n * D * 4,
            "flops": hq * (n * case["pos"] + n * (n + 1) // 2) * 4 * D}


# ------------------------------------------------------------------------------------------ 64 bits
def _exact_round(y, kind):
    """The nearest value of the 8-bit type, ties to the even one; |y| is at most its largest."""
    bits, low = (3, -6) if kind == "e4m3" else (2, -14)
    m, _ = torch.frexp(y)
    step = torch.where(y != 0, y / m, 0.0) * 2.0 ** (-1 - bits)  # y / m is a power of two
    step = step.clamp(min=2.0 ** (low - bits))
    return torch.round(y / step) * step


def _exact_append(case, seed):
    s = prepare(case, seed)
    pos, n, block, kind = case["pos"], case["n"], case["block"], case["type"]
    start, end = pos // block, (pos + n) // block
    codes, scales, opens = [], [], []
    for name in ("k", "v"):
        c, sc, op = (s["cache"][name + x] for x in ("", "_scale", "_open"))
        c, sc, op = c.view(CODES[kind]).double(), sc.double(), op.double()
        x = torch.cat([op[:, :pos % block].clone(), s[name].double()], 1)
        for b in range(start, end):
            part = x[:, (b - start) * block:(b - start + 1) * block]
            top = part.abs().amax((1, 2))
            m, _ = torch.frexp(top / LARGEST[kind])
            scale = torch.where(m == 0.5, 0.5, 1.0) * (top / LARGEST[kind] / m)
            scale = torch.where(top > 0, scale.clamp(min=2.0 ** LEAST_EXPONENT), 1.0)
            c[:, b * block:(b + 1) * block] = _exact_round(part / scale[:, None, None], kind)
            sc[:, b] = scale
        if end > start:
            op[:, :pos + n - end * block] = x[:, (end - start) * block:]
        else:
            op[:, :x.shape[1]] = x
        codes.append(c)
        scales.append(sc)
        opens.append(op)
    return codes + scales + opens


def _exact_keys(s, name, tokens):
    case, c = s["case"], s["cache"]
    full = tokens - tokens % case["block"]
    x = torch.empty((case["hkv"], tokens, D), dtype=torch.float64, device="cuda")
    x[:, :full] = c[name][:, :full].view(CODES[case["type"]]).double()
    x[:, :full] *= c[name + "_scale"][:, :full // case["block"]].double().repeat_interleave(case["block"], 1)[..., None]
    x[:, full:] = c[name + "_open"][:, :tokens - full].double()
    return x


def _exact_rotate(case, seed):
    s = prepare(case, seed)
    w, amplitude = _frequencies(case)
    pos = s["positions"].double() if case["packed"] else (torch.arange(case["n"], device="cuda") + case["pos"]).double()
    z = torch.polar(torch.full_like(pos[:, None] * w, amplitude), pos[:, None] * w * (-1 if case["transposed"] else 1))
    out = []
    for x in (s["q"], s["k"]):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[0]):
            r = x[h].double()
            half = case["dim"] // 2
            if case["layout"] == "half":
                t = torch.complex(r[:, :half], r[:, half:case["dim"]]) * z
                r[:, :case["dim"]] = torch.cat([t.real, t.imag], 1)
            else:
                t = torch.complex(r[:, 0:case["dim"]:2], r[:, 1:case["dim"]:2]) * z
                r[:, 0:case["dim"]:2], r[:, 1:case["dim"]:2] = t.real, t.imag
            y[h] = r
        out.append(y)
    return out


def _exact_softmax(q, k, v):
    """One query [128] over its kept keys."""
    p = torch.softmax(k @ q / math.sqrt(D), 0)
    return p @ v


def exact(case, seed):
    if case["kind"] == "append":
        return _exact_append(case, seed)
    if case["kind"] == "rotate":
        return _exact_rotate(case, seed)
    s = prepare(case, seed)
    g = case["hq"] // case["hkv"]
    q = s["q"].double()
    o = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    if case["kind"] == "decode":
        n, pos, block, ix = case["n"], case["n"] + case["generated"] - 1, case["block"], s["index"]
        k, v = _exact_keys(s, "k", pos + 1), _exact_keys(s, "v", pos + 1)
        for h in range(case["hq"]):
            a, b = ix["rowptr"][h, n // block - 1].item(), ix["rowptr"][h, n // block].item()
            keys = set(range(n, pos + 1)) | set(ix["cols"][h, :ix["n_cols"][h]].tolist())
            keys |= {pos - x for x in ix["offs"][h, :ix["n_offs"][h]].tolist()}
            for c in ix["blkcols"][h, a:b].tolist():
                keys |= set(range(c * block, (c + 1) * block))
            at = torch.tensor(sorted(keys), device="cuda")
            o[h] = _exact_softmax(q[h], k[h // g, at], v[h // g, at])
        return o
    n, pos = case["n"], case["pos"]
    k, v = _exact_keys(s, "k", pos + n), _exact_keys(s, "v", pos + n)
    later = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    for h in range(case["hq"]):
        t = q[h] @ k[h // g].T / math.sqrt(D)
        t[:, pos:].masked_fill_(later, -math.inf)
        o[h] = torch.softmax(t, -1) @ v[h // g]
    return o
