"""Operators of a decoder whose attention reaches back a bounded way: positions as rotations of queries and keys, with norms of the
heads in the same pass, and attention over a sliding window and the first tokens, in training and over a cache.

In all of them sequence b has tokens i < len[b] (of S; all without `ragged`) at positions start[b] + i (0 without `far`).

A case is a dict of plain values with an "op":
  rotary      q [B, S, H dh] and k [B, S, Hkv dh] bf16, columns of one projection's q | k | v: with `norm` each head over the root of its mean
              square times a weight, then its first `rot` columns turned by position times frequency, as pairs of neighbours or of the two
              halves, with frequencies as they are or scaled for long contexts.  Rows behind a sequence become zero.  With `cache` rows a
              sequence, keys and values go to the cache, whose rows behind the first `sinks` are a ring.
  rotary_bwd  the gradients of q, k and the norms' weights from those of the results.
  window      attention of Sq query tokens over Sk rows of keys: a token sees the `window` last keys up to its own and the first `sinks`; H
              query heads over Hkv of dh columns, with the log2-sum-exp2 of the scores.  With `far` the rows are such a cache, which holds
              what the tokens up to start + len left.
  window_bwd  its gradients (Sq == Sk, no cache), from what a forward left.
"""
import math
import random

import torch

own = False

BASE = 10000.0


def listed():
    return [
        # one new token of one sequence, a narrow decoder: launch latency
        {"name": "rot_token_768", "op": "rotary", "B": 1, "S": 1, "H": 12, "Hkv": 12, "dh": 64, "rot": 64, "layout": "half", "norm": False,
         "scaled": "none", "ragged": False, "far": 900, "cache": 1024, "sinks": 0},
        # one new token of each of 32 sequences, far behind the length trained at, norms, into rings of 4096 rows behind four sinks
        {"name": "rot_token_ring", "op": "rotary", "B": 32, "S": 1, "H": 32, "Hkv": 8, "dh": 128, "rot": 128, "layout": "half", "norm": True,
         "scaled": "parts", "ragged": False, "far": 200000, "cache": 4100, "sinks": 4},
        # training forward of the width of 1600: neighbours turned, half of a head, texts of different lengths
        {"name": "rot_fwd_1600", "op": "rotary", "B": 8, "S": 511, "H": 25, "Hkv": 25, "dh": 64, "rot": 32, "layout": "pairs", "norm": False,
         "scaled": "none", "ragged": True, "far": 0, "cache": 0, "sinks": 0},
        # a long text in one piece, norms, shared heads: bound by memory
        {"name": "rot_fwd_long", "op": "rotary", "B": 1, "S": 65536, "H": 32, "Hkv": 8, "dh": 128, "rot": 128, "layout": "half", "norm": True,
         "scaled": "linear", "ragged": False, "far": 0, "cache": 0, "sinks": 0},
        # training backward of the narrow width, texts of different lengths, no norms
        {"name": "rot_bwd_768", "op": "rotary_bwd", "B": 8, "S": 384, "H": 12, "Hkv": 12, "dh": 64, "rot": 64, "layout": "half", "norm": False,
         "scaled": "none", "ragged": True, "far": 0, "cache": 0, "sinks": 0},
        # training backward of a width of 4096 with norms and their weights' gradients
        {"name": "rot_bwd_4096", "op": "rotary_bwd", "B": 4, "S": 4096, "H": 32, "Hkv": 8, "dh": 128, "rot": 128, "layout": "half", "norm": True,
         "scaled": "none", "ragged": False, "far": 0, "cache": 0, "sinks": 0},
        # one new token of one sequence that has not filled its window
        {"name": "win_token_768", "op": "window", "B": 1, "Sq": 1, "Sk": 1024, "H": 12, "Hkv": 12, "dh": 64, "window": 1000, "sinks": 0,
         "ragged": False, "far": 900},
        # one new token of each of 32 sequences over rings of 4096 keys behind four sinks: reading the cache once
        {"name": "win_token_ring", "op": "window", "B": 32, "Sq": 1, "Sk": 4100, "H": 32, "Hkv": 8, "dh": 128, "window": 4096, "sinks": 4,
         "ragged": False, "far": 200000},
        # training forward of the width of 1600, a short reach, texts of different lengths
        {"name": "win_fwd_1600", "op": "window", "B": 8, "Sq": 511, "Sk": 511, "H": 25, "Hkv": 25, "dh": 64, "window": 128, "sinks": 1,
         "ragged": True, "far": 0},
        # a long text in one piece, shared heads
        {"name": "win_fwd_long", "op": "window", "B": 1, "Sq": 32768, "Sk": 32768, "H": 32, "Hkv": 8, "dh": 128, "window": 4096, "sinks": 4,
         "ragged": False, "far": 0},
        # training backward of the narrow width
        {"name": "win_bwd_768", "op": "window_bwd", "B": 8, "Sq": 1000, "Sk": 1000, "H": 12, "Hkv": 12, "dh": 64, "window": 256, "sinks": 4,
         "ragged": True, "far": 0},
        # training backward over sequences of 4096, eight query heads to a key/value head
        {"name": "win_bwd_2048", "op": "window_bwd", "B": 4, "Sq": 4096, "Sk": 4096, "H": 16, "Hkv": 2, "dh": 128, "window": 1024, "sinks": 4,
         "ragged": False, "far": 0},
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "rotary_bwd", "window", "window", "window_bwd"])
    dh, share = rng.choice([64, 128]), rng.choice([1, 1, 2, 4, 8])
    H = share * rng.randint(1, 32 // share)
    Hkv = H // share
    sinks = rng.choice([0, 1, 4, 4, 16, 100])
    if op in ("rotary", "rotary_bwd"):
        while True:
            token = op == "rotary" and rng.random() < 0.4
            c = {"op": op, "B": _spread(rng, 1, 64), "S": 1 if token else _spread(rng, 1, 65536), "H": H, "Hkv": Hkv, "dh": dh,
                 "rot": dh if rng.random() < 0.5 else 16 * rng.randint(1, dh // 16), "layout": rng.choice(["half", "pairs"]),
                 "norm": rng.random() < 0.5, "scaled": rng.choice(["none", "none", "linear", "base", "parts"]), "ragged": rng.random() < 0.5,
                 "far": rng.choice([0, 5000, 1000000]), "cache": 0, "sinks": 0}
            if token or (op == "rotary" and rng.random() < 0.2):
                c["cache"], c["sinks"] = sinks + _spread(rng, 64, 8192), sinks
            if c["B"] * c["S"] * (H + 2 * Hkv) * dh <= 65536 * 40 * 128 // 2 and c["B"] * c["cache"] * Hkv * dh <= 1 << 28:
                return c
    while True:
        window = _spread(rng, 1, 8192)
        c = {"op": op, "B": _spread(rng, 1, 64), "Sq": _spread(rng, 1, 32768), "Sk": 0, "H": H, "Hkv": Hkv, "dh": dh, "window": window,
             "sinks": sinks, "ragged": rng.random() < 0.5, "far": 0}
        if op == "window" and rng.random() < 0.6:
            c["far"] = rng.choice([100, 5000, 1000000])
            c["Sq"] = 1 if rng.random() < 0.6 else _spread(rng, 2, 2048)
            c["ragged"] = c["ragged"] and c["Sq"] > 1
            c["Sk"] = sinks + window + c["Sq"] - 1 + rng.choice([0, 0, 1, 500])
        else:
            c["Sk"] = c["Sq"]
        pairs = c["B"] * H * c["Sq"] * min(c["Sk"], window + sinks)
        keys = c["B"] * c["Sk"] * Hkv * dh
        if pairs * dh <= 32 * 32768 * 4096 * 128 // (4 if op == "window_bwd" else 1) and max(keys, c["B"] * c["Sq"] * H * dh) <= 1 << 28:
            return c


# ---- what the case alone says ------------------------------------------------------------------

def _rng(c, what):
    return random.Random("%s %s" % (what, sorted((k, v) for k, v in c.items() if k not in ("name", "op"))))


def _lengths(c):
    """Tokens of each sequence; the last of more than two has none."""
    S = c["S"] if "S" in c else c["Sq"]
    if not c["ragged"]:
        return [S] * c["B"]
    r = _rng(c, "lengths")
    n = [r.randint((S + 1) // 2, S) for _ in range(c["B"])]
    n[0] = S
    if c["B"] > 2:
        n[-1] = 0
    return n


def _starts(c):
    """Tokens that each sequence had before."""
    if not c["far"]:
        return [0] * c["B"]
    r = _rng(c, "starts")
    return [r.randint(0, c["far"]) for _ in range(c["B"])]


def _spans(c, b):
    """Of sequence b: its tokens, the first one's position, and the oldest key behind the sinks that the rows still hold."""
    n, start = _lengths(c)[b], _starts(c)[b]
    return n, start, max(0, start + n - (c["Sk"] - min(c["sinks"], c["Sk"] - 1)))


def _pairs(c):
    """(visible pairs of a head, keys that anyone sees) over all sequences"""
    pairs = keys = 0
    for b in range(c["B"]):
        n, start, held = _spans(c, b)
        if n == 0:
            continue
        p = torch.arange(start, start + n, dtype=torch.int64)
        low = (p - c["window"] + 1).clamp(min=held).clamp(min=0)
        first = torch.minimum(low, torch.tensor(min(c["sinks"], c["Sk"] - 1)))
        pairs += int((p - low + 1 + torch.minimum(first, p + 1)).sum())
        keys += start + n - int(low[0]) + int(first[0])
    return pairs, keys


def work(case):
    c = case
    if c["op"] in ("rotary", "rotary_bwd"):
        tokens, every = sum(_lengths(c)), c["B"] * c["S"]
        q, kv = c["H"] * c["dh"] * 2, c["Hkv"] * c["dh"] * 2
        heads = c["H"] + c["Hkv"]
        if c["op"] == "rotary_bwd":
            return {"bytes": tokens * (q + kv) * (2 if c["norm"] else 1) + every * (q + kv), "flops": tokens * heads * c["dh"] * (12 if c["norm"] else 3)}
        if c["cache"]:
            return {"bytes": tokens * (q + 2 * kv) + every * q + tokens * 2 * kv, "flops": tokens * heads * c["dh"] * (7 if c["norm"] else 3)}
        return {"bytes": tokens * (q + kv) + every * (q + kv), "flops": tokens * heads * c["dh"] * (7 if c["norm"] else 3)}
    pairs, keys = _pairs(c)
    tokens = sum(_lengths(c))
    row = c["H"] * c["dh"] * 2
    kv = 2 * keys * c["Hkv"] * c["dh"] * 2
    lse = c["B"] * c["H"] * c["Sq"] * 4
    if c["op"] == "window":
        return {"bytes": tokens * row + c["B"] * c["Sq"] * row + kv + lse, "flops": 4 * c["H"] * pairs * c["dh"]}
    every = c["B"] * c["Sq"] * (row + 2 * c["Hkv"] * c["dh"] * 2)
    return {"bytes": 3 * tokens * row + kv + lse + every, "flops": 10 * c["H"] * pairs * c["dh"]}


# ---- inputs ------------------------------------------------------------------------------------

SCALED = {"none": (1.0, 0), "linear": (8.0, 0), "base": (8.0, 0), "parts": (32.0, 4096)}
LOW, HIGH = 1.0, 32.0                      # turns within the context, of "parts"


def _frequencies(c):
    """Radians a position, in 64 bits, and the factor of what is turned."""
    rot, (factor, context) = c["rot"], SCALED[c["scaled"]]
    base = BASE * factor ** (rot / (rot - 2)) if c["scaled"] == "base" else BASE
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if c["scaled"] == "linear":
        f = f / factor
    if c["scaled"] != "parts":
        return f, 1.0
    keep = ((context * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(torch.bfloat16)

    B, H, Hkv, dh = c["B"], c["H"], c["Hkv"], c["dh"]
    S = c["S"] if "S" in c else c["Sq"]
    on_gpu = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": c, "length": on_gpu(_lengths(c)) if c["ragged"] else None, "start": on_gpu(_starts(c)) if c["far"] else None}
    behind = None
    if c["ragged"]:
        behind = (torch.arange(S, device="cuda")[None, :] >= s["length"][:, None])[..., None]

    def clean(t):
        return t if behind is None else t.masked_fill_(behind, float("nan"))     # what padding holds is nobody's business

    if c["op"] in ("rotary", "rotary_bwd"):
        qkv = clean(normal(B, S, (H + 2 * Hkv) * dh, std=1.5))
        s["q"], s["k"], s["v"] = qkv[..., :H * dh], qkv[..., H * dh:(H + Hkv) * dh], qkv[..., (H + Hkv) * dh:]
        freq, s["amplitude"] = _frequencies(c)
        s["freq"] = freq.cuda()
        s["gamma_q"] = (1.0 + normal(dh, std=0.1).float()).to(torch.bfloat16) if c["norm"] else None
        s["gamma_k"] = (1.0 + normal(dh, std=0.1).float()).to(torch.bfloat16) if c["norm"] else None
        if c["cache"]:
            s["cache"] = normal(B, c["cache"], Hkv * dh), normal(B, c["cache"], Hkv * dh)
        if c["op"] == "rotary_bwd":
            s["dq"], s["dk"] = clean(normal(B, S, H * dh, std=1e-2)), clean(normal(B, S, Hkv * dh, std=1e-2))
        return s
    if c["far"]:
        # a cache of keys and one of values; rows that nothing has been written to hold anything
        s["q"] = clean(normal(B, S, H * dh, std=1.5))
        s["k"], s["v"] = normal(B, c["Sk"], Hkv * dh), normal(B, c["Sk"], Hkv * dh)
        unwritten = (torch.arange(c["Sk"], device="cuda")[None, :] >= torch.tensor([st + n for st, n in zip(_starts(c), _lengths(c))], device="cuda")[:, None])
        s["k"].masked_fill_(unwritten[..., None], float("nan"))
        s["v"].masked_fill_(unwritten[..., None], float("nan"))
    else:
        qkv = clean(normal(B, S, (H + 2 * Hkv) * dh, std=1.2))
        s["q"], s["k"], s["v"] = qkv[..., :H * dh], qkv[..., H * dh:(H + Hkv) * dh], qkv[..., (H + Hkv) * dh:]
    if c["op"] == "window_bwd":
        s["out"], s["lse2"] = _window(s)
        s["dout"] = clean(normal(B, S, H * dh, std=1e-2))
    return s


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"rotary": _rotary, "rotary_bwd": _rotary_bwd, "window": _window, "window_bwd": _window_bwd}[op](s)


def _own(s, op):
    from paper_2401_01728_amd import kernels
    c = s["case"]
    if op in ("rotary", "rotary_bwd"):
        how = dict(layout=c["layout"], amplitude=s["amplitude"], gamma_q=s["gamma_q"], gamma_k=s["gamma_k"], eps=1e-6, start=s["start"],
                   length=s["length"])
        if op == "rotary_bwd":
            # without norms the inputs are not read
            q, k = (s["q"], s["k"]) if c["norm"] else (None, None)
            return [t for t in kernels.rotary_bwd(s["dq"], s["dk"], s["freq"], c["H"], c["Hkv"], q=q, k=k, **how) if t is not None]
        if c["cache"]:
            return kernels.rotary_fwd(s["q"], s["k"], s["freq"], c["H"], c["Hkv"], v=s["v"], cache=s["cache"], sinks=c["sinks"], **how)
        return kernels.rotary_fwd(s["q"], s["k"], s["freq"], c["H"], c["Hkv"], **how)
    if op == "window":
        return kernels.window_attention_fwd(s["q"], s["k"], s["v"], c["H"], c["Hkv"], c["window"], c["sinks"], s["start"], s["length"])
    return kernels.window_attention_bwd(s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse2"], c["H"], c["Hkv"], c["window"], c["sinks"], s["length"])


# ---- the plain forms ---------------------------------------------------------------------------

def _heads(t, h):
    """[B, S, h * dh] -> [B, S, h, dh] in 32 bits"""
    return t.float().unflatten(-1, (h, -1))


def _positions(s):
    c = s["case"]
    p = torch.arange(c["S"], device="cuda")[None, :]
    return p.expand(c["B"], -1) if s["start"] is None else p + s["start"][:, None]


def _cos_sin(s):
    angle = (_positions(s).double()[..., None] * s["freq"])[:, :, None]         # [B, S, 1, rot / 2]
    return angle.cos().mul_(s["amplitude"]).float(), angle.sin().mul_(s["amplitude"]).float()


def _turn(x, cos, sin, c):
    rot = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., rot:]], -1)


def _live(s):
    """[B, S, 1], or None where every token is"""
    if s["length"] is None:
        return None
    c = s["case"]
    S = c["S"] if "S" in c else c["Sq"]
    return (torch.arange(S, device="cuda")[None, :] < s["length"][:, None])[..., None]


def _zero_behind(t, live):
    return t if live is None else torch.where(live, t, 0.0)


def _slots(position, sinks, rows):
    sinks = min(sinks, rows - 1)
    return torch.where(position < sinks, position, sinks + (position - sinks) % (rows - sinks))


def _rotary(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    live = _live(s)
    out = []
    for t, h, gamma in ((s["q"], c["H"], s["gamma_q"]), (s["k"], c["Hkv"], s["gamma_k"])):
        x = _heads(t, h)
        if gamma is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gamma.float()
        out.append(_zero_behind(_turn(x, cos, sin, c).flatten(-2).to(torch.bfloat16), live))
    if not c["cache"]:
        return out
    keys, values = s["cache"]
    p = _positions(s)
    n = torch.full((c["B"],), c["S"], device="cuda") if s["length"] is None else s["length"]
    first = torch.zeros_like(n) if s["start"] is None else s["start"]
    if c["S"] == 1 and s["length"] is None:
        b, row = torch.arange(c["B"], device="cuda"), _slots(p[:, 0], c["sinks"], c["cache"])
        keys[b, row], values[b, row] = out[1][:, 0], s["v"][:, 0]
        return out[0], keys, values
    # of two tokens with one row the later is kept
    sinks = min(c["sinks"], c["cache"] - 1)
    stays = (torch.arange(c["S"], device="cuda") < n[:, None]) & ((p < sinks) | (p + (c["cache"] - sinks) >= (first + n)[:, None]))
    b, i = stays.nonzero(as_tuple=True)
    row = _slots(p[b, i], c["sinks"], c["cache"])
    keys[b, row], values[b, row] = out[1][b, i], s["v"][b, i]
    return out[0], keys, values


def _rotary_bwd(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    live = _live(s)
    grads, weights = [], []
    for t, d, h, gamma in ((s["q"], s["dq"], c["H"], s["gamma_q"]), (s["k"], s["dk"], c["Hkv"], s["gamma_k"])):
        g = _turn(_heads(_zero_behind(d, live), h), cos, -sin, c)
        if gamma is not None:
            x = _heads(_zero_behind(t, live), h)
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
            xh = x * r
            weights.append((g * xh).double().sum((0, 1, 2)).float())
            g = g * gamma.float()
            g = r * (g - xh * (g * xh).mean(-1, keepdim=True))
        grads.append(g.flatten(-2).to(torch.bfloat16))
    return grads + weights


ROWS = 1024                                # tokens that are looked at together


def _walk(s, b):
    """Pieces of sequence b's tokens: (their slice, the rows of the keys that any of them may see, [tokens, keys] which sees which)."""
    c = s["case"]
    n, start, held = _spans(c, b)
    sinks = min(c["sinks"], c["Sk"] - 1)
    for i in range(0, n, ROWS):
        m = min(ROWS, n - i)
        low = max(0, held, start + i - c["window"] + 1)
        key = torch.arange(low, start + i + m, device="cuda")
        if sinks and low:
            key = torch.cat([torch.arange(min(sinks, low), device="cuda"), key])
        p = torch.arange(start + i, start + i + m, device="cuda")[:, None]
        sees = (key <= p) & ((key > p - c["window"]) | (key < sinks))
        yield slice(i, i + m), _slots(key, c["sinks"], c["Sk"]), sees


def _split(t, b, rows, h):
    """[h, rows, dh] in 32 bits"""
    return t[b, rows].float().unflatten(-1, (h, -1)).transpose(0, 1)


def _merge(t):
    return t.transpose(0, 1).flatten(-2)


def _window_token(s):
    """One token to a sequence: all sequences at once, over all rows."""
    c = s["case"]
    B, H, Hkv, Sk, dh = c["B"], c["H"], c["Hkv"], c["Sk"], c["dh"]
    sinks = min(c["sinks"], Sk - 1)
    p = s["start"][:, None].long()
    row = torch.arange(Sk, device="cuda")[None, :]
    key = torch.where(row < sinks, row, row + torch.div(p - row, Sk - sinks, rounding_mode="floor") * (Sk - sinks))    # which a row holds
    sees = ((key <= p) & (key >= row) & ((key > p - c["window"]) | (key < sinks)))[:, None, None]                       # [B, 1, 1, Sk]
    k, v = (torch.where(sees[:, 0, 0, :, None, None], _heads(t, Hkv), 0.0).transpose(1, 2).contiguous() for t in (s["k"], s["v"]))
    q = _heads(s["q"], H).reshape(B, Hkv, H // Hkv, dh)
    z = (q @ k.transpose(-1, -2).contiguous() * (math.log2(math.e) / math.sqrt(dh))).masked_fill(~sees, -math.inf)
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp2()
    total = e.sum(-1, keepdim=True)
    return ((e @ v) / total).reshape(B, 1, -1).to(torch.bfloat16), (top + total.log2()).reshape(B, H, 1)


def _window(s):
    c = s["case"]
    if c["Sq"] == 1 and s["start"] is not None and s["length"] is None:
        return _window_token(s)
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    lse2 = torch.full((c["B"], H, c["Sq"]), -math.inf, device="cuda")
    for b in range(c["B"]):
        for at, rows, sees in _walk(s, b):
            q = _split(s["q"], b, at, H).unflatten(0, (Hkv, -1))
            k, v = _split(s["k"], b, rows, Hkv), _split(s["v"], b, rows, Hkv)
            z = (q.flatten(1, 2) @ k.transpose(-1, -2).contiguous()).view(Hkv, H // Hkv, -1, len(rows)) * (math.log2(math.e) / math.sqrt(dh))
            z.masked_fill_(~sees, -math.inf)
            top = z.amax(-1, keepdim=True)
            p = (z - top).exp2_()
            total = p.sum(-1, keepdim=True)
            o = (p.flatten(1, 2) @ v).view(Hkv, H // Hkv, -1, dh) / total
            out[b, at] = _merge(o.flatten(0, 1)).to(torch.bfloat16)
            lse2[b, :, at] = (top + total.log2()).flatten(0, 1)[..., 0]
    return out, lse2


def _window_bwd(s):
    c = s["case"]
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    dq = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    dk, dv = (torch.zeros(c["B"], c["Sk"], Hkv, dh, device="cuda") for _ in range(2))
    for b in range(c["B"]):
        for at, rows, sees in _walk(s, b):
            q, o, do = (_split(s[n], b, at, H).reshape(Hkv, -1, dh) for n in ("q", "out", "dout"))
            k, v = _split(s["k"], b, rows, Hkv), _split(s["v"], b, rows, Hkv)
            z = (q @ k.transpose(-1, -2).contiguous()) * (math.log2(math.e) / math.sqrt(dh))
            p = (z - s["lse2"][b, :, at].reshape(Hkv, -1, 1)).exp2_()
            p = torch.where(sees.repeat(H // Hkv, 1), p, 0.0)
            ds = p * (do @ v.transpose(-1, -2).contiguous() - (do * o).sum(-1, keepdim=True)) / math.sqrt(dh)
            dq[b, at] = _merge((ds @ k).view(H, -1, dh)).to(torch.bfloat16)
            dk[b].index_add_(0, rows, (ds.transpose(-1, -2).contiguous() @ q).transpose(0, 1))
            dv[b].index_add_(0, rows, (p.transpose(-1, -2).contiguous() @ do).transpose(0, 1))
    return dq, dk.flatten(-2).to(torch.bfloat16), dv.flatten(-2).to(torch.bfloat16)


# ---- the definitions, in 64 bits ---------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_rotary if case["op"] in ("rotary", "rotary_bwd") else _exact_window)(s, case)


def _exact_rotary(s, c):
    """Every pair as a complex number times exp(i angle)."""
    B, S, rot, dh = c["B"], c["S"], c["rot"], c["dh"]
    n, start = _lengths(c), _starts(c)
    grads = c["op"] == "rotary_bwd"
    give = [[], []]
    freq = s["freq"].double()
    leaves = [None, None]
    weights = [w.double().requires_grad_(grads) if w is not None else None for w in (s["gamma_q"], s["gamma_k"])]
    total_w = [0.0, 0.0]
    for b in range(B):
        spin = torch.polar(torch.full((S, 1, rot // 2), s["amplitude"], dtype=torch.float64, device="cuda"),
                           (torch.arange(start[b], start[b] + S, device="cuda").double()[:, None] * freq)[:, None])[:n[b]]
        for i, (t, h, d) in enumerate(((s["q"], c["H"], s.get("dq")), (s["k"], c["Hkv"], s.get("dk")))):
            leaf = t[b, :n[b]].double().reshape(n[b], h, dh).requires_grad_(grads)
            x = leaf
            if weights[i] is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / dh + 1e-6) * weights[i]
            if c["layout"] == "half":
                y = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * spin
                y = torch.cat([y.real, y.imag, x[..., rot:]], -1)
            else:
                y = torch.view_as_complex(x[..., :rot].reshape(n[b], h, rot // 2, 2).contiguous()) * spin
                y = torch.cat([torch.view_as_real(y).reshape(n[b], h, rot), x[..., rot:]], -1)
            if grads:
                up = d[b, :n[b]].double().reshape(n[b], h, dh)
                if n[b] == 0:
                    y = torch.zeros_like(leaf)
                elif weights[i] is not None:
                    y, gw = torch.autograd.grad(y, (leaf, weights[i]), up)
                    total_w[i] = total_w[i] + gw
                else:
                    y = torch.autograd.grad(y, leaf, up)[0]
            give[i].append(torch.cat([y.detach().reshape(n[b], h * dh), torch.zeros(S - n[b], h * dh, dtype=torch.float64, device="cuda")]))
    q, k = torch.stack(give[0]), torch.stack(give[1])
    if grads:
        return [q, k] + ([total_w[0], total_w[1]] if c["norm"] else [])
    if not c["cache"]:
        return [q, k]
    keys, values = (t.double() for t in s["cache"])
    sinks = min(c["sinks"], c["cache"] - 1)
    ring = c["cache"] - sinks
    for b in range(B):
        # in order: first the tokens whose row is never taken again, by position
        p = torch.arange(start[b], start[b] + n[b], device="cuda")
        last = max(0, int(n[b]) - ring)
        late = p[last:]
        early = p[:last]
        early = early[early < sinks]
        for part in (early, late):
            row = torch.where(part < sinks, part, (part - sinks).remainder(ring) + sinks)
            keys[b].index_copy_(0, row, k[b].index_select(0, part - start[b]))
            values[b].index_copy_(0, row, s["v"][b].double().index_select(0, part - start[b]))
    return q, keys, values


def _exact_window(s, c):
    B, Sq, Sk, H, Hkv, dh = c["B"], c["Sq"], c["Sk"], c["H"], c["Hkv"], c["dh"]
    grads = c["op"] == "window_bwd"
    if B * H * Sq * (Sk if not c["far"] else c["window"] + Sq) > 1 << 36:
        return None
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse2 = torch.zeros(B, Sq, H * dh, **f64), torch.full((B, H, Sq), -math.inf, **f64)
    dq, dk, dv = (torch.zeros(*t.shape, **f64) for t in (s["q"], s["k"], s["v"]))
    sinks = min(c["sinks"], Sk - 1)
    for b in range(B):
        n, start = _lengths(c)[b], _starts(c)[b]
        if n == 0:
            continue
        # which position each row of the keys holds: the latest of those that share it
        end = start + n
        row = torch.arange(Sk, device="cuda")
        held = torch.where(row < sinks, row, row + torch.div(end - 1 - row, Sk - sinks, rounding_mode="floor") * (Sk - sinks))
        there = ((held < end) & (held >= row)).nonzero()[:, 0]
        held = held[there]
        for i in range(0, n, 4096):
            p = torch.arange(start + i, start + min(n, i + 4096), device="cuda")[:, None]
            at = slice(i, min(n, i + 4096))
            hide = (held > p) | ((held <= p - c["window"]) & (held >= sinks))
            for h in range(H):
                col, kcol = slice(h * dh, (h + 1) * dh), slice(h // (H // Hkv) * dh, (h // (H // Hkv) + 1) * dh)
                q, k, v = s["q"][b, at, col].double(), s["k"][b, there, kcol].double(), s["v"][b, there, kcol].double()
                for t in (q, k, v):
                    t.requires_grad_(grads)
                z = (q @ k.T / math.sqrt(dh)).masked_fill(hide, -math.inf)
                o = torch.softmax(z, -1) @ v
                if grads:
                    g = torch.autograd.grad(o, (q, k, v), s["dout"][b, at, col].double())
                    dq[b, at, col] = g[0]
                    dk[b, :, kcol].index_add_(0, there, g[1])
                    dv[b, :, kcol].index_add_(0, there, g[2])
                else:
                    out[b, at, col] = o
                    lse2[b, h, at] = torch.logsumexp(z, -1) / math.log(2.0)
    return (dq, dk, dv) if grads else (out, lse2)
