"""Operators of a conditional language model that a chain of decoder peers is trained with, beside the stage itself:
the loss at the chain's end, with its gradients, and the attention to an encoder's states.

A case is a dict of plain values with an "op":
  loss      loss and log-sum-exp of every token against a vocabulary: x [T, d] bf16 times w [V, d] bf16 transposed, softmax
            cross entropy with the token's label.  A share `masked` of the labels is -1 (prompt, padding): such rows take no
            part, whatever they hold.
  step      the same with its gradients: dx and, `update` false, dw, or, `update` true, the fp32 master weights after the
            SGD step of the chain's other peers and their bf16 version.
  cross     attention of Sq query tokens to an encoder's states of another length, H query heads over Hkv key/value heads of
            dh columns, with the log2-sum-exp2 of the scores.  `ragged`: the sequences have lengths of their own up to Sk,
            the last one of more than two has none; what lies behind a length is not a number.
  cross_bwd its gradients, from what a forward left.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # evaluation of a single token: one row against the whole vocabulary, bound by reading the weights once
        {"name": "loss_token", "op": "loss", "T": 1, "V": 32000, "d": 1024, "masked": 0.0},
        # validation of a batch of ragged texts under the decoder of width 1600: an odd vocabulary, odd rows
        {"name": "loss_eval_1600", "op": "loss", "T": 3001, "V": 50257, "d": 1600, "masked": 0.1},
        # the last peer of the narrow chain (width 448, two sequences of 128): few rows, a vocabulary of word pieces
        {"name": "step_narrow", "op": "step", "T": 256, "V": 30522, "d": 448, "masked": 0.15, "update": False},
        # the last peer of the chain of width 1024 in tuning on answers: half of the tokens are prompt
        {"name": "step_1024_half", "op": "step", "T": 4096, "V": 50257, "d": 1024, "masked": 0.5, "update": False},
        # the last peer of the chain of width 2048, its head updated in the same call (staleness 0)
        {"name": "step_2048_update", "op": "step", "T": 4096, "V": 32000, "d": 2048, "masked": 0.0, "update": True},
        # a large vocabulary over the largest microbatch of the benchmark
        {"name": "step_large", "op": "step", "T": 8192, "V": 128000, "d": 2048, "masked": 0.05, "update": False},
        # one new token of each of 16 sequences against an encoder's states of up to 1500 frames
        {"name": "cross_token", "op": "cross", "B": 16, "Sq": 1, "Sk": 1500, "H": 16, "Hkv": 16, "dh": 64, "ragged": True},
        # one new token against a long document, shared heads: the work is reading the states once
        {"name": "cross_token_long", "op": "cross", "B": 2, "Sq": 1, "Sk": 100001, "H": 32, "Hkv": 8, "dh": 128, "ragged": False},
        # training forward with the heads of the decoder of width 1600 over the patches of an image and a class token
        {"name": "cross_fwd_patches", "op": "cross", "B": 8, "Sq": 512, "Sk": 577, "H": 25, "Hkv": 25, "dh": 64, "ragged": False},
        # a long target over a longer source, shared heads
        {"name": "cross_fwd_large", "op": "cross", "B": 4, "Sq": 2048, "Sk": 8192, "H": 32, "Hkv": 8, "dh": 128, "ragged": True},
        # training backward of the width of 768 over sources of different lengths, one of them empty
        {"name": "cross_bwd_768", "op": "cross_bwd", "B": 8, "Sq": 384, "Sk": 1000, "H": 12, "Hkv": 12, "dh": 64, "ragged": True},
        # training backward of the width of 2048, four query heads to a key/value head
        {"name": "cross_bwd_2048", "op": "cross_bwd", "B": 4, "Sq": 1024, "Sk": 2048, "H": 16, "Hkv": 4, "dh": 128, "ragged": True},
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["loss", "step", "step", "cross", "cross", "cross_bwd"])
    if op in ("loss", "step"):
        while True:
            c = {"op": op, "T": _spread(rng, 1, 16384), "V": _spread(rng, 1000, 131072), "d": 64 * _spread(rng, 2, 64),
                 "masked": rng.choice([0.0, 0.0, 0.1, 0.3, 0.7])}
            # no more than the largest listed step: in products, and in what is written
            if c["T"] * c["V"] * c["d"] <= 8192 * 128000 * 2048 and c["T"] * c["V"] <= 8192 * 128000 and c["V"] * c["d"] <= 128000 * 2048:
                break
        if op == "step":
            c["update"] = rng.random() < 0.4
        return c
    while True:
        dh, share = rng.choice([64, 128]), rng.choice([1, 1, 2, 4, 8])
        token = op == "cross" and rng.random() < 0.4
        c = {"op": op, "B": _spread(rng, 1, 32), "Sq": 1 if token else _spread(rng, 1, 4096),
             "Sk": _spread(rng, 1, 131072 if token else 16384), "H": share * rng.randint(1, 32 // share), "Hkv": 0, "dh": dh,
             "ragged": rng.random() < 0.6}
        c["Hkv"] = c["H"] // share
        scores = c["B"] * c["H"] * c["Sq"] * c["Sk"]
        if scores <= 4 * 32 * 2048 * 8192 // (4 if op == "cross_bwd" else 1) and c["B"] * c["Sk"] * c["Hkv"] * dh <= 1 << 29:
            return c


def _lengths(c):
    """The sequences' numbers of keys: of the case alone, so that the work does not depend on the seed."""
    if not c["ragged"]:
        return [c["Sk"]] * c["B"]
    r = random.Random(c["Sk"] * 64 + c["B"])
    n = [r.randint((c["Sk"] + 1) // 2, c["Sk"]) for _ in range(c["B"])]
    n[0] = c["Sk"]
    if c["B"] > 2:
        n[-1] = 0
    return n


def _kept(c):
    return c["T"] - int(c["T"] * c["masked"])


def work(case):
    c = case
    if c["op"] in ("loss", "step"):
        T, V, d = c["T"], c["V"], c["d"]
        n = _kept(c)
        read = n * d * 2 + V * d * 2 + T * 8
        if c["op"] == "loss":
            return {"bytes": read + T * 8, "flops": 2 * n * V * d}
        weights = V * d * (4 + 4 + 2) if c["update"] else V * d * 2
        return {"bytes": read + T * 4 + T * d * 2 + weights, "flops": 6 * n * V * d}
    keys = sum(_lengths(c))
    q = c["B"] * c["Sq"] * c["H"] * c["dh"] * 2
    kv = 2 * keys * c["Hkv"] * c["dh"] * 2
    lse = c["B"] * c["H"] * c["Sq"] * 4
    pairs = c["H"] * c["Sq"] * keys
    if c["op"] == "cross":
        return {"bytes": 2 * q + kv + lse, "flops": 4 * pairs * c["dh"]}
    return {"bytes": 4 * q + 2 * kv + lse, "flops": 10 * pairs * c["dh"]}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std)

    if c["op"] in ("loss", "step"):
        T, V, d = c["T"], c["V"], c["d"]
        w32 = normal(V, d, std=0.02)
        w = w32.to(torch.bfloat16)
        label = torch.randint(0, V, (T,), generator=g, device="cuda")
        # hidden states as a normalised decoder gives them; some tokens are nearly certain, most are not
        sure = torch.rand(T, 1, generator=g, device="cuda") ** 2 * (18.0 / (0.02 ** 2 * d) * 0.02)
        x = (normal(T, d) + sure * w32[label] / 0.02).to(torch.bfloat16)
        out = torch.randperm(T, generator=g, device="cuda")[:T - _kept(c)]
        label[out] = -1
        x[out] = float("nan")               # what padding holds is nobody's business
        s = {"case": c, "x": x, "w": w, "label": label, "scale": 1.0 / max(1, _kept(c))}
        if c["op"] == "step" and c["update"]:
            s |= {"master": w32, "eta": 0.1, "master_out": torch.empty_like(w32), "version": torch.empty_like(w)}
        return s
    B, Sq, Sk, H, Hkv, dh = c["B"], c["Sq"], c["Sk"], c["H"], c["Hkv"], c["dh"]
    length = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    q = normal(B, Sq, H * dh, std=1.5).to(torch.bfloat16)
    # keys and values as one projection gives them: columns of one matrix
    kv = torch.empty(B, Sk, 2 * Hkv * dh, dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        kv[b] = normal(Sk, 2 * Hkv * dh).to(torch.bfloat16)
    behind = torch.arange(Sk, device="cuda")[None, :] >= length[:, None]
    kv.masked_fill_(behind[..., None], float("nan"))
    s = {"case": c, "q": q, "k": kv[..., :Hkv * dh], "v": kv[..., Hkv * dh:], "length": length if c["ragged"] else None}
    if c["op"] == "cross_bwd":
        s["out"], s["lse2"] = _cross(s)
        s["dout"] = normal(B, Sq, H * dh, std=1e-2).to(torch.bfloat16)
    return s


def run(state):
    s = state
    c = s["case"]
    if own:
        return _own(s, c["op"])
    if c["op"] == "loss":
        return _loss(s)
    if c["op"] == "step":
        return _step(s)
    if c["op"] == "cross":
        return _cross(s)
    return _cross_bwd(s)


def _own(s, op):
    import paper_2401_01728_amd as rv
    from paper_2401_01728_amd import kernels
    c = s["case"]
    if op == "loss":
        return rv.loss_forward(s["x"], s["w"], s["label"])
    if op == "step":
        if c["update"]:
            return rv.loss_step(s["x"], s["w"], s["label"], scale=s["scale"], master=s["master"], eta=s["eta"],
                                master_out=s["master_out"], version=s["version"])
        return rv.loss_step(s["x"], s["w"], s["label"], scale=s["scale"])
    if op == "cross":
        return kernels.cross_attention_fwd(s["q"], s["k"], s["v"], c["H"], c["Hkv"], s["length"])
    return kernels.cross_attention_bwd(s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse2"], c["H"], c["Hkv"], s["length"])


# ---- the plain forms --------------------------------------------------------------------------

def _logits(s):
    takes = (s["label"] >= 0)[:, None]
    x = torch.where(takes, s["x"].float(), 0.0)
    return takes, x, s["w"].float(), s["label"].clamp(min=0)[:, None]


def _softmax_parts(logits):
    top = logits.amax(-1, keepdim=True)
    p = (logits - top).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, top + total.log()


def _loss(s):
    takes, x, w, label = _logits(s)
    logits = x @ w.T
    _, _, lse = _softmax_parts(logits)
    loss = torch.where(takes, lse - logits.gather(1, label), 0.0)
    return loss[:, 0], torch.where(takes, lse, 0.0)[:, 0]


def _step(s):
    takes, x, w, label = _logits(s)
    logits = x @ w.T
    p, total, lse = _softmax_parts(logits)
    at = logits.gather(1, label)
    loss = torch.where(takes, lse - at, 0.0)[:, 0]
    p /= total
    p.scatter_(1, label, torch.expm1(at - lse))          # p - 1, without the difference of two nearly equal values
    p *= torch.where(takes, s["scale"], 0.0)
    dx, dw = (p @ w).to(torch.bfloat16), p.T @ x
    if "master" not in s:
        return loss, dx, dw.to(torch.bfloat16)
    new = s["master"] - s["eta"] * dw
    return loss, dx, new, new.to(torch.bfloat16)


def _heads(t, h):
    """[B, S, h * dh] -> [B, h, S, dh] in 32 bits"""
    return t.float().unflatten(-1, (h, -1)).transpose(1, 2)


def _keys(s):
    c = s["case"]
    k, v = _heads(s["k"], c["Hkv"]), _heads(s["v"], c["Hkv"])
    if s["length"] is None:
        return k, v, None
    seen = (torch.arange(c["Sk"], device=k.device)[None, :] < s["length"][:, None])[:, None, None, :]
    here = seen.transpose(-1, -2)
    return torch.where(here, k, 0.0), torch.where(here, v, 0.0), seen


def _scores2(s, q, k, seen):
    """[B, Hkv, (H / Hkv) * Sq, Sk], of base 2"""
    c = s["case"]
    z = (q.reshape(c["B"], c["Hkv"], -1, c["dh"]) @ k.transpose(-1, -2)) * (math.log2(math.e) / math.sqrt(c["dh"]))
    return z if seen is None else z.masked_fill_(~seen, -math.inf)


def _merge(t, c):
    return t.reshape(c["B"], c["H"], c["Sq"], c["dh"]).transpose(1, 2).reshape(c["B"], c["Sq"], -1)


def _cross(s):
    c = s["case"]
    k, v, seen = _keys(s)
    z = _scores2(s, _heads(s["q"], c["H"]), k, seen)
    top = z.amax(-1, keepdim=True)
    p = (z - torch.where(top == -math.inf, 0.0, top)).exp2_()
    total = p.sum(-1, keepdim=True)
    lse2 = top + total.log2()
    out = (p @ v) / torch.where(total == 0, 1.0, total)
    return _merge(out, c).to(torch.bfloat16), lse2.reshape(c["B"], c["H"], c["Sq"])


def _cross_bwd(s):
    c = s["case"]
    k, v, seen = _keys(s)
    q, o, do = (_heads(s[n], c["H"]).reshape(c["B"], c["Hkv"], -1, c["dh"]) for n in ("q", "out", "dout"))
    z = _scores2(s, q, k, seen)
    lse2 = s["lse2"].reshape(c["B"], c["Hkv"], -1, 1)
    p = (z - torch.where(lse2 == -math.inf, 0.0, lse2)).exp2_()
    ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) / math.sqrt(c["dh"])
    back = lambda t: t.transpose(1, 2).reshape(c["B"], c["Sk"], -1).to(torch.bfloat16)  # noqa: E731
    return _merge(ds @ k, c).to(torch.bfloat16), back(ds.transpose(-1, -2) @ q), back(p.transpose(-1, -2) @ do)


# ---- the definitions, in 64 bits --------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_loss if case["op"] in ("loss", "step") else _exact_cross)(s, case)


def _exact_loss(s, c):
    take = (s["label"] >= 0).nonzero()[:, 0]
    T, d = s["x"].shape
    x = s["x"][take].double().requires_grad_(c["op"] == "step")
    w = s["w"].double().requires_grad_(c["op"] == "step")
    z = torch.nn.functional.linear(x, w)
    each = torch.nn.functional.cross_entropy(z, s["label"][take], reduction="none")
    full = lambda v, *shape: torch.zeros(T, *shape, dtype=torch.float64, device="cuda").index_copy_(0, take, v.detach())  # noqa: E731
    if c["op"] == "loss":
        return full(each), full(torch.logsumexp(z, 1))
    dx, dw = torch.autograd.grad(each.sum() * s["scale"], (x, w))
    if not c["update"]:
        return full(each), full(dx, d), dw
    new = s["master"].double() - s["eta"] * dw
    return full(each), full(dx, d), new, new


def _exact_cross(s, c):
    if c["B"] * c["H"] * c["Sq"] * c["Sk"] > 1 << 30 and c["op"] == "cross_bwd":
        return None
    grads = c["op"] == "cross_bwd"
    q = s["q"].double().requires_grad_(grads)
    n = _lengths(c)
    outs, lses, gq, gk, gv = [], [], [], [], []
    share = c["H"] // c["Hkv"]
    for b in range(c["B"]):
        kb = s["k"][b, :n[b]].double().requires_grad_(grads)
        vb = s["v"][b, :n[b]].double().requires_grad_(grads)
        if n[b] == 0:
            outs.append(torch.zeros(c["Sq"], c["H"] * c["dh"], dtype=torch.float64, device="cuda"))
            lses.append(torch.full((c["H"], c["Sq"]), -math.inf, dtype=torch.float64, device="cuda"))
            got = [torch.zeros_like(t[b], dtype=torch.float64) for t in (s["q"], s["k"], s["v"])]
        else:
            per_head, lse = [], []
            for h in range(c["H"]):
                col, kcol = slice(h * c["dh"], (h + 1) * c["dh"]), slice(h // share * c["dh"], (h // share + 1) * c["dh"])
                z = q[b, :, col] @ kb[:, kcol].T / math.sqrt(c["dh"])
                per_head.append(torch.softmax(z, -1) @ vb[:, kcol])
                lse.append(torch.logsumexp(z.detach(), -1) / math.log(2.0))
            o = torch.cat(per_head, -1)
            outs.append(o.detach())
            lses.append(torch.stack(lse))
            if grads:
                dq, dk, dv = torch.autograd.grad(o, (q, kb, vb), s["dout"][b].double())
                got = [dq[b]] + [torch.cat([t, torch.zeros(c["Sk"] - n[b], t.shape[1], dtype=torch.float64, device="cuda")]) for t in (dk, dv)]
        if grads:
            for to, t in zip((gq, gk, gv), got):
                to.append(t)
    if grads:
        return torch.stack(gq), torch.stack(gk), torch.stack(gv)
    return torch.stack(outs), torch.stack(lses)
