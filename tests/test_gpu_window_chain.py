"""Rotary positions, norms of heads, a cache and attention over a window together: between two stages of a chain that is trained, and token by token over
a ring as it is served.

Bars: the stages' own parity bars are 2e-2 (normwise, their bf16 activations and gradients), and the operators between them add roundings of 2^-8 each:
3e-2 for what has passed through everything.  Serving reads keys that are bit for bit the training's; probabilities and results are rounded once each
(2^-8), in two orders of additions: 1e-2."""
import math

import numpy as np
import pytest
import torch

import paper_2401_01728_amd as rv
from oracle import stage as ostage
from paper_2401_01728_amd import kernels
from paper_2401_01728_amd.inputs import gen
from util import bf16_normal, close, dev, host64

pytestmark = pytest.mark.gpu


def _params(seed, L, d, f):
    per = 4 * d * d + 2 * d * f + 9 * d + f
    w = gen.normal_f32(seed, 0, L * per, 0.0, 0.02)
    for l in range(L):
        w[l * per:l * per + d] += np.float32(1.0)
        o = l * per + 2 * d + 3 * d * d + 3 * d + d * d + d
        w[o:o + d] += np.float32(1.0)
    return w


def _project(x, w):
    T, d = x.shape
    out = torch.empty(T, w.shape[1], dtype=torch.bfloat16, device="cuda")
    bias = torch.zeros(w.shape[1], dtype=torch.bfloat16, device="cuda")
    return kernels.gemm_bf16(x, 0, w, 1, T, w.shape[1], d, kernels.EPI_BF16_BIAS, out, bias=bias)


def _definition(a, w, gq, gk, freq, H, Hkv, dh, window, sinks):
    """[B, S, d] in 64 bits -> what the attention adds to it."""
    B, S, _ = a.shape
    qkv = a @ w
    angle = torch.arange(S, dtype=torch.float64)[:, None] * freq

    def head(x, g):
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * g
        p, q = x[..., :dh // 2], x[..., dh // 2:]
        return torch.cat([p * angle.cos() - q * angle.sin(), q * angle.cos() + p * angle.sin()], -1)

    p, j = torch.arange(S)[:, None], torch.arange(S)[None, :]
    hide = ~((j <= p) & ((j > p - window) | (j < sinks)))
    out = []
    for h in range(H):
        kv = h // (H // Hkv)
        q = head(qkv[..., h * dh:(h + 1) * dh], gq)
        k = head(qkv[..., (H + kv) * dh:(H + kv + 1) * dh], gk)
        v = qkv[..., (H + Hkv + kv) * dh:(H + Hkv + kv + 1) * dh]
        out.append(torch.softmax((q @ k.transpose(-1, -2) / math.sqrt(dh)).masked_fill(hide, -math.inf), -1) @ v)
    return torch.cat(out, -1)


def test_chain_with_window_attention():
    L, d, H, Hkv, f, S, mb, V, eta, window, sinks = 1, 128, 2, 1, 256, 128, 2, 300, 1e-2, 24, 2
    dh = d // H
    stages = [rv.Stage.decoder(L, d, H, f, S, mb, 0, eta, keep_grad=True) for _ in range(2)]
    oracles = []
    for i, st in enumerate(stages):
        w = _params(60 + i, L, d, f)
        st.set_params(dev(w))
        oracles.append(ostage.Stage("decoder", 0, eta, w, n_blocks=L, d=d, h=H, f=f))
    x, x64 = bf16_normal(61, 1, (mb, S, d))
    wq, wq64 = bf16_normal(61, 2, (d, (H + 2 * Hkv) * dh), std=0.1)
    gq, gq64 = bf16_normal(61, 3, (dh,), mean=1.0, std=0.1)
    gk, gk64 = bf16_normal(61, 4, (dh,), mean=1.0, std=0.1)
    head, head64 = bf16_normal(61, 5, (V, d), std=0.1)
    label = torch.from_numpy(np.random.default_rng(6).integers(0, V, mb * S))
    freq = kernels.rotary_frequencies(dh)[0]
    norms = dict(gamma_q=gq, gamma_k=gk, eps=1e-6)

    a = stages[0].forward(0, x)
    qkv = _project(a.reshape(mb * S, d), wq).view(mb, S, -1)
    q, k, v = qkv[..., :H * dh], qkv[..., H * dh:(H + Hkv) * dh], qkv[..., (H + Hkv) * dh:]
    q2, k2 = kernels.rotary_fwd(q, k, freq.cuda(), H, Hkv, **norms)
    o, lse2 = kernels.window_attention_fwd(q2, k2, v, H, Hkv, window, sinks)
    mid = (a.float() + o.float()).to(torch.bfloat16)
    y = stages[1].forward(0, mid)
    loss, dy, dhead = rv.loss_step(y.reshape(mb * S, d), head, label.cuda(), scale=1.0 / (mb * S))
    dmid = stages[1].backward(0, dy.reshape(mb, S, d))
    # the gradients of q, k and v as columns of one matrix, turned back in place
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = dqkv[..., :H * dh], dqkv[..., H * dh:(H + Hkv) * dh], dqkv[..., (H + Hkv) * dh:]
    kernels.window_attention_bwd(q2, k2, v, o, dmid, lse2, H, Hkv, window, sinks, dq=dq, dk=dk, dv=dv)
    _, _, dgq, dgk = kernels.rotary_bwd(dq, dk, freq.cuda(), H, Hkv, q=q, k=k, dq=dq, dk=dk, **norms)
    back = torch.empty(mb * S, d, dtype=torch.bfloat16, device="cuda")
    kernels.gemm_bf16(dqkv.view(mb * S, -1), 0, wq, 0, mb * S, d, wq.shape[1], kernels.EPI_BF16, back)
    da = (dmid.float() + back.view(mb, S, d).float()).to(torch.bfloat16)
    dx = stages[0].backward(0, da)

    a64 = torch.from_numpy(oracles[0].forward(0, x64)).requires_grad_()
    leaves = [torch.from_numpy(t).requires_grad_() for t in (wq64, gq64, gk64)]
    mid64 = a64 + _definition(a64, *leaves, freq, H, Hkv, dh, window, sinks)
    y64 = torch.from_numpy(oracles[1].forward(0, mid64.detach().numpy())).requires_grad_()
    head_t = torch.from_numpy(head64).requires_grad_()
    each = torch.nn.functional.cross_entropy(y64.reshape(mb * S, d) @ head_t.T, label, reduction="none")
    dy64, dhead64 = torch.autograd.grad(each.mean(), (y64, head_t))
    dmid64 = torch.from_numpy(oracles[1].backward(0, dy64.numpy()))
    da64, _, dgq64, dgk64 = torch.autograd.grad(mid64, (a64, *leaves), dmid64)
    dx64 = oracles[0].backward(0, da64.numpy())

    grp = "chain with window attention and loss, bar 3e-2"
    close(host64(mid), mid64.detach().numpy(), 3e-2, "mid", group=grp)
    close(host64(loss), each.detach().numpy(), 3e-2, "loss", group=grp)
    close(host64(dhead), dhead64.numpy(), 3e-2, "dhead", group=grp)
    close(host64(dgq), dgq64.numpy(), 3e-2, "dgamma_q", group=grp)
    close(host64(dgk), dgk64.numpy(), 3e-2, "dgamma_k", group=grp)
    close(host64(dx), dx64, 3e-2, "dx", group=grp)


# prompts that fill the ring partly and several times over, sinks or none, in chunks and tokens
@pytest.mark.parametrize("H,Hkv,dh,window,sinks,prompt,more,layout", [(4, 2, 64, 40, 4, 100, 30, "half"), (8, 1, 128, 33, 0, 20, 25, "pairs"), (3, 3, 64, 64, 1, 7, 90, "half")])
def test_serving_over_a_ring_is_what_training_sees(H, Hkv, dh, window, sinks, prompt, more, layout):
    B, chunk = 2, 16
    S, rows = prompt + more, sinks + window + chunk - 1
    qkv, _ = bf16_normal(70, 1, (B, S, (H + 2 * Hkv) * dh))
    gq, _ = bf16_normal(70, 2, (dh,), mean=1.0, std=0.1)
    freq, amplitude = kernels.rotary_frequencies(dh, rule="parts", factor=4.0, context=64.0)
    q, k, v = qkv[..., :H * dh], qkv[..., H * dh:(H + Hkv) * dh], qkv[..., (H + Hkv) * dh:]
    how = dict(layout=layout, amplitude=amplitude, gamma_q=gq, gamma_k=gq)
    q2, k2 = kernels.rotary_fwd(q, k, freq.cuda(), H, Hkv, **how)
    ref, ref_lse = kernels.window_attention_fwd(q2, k2, v, H, Hkv, window, sinks)
    cache = [torch.full((B, rows, Hkv * dh), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out, lse, at = [], [], 0
    while at < S:
        n = min(chunk, prompt - at) if at < prompt else 1
        start = torch.full((B,), at, dtype=torch.int32, device="cuda")
        some = [t[:, at:at + n].contiguous() for t in (q, k, v)]
        turned, keys, values = kernels.rotary_fwd(some[0], some[1], freq.cuda(), H, Hkv, v=some[2], cache=cache, sinks=sinks, start=start, **how)
        assert torch.equal(turned, q2[:, at:at + n])
        o, l2 = kernels.window_attention_fwd(turned, keys, values, H, Hkv, window, sinks, start)
        out.append(o)
        lse.append(l2)
        at += n
    close(host64(torch.cat(out, 1)), host64(ref), 1e-2, "served", group="tokens over a ring against training, bar 1e-2")
    assert float((torch.cat(lse, 2) - ref_lse).abs().max()) <= 2.0 ** -11
