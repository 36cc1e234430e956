"""The operators together, as a chain of decoder peers is trained with them on pairs of texts: two stages with cross-attention to an
encoder's states between them and the loss behind, against the same chain in 64 bits.

Bars: the two stages' own parity bars are 2e-2 (normwise, their bf16 activations and gradients), and the operators between them add roundings of
2^-8 each: 3e-2 for what has passed through everything."""
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


def test_chain_with_cross_attention_and_loss():
    L, d, H, Hkv, f, S, mb, Sk, V, eta = 1, 128, 2, 1, 256, 64, 2, 77, 501, 1e-2
    dh = d // H
    stages = [rv.Stage.decoder(L, d, H, f, S, mb, 0, eta, keep_grad=True) for _ in range(2)]
    oracles = []
    for i, st in enumerate(stages):
        w = _params(40 + i, L, d, f)
        st.set_params(dev(w))
        oracles.append(ostage.Stage("decoder", 0, eta, w, n_blocks=L, d=d, h=H, f=f))
    x, x64 = bf16_normal(41, 1, (mb, S, d))
    kv, kv64 = bf16_normal(41, 2, (mb, Sk, 2 * Hkv * dh))
    klen = [77, 30]
    kv[1, 30:] = float("nan")
    master32 = gen.normal_f32(41, 3, V * d, 0.0, 0.1).reshape(V, d)
    master = dev(master32)
    head = master.to(torch.bfloat16)
    head64 = host64(head)
    label = torch.from_numpy(np.random.default_rng(5).integers(0, V, mb * S))
    label[:20] = -1                                        # a prompt
    kept = int((label >= 0).sum())
    length = torch.tensor(klen, dtype=torch.int32, device="cuda")

    # forward: stage 0, + cross-attention, stage 1, loss with its gradient and the head's update; then the way back
    a = stages[0].forward(0, x)
    c, lse2 = kernels.cross_attention_fwd(a, kv[..., :Hkv * dh], kv[..., Hkv * dh:], H, Hkv, length)
    mid = (a.float() + c.float()).to(torch.bfloat16)
    y = stages[1].forward(0, mid)
    loss, dy, new, version = rv.loss_step(y.reshape(mb * S, d), head, label.cuda(), scale=1.0 / kept, master=master, eta=eta)
    dmid = stages[1].backward(0, dy.reshape(mb, S, d))
    dq, dk, dv = kernels.cross_attention_bwd(a, kv[..., :Hkv * dh], kv[..., Hkv * dh:], c, dmid, lse2, H, Hkv, length)
    da = (dmid.float() + dq.float()).to(torch.bfloat16)
    dx = stages[0].backward(0, da)

    # the same in 64 bits
    a64 = torch.from_numpy(oracles[0].forward(0, x64)).requires_grad_()
    kv_t = torch.from_numpy(np.nan_to_num(kv64)).requires_grad_()
    out = []
    for b in range(mb):
        heads = []
        for h in range(H):
            kh = kv_t[b, :klen[b], :dh]
            p = torch.softmax(a64[b, :, h * dh:(h + 1) * dh] @ kh.T / math.sqrt(dh), -1)
            heads.append(p @ kv_t[b, :klen[b], dh:])
        out.append(torch.cat(heads, -1))
    mid64 = a64 + torch.stack(out)
    y64 = torch.from_numpy(oracles[1].forward(0, mid64.detach().numpy())).requires_grad_()
    head_t = torch.from_numpy(head64).requires_grad_()
    z = y64.reshape(mb * S, d) @ head_t.T
    each = torch.nn.functional.cross_entropy(z, label, ignore_index=-1, reduction="none")
    dy64, dhead = torch.autograd.grad(each.sum() / kept, (y64, head_t))
    dmid64 = torch.from_numpy(oracles[1].backward(0, dy64.numpy()))
    da64, dkv = torch.autograd.grad(mid64, (a64, kv_t), dmid64)
    dx64 = oracles[0].backward(0, da64.numpy())

    grp = "chain with cross-attention and loss, bar 3e-2"
    close(host64(loss), each.detach().numpy(), 3e-2, "loss", group=grp)
    close(host64(dy), dy64.reshape(mb * S, d).numpy(), 3e-2, "dy", group=grp)
    close(master32 - host64(new), eta * dhead.numpy(), 3e-2, "head step", group=grp)
    assert torch.equal(version, new.to(torch.bfloat16))
    close(host64(dk), dkv[..., :dh].numpy(), 3e-2, "dk", group=grp)
    close(host64(dv), dkv[..., dh:].numpy(), 3e-2, "dv", group=grp)
    close(host64(dx), dx64, 3e-2, "dx", group=grp)
    for st, o in zip(stages, oracles):
        close(host64(st.last_grad()), o.last_grad, 3e-2, "parameters", group=grp)
