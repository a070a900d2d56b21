"""The proposal block: its gradients against autograd's on the same formulas in
64 bits, one hypothesis at a time against the batch, and training that learns."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(block, poses, states, q_pos, k_pos, kv_len):
    """The block in 64 bits, its parameters as leaves."""
    p = {k: v.double().requires_grad_() for k, v in block.p.items()}
    B, S, _ = poses.shape
    T, W, D, H, G = states.shape[1], block.width, 64, block.heads, block.kv_heads

    def norm(x, w):
        return x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w

    def rotate(x, pos):
        c, s = (block.table[pos.long(), i].double()[:, None] for i in (0, 1))
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    x = poses.double().reshape(B * S, -1) @ p["w_in"] + p["b_in"]
    q = (norm(x, p["n1"]) @ p["w_q"]).view(B * S, H, D)
    kv = (states.double().reshape(B * T, -1) @ p["w_kv"]).view(B * T, 2, G, D)
    q = rotate(norm(q, p["nq"]), q_pos).view(B, S, H, D)
    k = rotate(norm(kv[:, 0], p["nk"]), k_pos).view(B, T, G, D)
    v = kv[:, 1].reshape(B, T, G, D)
    o = []
    for b in range(B):
        n = int(kv_len[b])
        heads = [torch.softmax(q[b, :, h] @ k[b, :n, h * G // H].t() / 8.0, 1) @ v[b, :n, h * G // H] for h in range(H)]
        o.append(torch.stack(heads, 1))
    x1 = torch.stack(o).reshape(B * S, W) @ p["w_o"] + p["b_o"] + x
    z = norm(x1, p["n2"]) @ p["w_1"] + p["b_1"]
    x2 = (z * 0.5 * torch.special.erfc(-z * math.sqrt(0.5))) @ p["w_2"] + p["b_2"] + x1
    return (x2 @ p["w_out"] + p["b_out"]).view(B, S, 8), p


@pytest.mark.parametrize("dtype,u", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
def test_gradients_of_the_block(dtype, u):
    from paper_2210_10108_amd import propose
    block = propose.ProposalBlock(dtype=dtype, seed=3)
    g = torch.Generator("cuda").manual_seed(5)
    B, S, T = 3, 37, 150
    poses = torch.randn(B, S, 16, generator=g, device="cuda").to(dtype)
    states = torch.randn(B, T, 48, generator=g, device="cuda").to(dtype)
    q_pos = torch.randint(0, 99, (B * S,), generator=g, device="cuda", dtype=torch.int32)
    k_pos = torch.arange(B * T, device="cuda", dtype=torch.int32)
    kv_len = torch.tensor([150, 64, 9], dtype=torch.int32, device="cuda")
    dy = torch.randn(B, S, 8, generator=g, device="cuda").to(dtype)
    y, kept = block.forward(poses, states, q_pos, k_pos, kv_len=kv_len, keep=True)
    grads = block.backward(dy, kept)
    ref, p = reference(block, poses, states, q_pos, k_pos, kv_len)
    want = torch.autograd.grad((ref * dy.double()).sum(), list(p.values()))
    # about 12 roundings of a 16-bit tensor lie between a parameter and the result, each
    # u relative at most; in the 2-norm they add up as the root of their number, with a
    # factor of 4 for what the block's products and norms may raise them by
    bound = 4 * math.sqrt(12) * u

    def off(a, b):
        return float((a.double() - b).norm() / b.norm())
    assert off(y, ref.detach()) <= bound
    for (name, _), w in zip(p.items(), want):
        assert off(grads[name], w) <= bound, (name, off(grads[name], w), bound)
    # one hypothesis at a time, over the states that are there already
    for b in range(B):
        one = block.forward(poses[b:b + 1, 5:6].contiguous(), states[b:b + 1], q_pos[b * S + 5:b * S + 6],
                            k_pos[b * T:(b + 1) * T], kv_len=kv_len[b:b + 1])
        assert off(one[0, 0], ref[b, 5].detach()) <= bound


def test_proposals_learn():
    from paper_2210_10108_amd import propose
    views = propose.Views("tiny_bump")
    block = propose.ProposalBlock(state_dim=views.state_dim)
    losses = propose.train(block, views, 60)
    assert np.isfinite(losses).all()
    assert np.mean(losses[-10:]) < 0.5 * losses[0], (losses[0], losses[-10:])
    views.field.close()
