"""The proposal block with layer norms and patch positions: its gradients against
autograd's on the same formulas in 64 bits, proposals from states kept in 16 and 8
bits, and a training step with clipped gradients."""
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
    axis = torch.tensor(list(block.pair_axis), device="cuda")

    def layer_norm(x, w, b):
        d = x - x.mean(-1, keepdim=True)
        return d / torch.sqrt(d.square().mean(-1, keepdim=True) + 1e-5) * w + b

    def heads(x, w, pos):
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        at, pairs = pos.long()[:, axis], torch.arange(D // 2, device="cuda")
        c, s = (block.table[at, i, pairs].double()[:, None] for i in (0, 1))
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    x = poses.double().reshape(B * S, -1) @ p["w_in"] + p["b_in"]
    q = (layer_norm(x, p["n1"], p["c1"]) @ p["w_q"]).view(B * S, H, D)
    kv = (states.double().reshape(B * T, -1) @ p["w_kv"]).view(B * T, 2, G, D)
    q = heads(q, p["nq"], q_pos).view(B, S, H, D)
    k = heads(kv[:, 0], p["nk"], k_pos).view(B, T, G, D)
    v = kv[:, 1].reshape(B, T, G, D)
    o = []
    for b in range(B):
        n = int(kv_len[b])
        one = [torch.softmax(q[b, :, h] @ k[b, :n, h * G // H].t() / 8.0, 1) @ v[b, :n, h * G // H] for h in range(H)]
        o.append(torch.stack(one, 1))
    x1 = torch.stack(o).reshape(B * S, W) @ p["w_o"] + p["b_o"] + x
    z = layer_norm(x1, p["n2"], p["c2"]) @ p["w_1"] + p["b_1"]
    x2 = (z * 0.5 * torch.special.erfc(-z * math.sqrt(0.5))) @ p["w_2"] + p["b_2"] + x1
    return (x2 @ p["w_out"] + p["b_out"]).view(B, S, 8), p


def inputs(dtype, B=3, S=37, T=150):
    g = torch.Generator("cuda").manual_seed(5)
    poses = torch.randn(B, S, 16, generator=g, device="cuda").to(dtype)
    states = torch.randn(B, T, 48, generator=g, device="cuda").to(dtype)
    q_pos = torch.randint(0, 99, (B * S, 2), generator=g, device="cuda", dtype=torch.int32)
    patch = torch.arange(T, device="cuda")
    k_pos = torch.stack([patch // 15, patch % 15], 1).int().repeat(B, 1)
    kv_len = torch.tensor([T, 64, 9], dtype=torch.int32, device="cuda")
    return poses, states, q_pos, k_pos, kv_len, torch.randn(B, S, 8, generator=g, device="cuda").to(dtype)


def off(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("width", [256, 512])
@pytest.mark.parametrize("dtype,u", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
def test_gradients_of_the_image_block(dtype, u, width):
    from paper_2210_10108_amd import propose
    block = propose.ProposalBlock(width=width, dtype=dtype, seed=3, image=True)
    poses, states, q_pos, k_pos, kv_len, dy = inputs(dtype)
    y, kept = block.forward(poses, states, q_pos, k_pos, kv_len=kv_len, keep=True)
    grads = block.backward(dy, kept)
    ref, p = reference(block, poses, states, q_pos, k_pos, kv_len)
    want = torch.autograd.grad((ref * dy.double()).sum(), list(p.values()))
    # about 12 roundings of a 16-bit tensor lie between a parameter and the result, each
    # u relative at most; in the 2-norm they add up as the root of their number, with a
    # factor of 4 for what the block's products and norms may raise them by
    bound = 4 * math.sqrt(12) * u
    assert off(y, ref.detach()) <= bound
    assert set(grads) == set(p)
    for (name, _), w in zip(p.items(), want):
        assert off(grads[name], w) <= bound, (name, off(grads[name], w), bound)
    # from states that were made before
    enc = block.encode(states, k_pos)
    assert off(block.propose(poses, enc, q_pos, kv_len=kv_len), ref.detach()) <= bound
    for b in range(3):
        one = block.propose(poses[b:b + 1, 5:6].contiguous(), [t[b:b + 1] for t in enc], q_pos[b * 37 + 5:b * 37 + 6],
                            kv_len=kv_len[b:b + 1])
        assert off(one[0, 0], ref[b, 5].detach()) <= bound


@pytest.mark.parametrize("image", [True, False])
@pytest.mark.parametrize("dtype,u", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
def test_proposals_from_8_bit_states(dtype, u, image):
    # the block with the states that the 8-bit ones stand for, and nothing else changed
    from paper_2210_10108_amd import propose
    block = propose.ProposalBlock(dtype=dtype, seed=3, image=image)
    poses, states, q_pos, k_pos, kv_len, _ = inputs(dtype)
    if not image:
        q_pos, k_pos = q_pos[:, 0].contiguous(), torch.arange(len(k_pos), device="cuda", dtype=torch.int32)
    packed = block.encode(states, k_pos, kv_len=kv_len, bits=8)
    y = block.propose(poses, packed, q_pos, kv_len=kv_len)
    wide = [(x.float() * s.repeat_interleave(64, 1)[:, :x.shape[1], :, None]).to(dtype)
            for x, s in zip(packed[:2], packed[2:])]  # exact: e4m3 times a power of two
    want = block.propose(poses, wide, q_pos, kv_len=kv_len)
    # the attentions' results differ by a rounding each, and what follows rounds 6 times
    assert off(y, want.double()) <= 4 * math.sqrt(12) * u
    # one at a time
    one = block.propose(poses[:1, :1].contiguous(), [t[:1] for t in packed], q_pos[:1], kv_len=kv_len[:1])
    assert off(one[0, 0], y[0, 0].double()) <= 4 * math.sqrt(12) * u


def test_image_block_trains_with_clipped_gradients():
    from paper_2210_10108_amd import propose
    views = propose.Views("tiny_bump")
    for max_norm in (math.inf, 1.0):
        block = propose.ProposalBlock(state_dim=views.state_dim, image=True)
        before = {k: v.clone() for k, v in block.master.items()}
        losses = propose.train(block, views, 3, max_norm=max_norm)
        assert len(losses) == 3 and np.isfinite(losses).all()
        assert all(bool(torch.isfinite(v).all()) and not torch.equal(v, before[k]) for k, v in block.master.items() if k != "b_out")
    q_pos, k_pos = views.patch_positions(2, 5)
    h = views.w.height // views.patch
    assert q_pos.shape == (10, 2) and k_pos.shape == (2 * views.tokens, 2)
    assert int(k_pos[:, 0].max()) == h - 1 and torch.equal(k_pos[:views.tokens], k_pos[views.tokens:])
    views.field.close()
