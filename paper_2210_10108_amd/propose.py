"""Pose proposals: a small network that reads the observed image and moves each
pose hypothesis towards it before the optimisation starts (Sec. IV-B starts
from random hypotheses).

The network is one decoder block whose tokens are the hypotheses and whose
encoder's states are the image's patches, made of the layer operators alone:

  h  = norm(x)                       q = h Wq          (k, v) = states Wkv
  q', k' = norm and rotation of every head at its position
  x1 = cross attention(q', k', v) Wo + bo + x
  x2 = gelu(norm(x1) W1 + b1) W2 + b2 + x1,   correction = x2 Wout + bout

ProposalBlock runs it forward, for a batch of hypotheses or one at a time, and
backward.  With image=True its token norms are layer norms, heads turn by a
patch's row and column, and an image's keys and values can be made once
(encode, in 16 or 8 bits) for any number of proposals (propose).
`python -m paper_2210_10108_amd.propose` trains it on views of a synthetic field
and reports how far the hypotheses are from the true pose before and after;
--image trains it that way, its gradients clipped, and proposes from states in
8 bits.  The proposals are poses as Field.render_loss_grad takes them;
the optimisation itself is not run here.
"""
from __future__ import annotations

import argparse
import math

import numpy as np

from . import layers as L
from . import pnerf, synth

POSE_FEATURES = 16  # a pose's 12 numbers, padded to a whole chunk


class ProposalBlock:
    """The block's parameters (float32 masters and copies in `dtype`) and its
    passes.  width: a multiple of 64, up to 256 (the heads' norm) but for image;
    heads of 64, kv_heads of which the states have; state_dim: features of a patch.
    image: layer norms, and positions are (row, column), [tokens, 2]: the first
    half of the pairs turns by the row, the second by the column, each half with
    all of the frequencies."""

    def __init__(self, width=256, kv_heads=2, state_dim=48, n_positions=4096, dtype=None, seed=0,
                 device="cuda", image=False):
        import torch
        self.image = image
        self.width, self.heads, self.kv_heads, self.D = width, width // 64, kv_heads, 64
        self.dtype = dtype or torch.bfloat16
        g = torch.Generator(device).manual_seed(seed)

        def matrix(k, n, gain=1.0):
            return torch.randn(k, n, generator=g, device=device) * (gain / math.sqrt(k))
        kv = 2 * kv_heads * self.D
        one, zero = torch.ones, torch.zeros
        self.master = {
            "w_in": matrix(POSE_FEATURES, width), "b_in": zero(width, device=device),
            "n1": one(width, device=device), "w_q": matrix(width, width), "w_kv": matrix(state_dim, kv),
            "nq": one(self.D, device=device), "nk": one(self.D, device=device),
            "w_o": matrix(width, width, 0.5), "b_o": zero(width, device=device),
            "n2": one(width, device=device), "w_1": matrix(width, 4 * width),
            "b_1": zero(4 * width, device=device), "w_2": matrix(4 * width, width, 0.5),
            "b_2": zero(width, device=device), "w_out": matrix(width, 8, 0.1),
            "b_out": zero(8, device=device)}
        pairs = self.D // 2
        freq = 10000.0 ** (-torch.arange(pairs, device=device, dtype=torch.float64) / pairs)
        if image:
            self.master.update(c1=zero(width, device=device), c2=zero(width, device=device))
            self.pair_axis = bytes(2 * j // pairs for j in range(pairs))
            freq = freq[::2].repeat(2)
        angle = torch.arange(n_positions, device=device, dtype=torch.float64)[:, None] * freq
        self.table = torch.stack([angle.cos(), angle.sin()], 1).float()
        self.refresh()

    def refresh(self):
        """The parameters as the operators take them, after a change of the masters."""
        self.p = {k: v.to(self.dtype) for k, v in self.master.items()}

    def _norm(self, x, i):
        w = self.p[f"n{i}"]
        if self.image:
            return L.layer_norm(x, w, self.p[f"c{i}"])
        return L.norm_rotate(x[:, None], None, w, None, None, None, None)[0][:, 0]

    def _norm_backward(self, dy, x, i, dres, g):
        """The gradient of the norm's argument, dres (what reaches it past the norm) included."""
        w = self.p[f"n{i}"]
        if self.image:
            dx, g[f"n{i}"], g[f"c{i}"] = L.layer_norm_backward(dy, x, w, residual_grad=dres, dx=dres)
            return dx
        dn, _, g[f"n{i}"], _ = L.norm_rotate_backward(dy[:, None], None, x[:, None], None, w, None, None, None, None)
        return dres.add_(dn[:, 0])

    def _heads(self, q, k, q_pos, k_pos):
        """Heads normed and turned; k may be None."""
        p, wk = self.p, None if k is None else self.p["nk"]
        if self.image:
            return L.rotate_axes(q, k, self.table, q_pos, k_pos, self.pair_axis, p["nq"], wk, eps=1e-6)
        return L.norm_rotate(q, k, p["nq"], wk, self.table, q_pos, k_pos)

    def encode(self, states, k_pos, kv_len=None, kv_mask=None, bits=16):
        """An image's keys and values for propose: (k, v) of states [B, T, state_dim],
        or with bits=8 (k8, v8, k_scale, v_scale), which take half the memory.  (Not less
        time, with these heads of 64: 64 hypotheses over 300 patches, attention 10.4 us
        where 16 bits take 8.5; over one set of 131109 states a single one 17 and 21.)"""
        B, T, _ = states.shape
        kv = L.linear(states.reshape(B * T, -1), self.p["w_kv"]).view(B * T, 2, self.kv_heads, self.D)
        if self.image:
            k, _ = L.rotate_axes(kv[:, 0], None, self.table, k_pos, None, self.pair_axis, self.p["nk"], eps=1e-6)
        else:
            k, _ = L.norm_rotate(kv[:, 0], None, self.p["nk"], None, self.table, k_pos, None)
        k, v = k.view(B, T, self.kv_heads, self.D), kv.view(B, T, 2, self.kv_heads, self.D)[:, :, 1]
        return (k, v) if bits == 16 else L.quantize_states(k, v, kv_len=kv_len, kv_mask=kv_mask)

    def propose(self, poses, encoded, q_pos, kv_len=None, kv_mask=None):
        """Corrections [B, S, 8] of poses [B, S, POSE_FEATURES] for states that encode made."""
        p, W, D = self.p, self.width, self.D
        B, S, _ = poses.shape
        x = L.linear(poses.reshape(B * S, -1), p["w_in"], p["b_in"])
        q = L.linear(self._norm(x, 1), p["w_q"]).view(B * S, self.heads, D)
        qa = self._heads(q, None, q_pos, None)[0].view(B, S, self.heads, D)
        attend = L.cross_attention if len(encoded) == 2 else L.cross_attention_q8
        o = attend(qa, *encoded, kv_len=kv_len, kv_mask=kv_mask)
        x1 = L.linear(o.view(B * S, W), p["w_o"], p["b_o"], x)
        u = L.linear(self._norm(x1, 2), p["w_1"], p["b_1"], activation="gelu")
        x2 = L.linear(u, p["w_2"], p["b_2"], x1)
        return L.linear(x2, p["w_out"], p["b_out"]).view(B, S, 8)

    def forward(self, poses, states, q_pos, k_pos, kv_len=None, kv_mask=None, keep=False):
        """poses [B, S, POSE_FEATURES], states [B, T, state_dim] (of `dtype`),
        positions int32 [B * S] and [B * T] (image: [B * S, 2] and [B * T, 2]):
        corrections [B, S, 8], of which 6 are used (rotation, translation); keep: also what backward needs."""
        p, W, D = self.p, self.width, self.D
        (B, S, _), T = poses.shape, states.shape[1]
        st = states.reshape(B * T, -1)
        x = L.linear(poses.reshape(B * S, -1), p["w_in"], p["b_in"])
        h = self._norm(x, 1)
        q = L.linear(h, p["w_q"]).view(B * S, self.heads, D)
        kv = L.linear(st, p["w_kv"]).view(B * T, 2, self.kv_heads, D)
        qr, kr = self._heads(q, kv[:, 0], q_pos, k_pos)
        qa, ka, va = (qr.view(B, S, self.heads, D), kr.view(B, T, self.kv_heads, D),
                      kv.view(B, T, 2, self.kv_heads, D)[:, :, 1])
        o, lse = L.cross_attention(qa, ka, va, kv_len=kv_len, kv_mask=kv_mask, return_lse=True)
        x1 = L.linear(o.view(B * S, W), p["w_o"], p["b_o"], x)
        h2 = self._norm(x1, 2)
        u, z = L.linear(h2, p["w_1"], p["b_1"], activation="gelu", return_preact=True)
        x2 = L.linear(u, p["w_2"], p["b_2"], x1)
        y = L.linear(x2, p["w_out"], p["b_out"]).view(B, S, 8)
        if not keep:
            return y
        return y, (poses, st, q_pos, k_pos, kv_len, kv_mask, x, h, q, kv, qa, ka, va, o, lse, x1, h2, u, z, x2)

    def backward(self, dy, kept):
        """Gradients of every parameter for dy = dL/d(corrections)."""
        import torch
        poses, st, q_pos, k_pos, kv_len, kv_mask, x, h, q, kv, qa, ka, va, o, lse, x1, h2, u, z, x2 = kept
        p, g, W = self.p, {}, self.width
        B, S, T = qa.shape[0], qa.shape[1], ka.shape[1]
        dx2, g["w_out"], g["b_out"] = L.linear_backward(dy.view(B * S, 8), x2, p["w_out"])
        du, g["w_2"], g["b_2"] = L.linear_backward(dx2, u, p["w_2"])
        dh2, g["w_1"], g["b_1"] = L.linear_backward(du, h2, p["w_1"], z, activation="gelu")
        dx1 = self._norm_backward(dh2, x1, 2, dx2, g)
        do, g["w_o"], g["b_o"] = L.linear_backward(dx1, o.view(B * S, W), p["w_o"])
        dkv = torch.empty_like(kv)  # the keys' and the values' gradients side by side
        side = dkv.view(B, T, 2, self.kv_heads, self.D)
        dq, dk, _ = L.cross_attention_backward(do.view_as(o), qa, ka, va, o, lse, kv_len=kv_len,
                                               kv_mask=kv_mask, dk=side[:, :, 0], dv=side[:, :, 1])
        if self.image:
            dq, _, g["nq"], g["nk"] = L.rotate_axes_backward(
                dq.view(q.shape), dkv[:, 0], q, kv[:, 0], self.table, q_pos, k_pos, self.pair_axis, p["nq"], p["nk"],
                eps=1e-6, dk=dkv[:, 0])
        else:
            dq, _, g["nq"], g["nk"] = L.norm_rotate_backward(
                dq.view(q.shape), dkv[:, 0], q, kv[:, 0], p["nq"], p["nk"], self.table, q_pos, k_pos, dk=dkv[:, 0])
        _, g["w_kv"], _ = L.linear_backward(dkv.view(B * T, -1), st, p["w_kv"], bias=False)
        dh, g["w_q"], _ = L.linear_backward(dq.view(B * S, W), h, p["w_q"], bias=False)
        dx = self._norm_backward(dh, x, 1, dx1, g)
        _, g["w_in"], g["b_in"] = L.linear_backward(dx, poses.reshape(B * S, -1), p["w_in"])
        return g


# ---------------------------------------------------------------- poses and views
def corrections(poses, target):
    """(w, t) with Exp(w) R = R_target, o + t = o_target, of poses [..., 3, 4]."""
    R = target[..., :3] @ np.swapaxes(poses[..., :3], -1, -2)
    c = np.clip((np.trace(R, axis1=-2, axis2=-1) - 1) / 2, -1, 1)
    a = np.arccos(c)
    v = np.stack([R[..., 2, 1] - R[..., 1, 2], R[..., 0, 2] - R[..., 2, 0], R[..., 1, 0] - R[..., 0, 1]], -1)
    w = v * (a / np.maximum(2 * np.sin(a), 1e-8))[..., None]
    return np.concatenate([w, target[..., 3] - poses[..., 3]], -1)


def corrected(poses, c):
    """poses moved by corrections (w, t)."""
    w, out = c[..., :3], poses.copy()
    a = np.linalg.norm(w, axis=-1)[..., None, None]
    K = np.zeros(w.shape[:-1] + (3, 3))
    K[..., 2, 1], K[..., 0, 2], K[..., 1, 0] = w[..., 0], w[..., 1], w[..., 2]
    K = K - np.swapaxes(K, -1, -2)
    s = np.where(a > 1e-8, np.sin(a) / np.maximum(a, 1e-8), 1.0)
    t = np.where(a > 1e-8, (1 - np.cos(a)) / np.maximum(a * a, 1e-16), 0.5)
    out[..., :3] = (np.eye(3) + s * K + t * (K @ K)) @ poses[..., :3]
    out[..., 3] += c[..., 3:6]
    return out


class Views:
    """Batches of observed views of a field: their patches, hypotheses around
    their poses and the corrections that lead to them."""

    def __init__(self, workload="tiny_bump", patch=4, seed=0):
        self.w, self.patch = synth.WORKLOADS[workload], patch
        self.field = pnerf.Field(synth.field_spec(self.w, synth.make_field(self.w, seed)))
        self.intr = synth.intrinsics(self.w)
        self.gt = synth.ground_truth_pose(self.w, seed)
        self.tokens = (self.w.width // patch) * (self.w.height // patch)
        self.state_dim = 3 * patch * patch

    def batch(self, B, S, seed, dtype):
        import torch
        w, n = self.w, self.w.width * self.w.height
        views = synth.perturb_poses(self.gt, B, w.max_rot_deg, w.max_trans, seed)
        hyps = np.stack([synth.perturb_poses(v, S, w.max_rot_deg, w.max_trans, seed * 1000 + i)
                         for i, v in enumerate(views)])
        pix = torch.arange(n, dtype=torch.int32, device="cuda").repeat(B, 1)
        rgb = self.field.render(torch.from_numpy(views.astype(np.float32)).cuda(), pix, self.intr)
        h, v, p = w.height // self.patch, w.width // self.patch, self.patch
        states = rgb.view(B, h, p, v, p, 3).permute(0, 1, 3, 2, 4, 5).reshape(B, h * v, -1)
        feat = np.zeros((B, S, POSE_FEATURES), np.float32)
        feat[..., :12] = (hyps - self.gt).reshape(B, S, 12) * 4
        target = corrections(hyps, views[:, None])
        q_pos = torch.zeros(B * S, dtype=torch.int32, device="cuda")
        k_pos = torch.arange(h * v, dtype=torch.int32, device="cuda").repeat(B)
        return (torch.from_numpy(feat).cuda().to(dtype), ((states - 0.5) * 2).to(dtype), q_pos, k_pos,
                torch.from_numpy(target.astype(np.float32)).cuda(), hyps, views)


    def patch_positions(self, B, S):
        """(row, column) of B * S hypotheses (the origin) and of the patches of B views."""
        import torch
        h, v = self.w.height // self.patch, self.w.width // self.patch
        patch = torch.arange(h * v, dtype=torch.int32, device="cuda")
        return (torch.zeros(B * S, 2, dtype=torch.int32, device="cuda"),
                torch.stack([patch // v, patch % v], 1).int().repeat(B, 1))


def train(block, views, steps, B=16, S=64, lr=2e-3, report=None, max_norm=None):
    """Adam on the mean squared error of the corrections; the losses.  max_norm: a
    bound on the norm over all gradients of a step."""
    import torch
    m = {k: torch.zeros_like(v) for k, v in block.master.items()}
    v2 = {k: torch.zeros_like(v) for k, v in block.master.items()}
    losses = []
    for i in range(1, steps + 1):
        poses, states, q_pos, k_pos, target, _, _ = views.batch(B, S, i, block.dtype)
        if block.image:
            q_pos, k_pos = views.patch_positions(B, S)
        y, kept = block.forward(poses, states, q_pos, k_pos, keep=True)
        diff = torch.zeros_like(y, dtype=torch.float32)
        diff[..., :6] = y[..., :6].float() - target
        losses.append(float(diff.square().sum() / target.numel()))
        # the gradient is scaled to the order of 1 for its way through 16-bit tensors; Adam's step does not see it
        grads = block.backward(diff.to(block.dtype), kept)
        if max_norm is not None:  # into float32, as Adam takes them
            clipped = [torch.empty_like(g, dtype=torch.float32) for g in grads.values()]
            L.clip_gradients(list(grads.values()), max_norm, out=clipped)
            grads = dict(zip(grads, clipped))
        for k, g in grads.items():
            m[k].mul_(0.9).add_(g.float(), alpha=0.1)
            v2[k].mul_(0.99).addcmul_(g.float(), g.float(), value=0.01)
            step = m[k] / (1 - 0.9 ** i) / ((v2[k] / (1 - 0.99 ** i)).sqrt() + 1e-8)
            block.master[k].sub_(step, alpha=lr * min(1.0, 2 * (1 - i / (steps + 1))))
        block.refresh()
        if report and i % report == 0:
            print(f"step {i}: mean squared error {np.mean(losses[-report:]):.5f}", flush=True)
    return losses


def errors(poses, target):
    """Mean rotation error (degrees) and translation error."""
    c = corrections(poses, np.broadcast_to(target, poses.shape))
    return (float(np.degrees(np.linalg.norm(c[..., :3], axis=-1)).mean()),
            float(np.linalg.norm(c[..., 3:], axis=-1).mean()))


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--workload", default="tiny_bump", choices=synth.ORDER)
    ap.add_argument("--image", action="store_true", help="layer norms, and heads turned by a patch's row and column")
    ap.add_argument("--max-norm", type=float, help="bound on the gradients' norm (default: 100 with --image, else none)")
    ap.add_argument("--bits", type=int, choices=(8, 16), help="of the states that proposals read (default: 8 with --image, else 16)")
    args = ap.parse_args()
    views = Views(args.workload)
    block = ProposalBlock(state_dim=views.state_dim, image=args.image)
    max_norm = 100.0 if args.image and args.max_norm is None else args.max_norm
    bits = args.bits or (8 if args.image else 16)
    train(block, views, args.steps, report=max(1, args.steps // 10), max_norm=max_norm)
    poses, states, q_pos, k_pos, _, hyps, gt = views.batch(4, 64, 10 ** 6, block.dtype)
    if args.image:
        q_pos, k_pos = views.patch_positions(4, 64)
    y = block.propose(poses, block.encode(states, k_pos, bits=bits), q_pos)
    moved = corrected(hyps, y[..., :6].double().cpu().numpy())
    for name, p in (("hypotheses", hyps), ("proposals", moved)):
        r, t = errors(p, gt[:, None])
        print(f"{name}: {r:.2f} degrees, {t:.4f} from the true pose")


if __name__ == "__main__":
    main()
