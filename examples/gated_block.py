"""A gated recurrent block over recorded episodes: its training step, and a dream with it.

The block predicts the next latent from the latents and actions so far, as the world model's LSTM
does, but its recurrence is linear in the state, so a whole recording is one scan over time:

    u = embed(action) + z W_in;  y = layer_norm(u);  [gate | x] = y W_proj + b_proj
    h_t = sig(gate_t) h_{t-1} + (1 - sig(gate_t)) x_t;  prediction of z_{t+1} = h_t W_out

The training step runs every operator forward and backward, the matrix products by torch, and
clips the gradients by their global norm before the update.  A dream takes the same block one step
at a time, the state in hand.

    python examples/gated_block.py [--steps 200] [--precision bf16]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import torch  # noqa: E402

import paper_2205_01435_gb300 as pkg  # noqa: E402
import synth  # noqa: E402


class GatedBlock:
    def __init__(self, z_dim, a_dim, width, h_dim, precision="fp32", device="cuda", seed=0):
        self.ops = pkg.load_seq().SequenceOps()
        self.H, self.scale = h_dim, math.sqrt(width)
        dt = torch.bfloat16 if precision == "bf16" else torch.float32
        gen = torch.Generator(device=device).manual_seed(seed)

        def init(*shape, std):
            return (torch.randn(shape, generator=gen, device=device) * std).to(dt)

        self.p = {"embed": init(a_dim, width, std=1.0 / width), "w_in": init(z_dim, width, std=z_dim ** -0.5),
                  "w_proj": init(width, 2 * h_dim, std=width ** -0.5), "b_proj": torch.zeros(2 * h_dim, device=device, dtype=dt),
                  "w_out": init(h_dim, z_dim, std=h_dim ** -0.5),
                  # the layer norm's parameters are fp32 whatever the precision
                  "ln_weight": torch.ones(width, device=device), "ln_bias": torch.zeros(width, device=device)}
        self.p["b_proj"][:h_dim] = 1.0  # start out remembering

    def forward(self, z, actions, starts=None, lengths=None, h0=None):
        """z [T, N, Z], actions [T, N] int32: the predictions [T, N, Z], and what the backward takes."""
        p, ops = self.p, self.ops
        u = torch.addmm(ops.embed(p["embed"], actions, scale=self.scale).flatten(0, 1), z.flatten(0, 1), p["w_in"])
        y, mean, rstd = ops.layer_norm(u, p["ln_weight"], p["ln_bias"], want_stats=True)
        proj = torch.addmm(p["b_proj"], y, p["w_proj"]).view(*z.shape[:2], 2 * self.H)
        h, last = ops.gated_scan(proj[..., :self.H], proj[..., self.H:], h0=h0, reset=starts, lengths=lengths)
        pred = (h.flatten(0, 1) @ p["w_out"]).view_as(z)
        return pred, dict(z=z, actions=actions, starts=starts, lengths=lengths, h0=h0, u=u, y=y, mean=mean, rstd=rstd, proj=proj, h=h,
                          last=last)

    def backward(self, s, dpred):
        """The parameters' gradients from the prediction's gradient [T, N, Z]."""
        p, ops, H = self.p, self.ops, self.H
        d = dpred.flatten(0, 1)
        g = {"w_out": s["h"].flatten(0, 1).T @ d}
        dh = (d @ p["w_out"].T).view_as(s["h"])
        # both gradients into one array, as the projection's backward products take it
        dproj = torch.empty_like(s["proj"])
        ops.gated_scan_backward(s["proj"][..., :H], s["proj"][..., H:], s["h"], dh, h0=s["h0"], reset=s["starts"],
                                lengths=s["lengths"], dgate=dproj[..., :H], dx=dproj[..., H:], want_dh0=False)
        dp = dproj.flatten(0, 1)
        g["w_proj"], g["b_proj"] = s["y"].T @ dp, dp.sum(0)
        du, g["ln_weight"], g["ln_bias"] = ops.layer_norm_backward(s["u"], p["ln_weight"], s["mean"], s["rstd"], dp @ p["w_proj"].T)
        g["w_in"] = s["z"].flatten(0, 1).T @ du
        g["embed"] = ops.embed_backward(s["actions"], du.view(*s["actions"].shape, -1), p["embed"].shape[0], scale=self.scale)
        return g

    def train_step(self, z, actions, lr, starts=None, lengths=None, max_norm=1.0):
        """One step on latents [T + 1, N, Z] and actions [T, N]; returns (loss, gradient norm) on the device."""
        pred, saved = self.forward(z[:-1], actions, starts, lengths)
        err = (pred - z[1:]).float()
        if lengths is not None:  # padding is not in the loss
            live = torch.arange(len(actions), device=z.device)[:, None] < lengths[None, :]
            err = torch.where(live[..., None], err, 0.0)
        count = float(err.numel())
        grads = self.backward(saved, (err / count).to(z.dtype))
        norm = self.ops.clip_grads(list(grads.values()), max_norm)
        for k, g in grads.items():
            self.p[k].add_(g, alpha=-lr)
        return err.square().sum() / (2 * count), norm

    def dream(self, z, actions, state):
        """One episode step for N episodes: z [N, Z], actions [N], state [N, H] fp32 (updated in place)."""
        p, ops, H = self.p, self.ops, self.H
        u = torch.addmm(ops.embed(p["embed"], actions, scale=self.scale), z, p["w_in"])
        proj = torch.addmm(p["b_proj"], ops.layer_norm(u, p["ln_weight"], p["ln_bias"]), p["w_proj"])
        h, _ = ops.gated_step(proj[:, :H], proj[:, H:], state, out_state=state)
        return h @ p["w_out"]


def recordings(T, N, z_dim, a_dim, precision, seed=0):
    """Latents that move by what the actions say, so that there is something to learn."""
    z, actions = (torch.from_numpy(v).cuda() for v in synth.teacher_inputs(N, T, z_dim, a_dim, seed=seed)[:2])
    push = torch.randn(a_dim, z_dim, generator=torch.Generator().manual_seed(1)).cuda()
    out = z * 0.1
    for t in range(T):
        out[t + 1] += 0.8 * out[t] + 0.3 * push[actions[t].long()]
    return out.to(torch.bfloat16 if precision == "bf16" else torch.float32), actions


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--precision", choices=("fp32", "bf16"), default="bf16")
    a = ap.parse_args()
    T, N, Z, A = 128, 64, 32, 64
    z, actions = recordings(T, N, Z, A, a.precision)
    block = GatedBlock(Z, A, 128, 256, a.precision)
    for i in range(a.steps):
        loss, norm = block.train_step(z, actions, lr=1.0)
        if i % max(1, a.steps // 10) == 0 or i + 1 == a.steps:
            print(f"step {i:4d}  loss {float(loss):.5f}  gradient norm {float(norm):.4f}")
    state = torch.zeros(N, 256, device="cuda")
    x = z[0]
    for t in range(8):  # a dream: its own predictions for latents
        x = block.dream(x, actions[t], state)
    block.ops.sync()
    print(f"after 8 dreamt steps the latents are {float((x.float() - z[8].float()).square().mean().sqrt()):.3f} off (rms), "
          f"their rms is {float(z[8].float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
