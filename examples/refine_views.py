"""A refiner of rendered views, trained and served with the framework's operators.

Two views of a scene are rendered with one sample per ray, and the same views
with eight: a small network learns to turn the first into the second.  It works
on the frames as they come, [views][pixels][4], channels last:

  features   a per-pixel linear layer, group norm with silu
  mixing     patches of both views attend to each other, their queries and keys
             turned by (view, row, column)
  colours    a per-pixel linear layer, added to the frame

Training keeps the norm's and the layers' inputs in 8 bits (the frame-size
arrays are what training a refiner holds in memory) and computes the gradients
from them; matrix products and the attention's softmax are torch's.  Serving
keeps nothing.

    python examples/refine_views.py [--steps 60] [--width 128] [--height 96]
"""
import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2312_11841_amd import mixrt, synth  # noqa: E402

CHANNELS, GROUPS, HEADS, DIM, PATCH = 32, 8, 2, 32, 8


class NormSilu(torch.autograd.Function):
    """silu(group norm), its input kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, gamma, beta, r):
        y, stats, kept = r.group_norm_train(x, GROUPS, gamma, beta, act="silu")
        ctx.r, ctx.kept = r, kept
        ctx.save_for_backward(stats, gamma, beta)
        return y

    @staticmethod
    def backward(ctx, dy):
        stats, gamma, beta = ctx.saved_tensors
        dx, dgamma, dbeta = ctx.r.group_norm_backward(dy.contiguous(), ctx.kept, stats, gamma,
                                                      beta, act="silu")
        return dx, dgamma, dbeta, None


class Linear(torch.autograd.Function):
    """rows @ w, the rows kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, w, r):
        ctx.r, ctx.kept = r, r.checkpoint_pack(x)
        ctx.save_for_backward(w)
        return x @ w.to(x.dtype)

    @staticmethod
    def backward(ctx, dy):
        (w,) = ctx.saved_tensors
        dw, _ = ctx.r.linear_weight_grad(ctx.kept, dy.contiguous(), bias=False)
        return dy @ w.to(dy.dtype).t(), dw, None


class Rotary(torch.autograd.Function):
    """Queries and keys turned by their tokens' positions; the gradient turns back."""

    @staticmethod
    def forward(ctx, q, k, pos, freq, axis, r):
        ctx.r = r
        ctx.save_for_backward(pos, freq, axis)
        return r.rotary((q, k), pos, freq, axis)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k = ctx.r.rotary((dq.contiguous(), dk.contiguous()), *ctx.saved_tensors, inverse=True)
        return q, k, None, None, None, None


class Refiner:
    def __init__(self, r, views, H, W, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda a, b, s: (s / math.sqrt(a) * torch.randn((a, b), generator=g,  # noqa: E731
                                                               device="cuda"))
        self.r, self.views, self.H, self.W = r, views, H, W
        self.w = {"in": draw(4, CHANNELS, 1.0), "qk": draw(CHANNELS, 2 * HEADS * DIM, 1.0),
                  "v": draw(CHANNELS, CHANNELS, 1.0), "mix": draw(CHANNELS, CHANNELS, 0.1),
                  "out": draw(CHANNELS, 4, 0.1),
                  "gamma": torch.ones(CHANNELS, device="cuda"),
                  "beta": torch.zeros(CHANNELS, device="cuda")}
        for t in self.w.values():
            t.requires_grad_()
        # patch positions (view, row, column); a third of the pairs for each
        self.ph, self.pw = H // PATCH, W // PATCH
        ax = [torch.arange(n, device="cuda") for n in (views, self.ph, self.pw)]
        self.pos = torch.stack(torch.meshgrid(*ax, indexing="ij"), -1).reshape(-1, 3).float()
        pairs = DIM // 2
        self.axis = (torch.arange(pairs, device="cuda") % 3).to(torch.uint8)
        self.freq = 100.0 ** (-(torch.arange(pairs, device="cuda") // 3).float() / (pairs / 3))

    def _patches(self, a):
        """Means of the patches: [views * patches][channels] in 32 bits."""
        a = a.float().reshape(self.views, self.ph, PATCH, self.pw, PATCH, CHANNELS)
        return a.mean(dim=(2, 4)).reshape(-1, CHANNELS)

    def _mix(self, a, turn):
        """What the patches' attention adds to the features."""
        t = self._patches(a)
        q, k = (t @ self.w["qk"]).reshape(-1, 2, HEADS, DIM).unbind(1)
        q, k = turn(q.contiguous(), k.contiguous())
        heads = lambda x: x.transpose(0, 1).contiguous()  # noqa: E731
        s = heads(q) @ heads(k).transpose(1, 2).contiguous() / math.sqrt(DIM)
        v = heads((t @ self.w["v"]).reshape(-1, HEADS, CHANNELS // HEADS))
        o = heads(torch.softmax(s, -1) @ v).reshape(-1, CHANNELS) @ self.w["mix"]
        o = o.reshape(self.views, self.ph, 1, self.pw, 1, CHANNELS)
        o = o.expand(-1, -1, PATCH, -1, PATCH, -1)
        return o.reshape(self.views, -1, CHANNELS).to(a.dtype)

    def train_forward(self, frames):
        """Refined frames [views][pixels][4] with what the gradients need."""
        w, r = self.w, self.r
        x = frames.to(torch.bfloat16)
        h = Linear.apply(x.reshape(-1, 4), w["in"], r).reshape(self.views, -1, CHANNELS)
        a = NormSilu.apply(h, w["gamma"], w["beta"], r)
        a = a + self._mix(a, lambda q, k: Rotary.apply(q, k, self.pos, self.freq, self.axis, r))
        return frames + Linear.apply(a.reshape(-1, CHANNELS), w["out"], r).reshape(frames.shape)

    @torch.no_grad()
    def serve(self, frames):
        """The same frames, nothing kept."""
        w, r = self.w, self.r
        x = frames.to(torch.bfloat16)
        h = (x.reshape(-1, 4) @ w["in"].to(x.dtype)).reshape(self.views, -1, CHANNELS)
        a = r.group_norm(h, GROUPS, w["gamma"].detach(), w["beta"].detach(), act="silu", out=h)
        a = a + self._mix(a, lambda q, k: r.rotary((q, k), self.pos, self.freq, self.axis))
        y = a.reshape(-1, CHANNELS) @ w["out"].to(a.dtype)
        return frames + y.reshape(frames.shape)


def render(r, cfg):
    """Frames of a scene, [views][pixels][4]."""
    ds = mixrt.DeviceScene.from_scene(synth.make_scene(cfg), device="cuda:0")
    return r.render(ds).reshape(cfg.views, cfg.H * cfg.W, 4)


def main(steps=60, width=128, height=96, say=print):
    """Trains; returns the losses and the largest difference between the served
    and the trained network's frames."""
    if width % PATCH or height % PATCH:
        raise SystemExit(f"width and height have to be multiples of {PATCH}")
    torch.cuda.set_device(0)
    r = mixrt.Renderer(0)
    base = synth.TINY64_DENSE.replace(name="refine", W=width, H=height, views=2)
    frames, target = render(r, base.replace(K=1)), render(r, base.replace(K=8))
    net = Refiner(r, 2, height, width)
    optimiser = torch.optim.Adam(net.w.values(), lr=5e-3)
    losses = []
    for step in range(steps):
        optimiser.zero_grad()
        loss = (net.train_forward(frames) - target).square().mean()
        loss.backward()
        optimiser.step()
        losses.append(float(loss.detach()))
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: mean squared error {losses[-1]:.3e}")
    apart = float((net.serve(frames) - net.train_forward(frames).detach()).abs().max())
    say(f"served and trained frames differ by at most {apart:.1e}")
    r.sync()
    return losses, apart


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--height", type=int, default=96)
    a = ap.parse_args()
    main(a.steps, a.width, a.height)
