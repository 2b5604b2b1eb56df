"""A rendered view refined by what reference views show, with the framework's
attention.

A scene is rendered from several cameras.  The first view is rendered with one sample
per ray, the others, which serve as references, with eight; a small network learns to
turn the first into its own render with eight.  Patches of the first view look at the
patches of the references:

  tokens     means of 8 x 8 patches, projected to queries, keys and values
  turned     queries and keys normed head by head and turned by (view, row, column)
  attention  over the references' patches, with a learned bias by the buckets of the
             distances in rows and columns; patches that show background alone lie
             behind the references' length
  colours    a linear layer of what was seen, added to the frame

Training takes the gradients from the framework's backward calls; serving keeps
nothing.  The products with weights are torch's.

    python examples/attend_views.py [--steps 60] [--width 128] [--height 96] [--views 3]
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

HEADS, KV_HEADS, DIM, PATCH, BUCKETS, REACH = 4, 2, 32, 8, 16, 32


class NormTurn(torch.autograd.Function):
    """Heads normed one by one and turned by their tokens' positions."""

    @staticmethod
    def forward(ctx, x, w, pos, freq, axis, r):
        ctx.r = r
        ctx.save_for_backward(x, w, pos, freq, axis)
        return r.rotary_norm(x, w, pos, freq, axis)

    @staticmethod
    def backward(ctx, dy):
        dx, dw = ctx.r.rotary_norm_backward(dy.contiguous(), *ctx.saved_tensors)
        return dx, dw, None, None, None, None


class Attend(torch.autograd.Function):
    """Attention with a bias by relative position; its table learns too."""

    @staticmethod
    def forward(ctx, q, k, v, table, lens, places, r):
        bias = mixrt.RelativeBias(table, *places)
        out, ctx.saved = r.attention_train(q, k, v, lens=lens, bias=bias)
        ctx.r, ctx.places = r, places
        ctx.save_for_backward(q, k, v, table, lens, out)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, table, lens, out = ctx.saved_tensors
        bias = mixrt.RelativeBias(table, *ctx.places)
        grads = ctx.r.attention_backward(dout.contiguous(), q, k, v, out, ctx.saved, lens=lens,
                                         bias=bias)
        return (*grads, None, None, None)


class Network:
    """references: frames [views][pixels][4]; the target's camera lies before theirs."""

    def __init__(self, r, references, H, W, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda a, b, s: (s / math.sqrt(a) * torch.randn((a, b), generator=g,  # noqa: E731
                                                               device="cuda"))
        self.r, self.dtype, self.H, self.W = r, dtype, H, W
        self.ph, self.pw = H // PATCH, W // PATCH
        self.w = {"q": draw(4, HEADS * DIM, 1.0), "kv": draw(4, 2 * KV_HEADS * DIM, 1.0),
                  "out": draw(HEADS * DIM, 4, 0.1),
                  "norm_q": torch.ones(DIM, device="cuda"),
                  "norm_k": torch.ones(DIM, device="cuda"),
                  "table": torch.zeros((2, BUCKETS, HEADS), device="cuda")}
        for t in self.w.values():
            t.requires_grad_()
        pairs = DIM // 2
        self.axis = (torch.arange(pairs, device="cuda") % 3).to(torch.uint8)
        self.freq = 100.0 ** (-(torch.arange(pairs, device="cuda") // 3).float() / (pairs / 3))
        views = references.shape[0]
        ax = [torch.arange(n, device="cuda") for n in (views + 1, self.ph, self.pw)]
        places = torch.stack(torch.meshgrid(*ax, indexing="ij"), -1).reshape(-1, 3)
        mine, theirs = places.split([self.ph * self.pw, views * self.ph * self.pw])
        # the references' patches that show something first, the others behind their length
        self.seen = self.patches(references)
        shown = self.seen[:, 3] > 0
        order = torch.argsort((~shown).to(torch.uint8), stable=True)
        self.seen, theirs = self.seen[order], theirs[order]
        self.lens = shown.sum().to(torch.int32).reshape(1)
        self.pos = (mine.float(), theirs.float())
        buckets = mixrt.distance_buckets(BUCKETS, REACH).cuda()
        self.places = (torch.stack([buckets, buckets]),
                       *[p[:, 1:].to(torch.int32).contiguous() for p in (mine, theirs)])

    def patches(self, frames):
        """Means of the patches, [views * patches][4]."""
        a = frames.reshape(-1, self.ph, PATCH, self.pw, PATCH, 4)
        return a.mean(dim=(2, 4)).reshape(-1, 4)

    def heads(self, tokens):
        """Queries [tokens][heads][D], keys and values [tokens][2][kv_heads][D]."""
        q = (tokens @ self.w["q"]).to(self.dtype).reshape(-1, HEADS, DIM)
        kv = (self.seen @ self.w["kv"]).to(self.dtype).reshape(-1, 2, KV_HEADS, DIM)
        return q, kv

    def add(self, frame, seen):
        """The frame with what its patches saw."""
        y = (seen.reshape(-1, HEADS * DIM).float() @ self.w["out"]).reshape(
            self.ph, 1, self.pw, 1, 4).expand(-1, PATCH, -1, PATCH, -1)
        return frame + y.reshape(frame.shape)

    def train_forward(self, frame):
        w, r = self.w, self.r
        q, kv = self.heads(self.patches(frame))
        q = NormTurn.apply(q, w["norm_q"], self.pos[0], self.freq, self.axis, r)
        k = NormTurn.apply(kv[:, 0].contiguous(), w["norm_k"], self.pos[1], self.freq, self.axis,
                           r)
        seen = Attend.apply(q[None], k[None], kv[:, 1][None], w["table"], self.lens, self.places, r)
        return self.add(frame, seen)

    @torch.no_grad()
    def serve(self, frame):
        w, r = self.w, self.r
        q, kv = self.heads(self.patches(frame))
        q = r.rotary_norm(q, w["norm_q"], self.pos[0], self.freq, self.axis)
        k = r.rotary_norm(kv[:, 0], w["norm_k"], self.pos[1], self.freq, self.axis)
        seen = r.attention(q[None], k[None], kv[:, 1][None], lens=self.lens,
                           bias=mixrt.RelativeBias(w["table"], *self.places))
        return self.add(frame, seen)


def render(r, cfg):
    """Frames of a scene, [views][pixels][4]."""
    ds = mixrt.DeviceScene.from_scene(synth.make_scene(cfg), device="cuda:0")
    return r.render(ds).reshape(cfg.views, cfg.H * cfg.W, 4)


def main(steps=60, width=128, height=96, views=3, say=print):
    """Trains; returns the losses, the largest difference between the served and the
    trained network's frames, and the network with its target frame."""
    if width % PATCH or height % PATCH:
        raise SystemExit(f"width and height have to be multiples of {PATCH}")
    torch.cuda.set_device(0)
    r = mixrt.Renderer(0)
    base = synth.TINY64_DENSE.replace(name="attend", W=width, H=height, views=views + 1)
    few, many = render(r, base.replace(K=1)), render(r, base.replace(K=8))
    frame, target = few[0], many[0]
    net = Network(r, many[1:], height, width)
    optimiser = torch.optim.Adam(net.w.values(), lr=5e-3)
    losses = []
    for step in range(steps):
        optimiser.zero_grad()
        loss = (net.train_forward(frame) - target).square().mean()
        loss.backward()
        optimiser.step()
        losses.append(float(loss.detach()))
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step}: mean squared error {losses[-1]:.3e}")
    apart = float((net.serve(frame) - net.train_forward(frame).detach()).abs().max())
    say(f"served and trained frames differ by at most {apart:.1e}")
    r.sync()
    return losses, apart, (net, frame, target)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--height", type=int, default=96)
    ap.add_argument("--views", type=int, default=3)
    a = ap.parse_args()
    main(a.steps, a.width, a.height, a.views)
