"""The example whose view attends to reference views runs, and the gradients that its
calls pass on are those of the network in 64 bits."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def _plain(ex, net, frame, w):
    """The network's frame in 64 bits, from torch's own operations on the CPU."""
    frame = frame.double().cpu()

    def patches(a):
        return a.reshape(net.ph, ex.PATCH, net.pw, ex.PATCH, 4).mean(dim=(1, 3)).reshape(-1, 4)

    def turned(x, weight, pos):
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
        angle = (pos.cpu()[:, net.axis.cpu().long()] * net.freq.cpu()).double()[:, None]
        a, b = n.chunk(2, -1)
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()],
                         -1)

    seen = net.seen.double().cpu()
    q = turned((patches(frame) @ w["q"]).reshape(-1, ex.HEADS, ex.DIM), w["norm_q"], net.pos[0])
    k, v = (seen @ w["kv"]).reshape(-1, 2, ex.KV_HEADS, ex.DIM).unbind(1)
    k = turned(k, w["norm_k"], net.pos[1])
    n = int(net.lens[0])
    share = ex.HEADS // ex.KV_HEADS
    k, v = (t[:n].repeat_interleave(share, 1) for t in (k, v))
    s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(ex.DIM)
    buckets, qp, kp = (t.cpu().long() for t in net.places)
    for a in range(2):
        d = (kp[None, :n, a] - qp[:, None, a]).clamp(-ex.REACH, ex.REACH) + ex.REACH
        s = s + w["table"][a][buckets[a][d]].permute(2, 0, 1)
    o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v).reshape(-1, ex.HEADS * ex.DIM)
    y = (o @ w["out"]).reshape(net.ph, 1, net.pw, 1, 4).expand(-1, ex.PATCH, -1, ex.PATCH, -1)
    return frame + y.reshape(frame.shape)


def test_attending_example_runs_and_passes_its_gradients():
    import attend_views as ex
    losses, apart, (net, frame, target) = ex.main(steps=8, width=64, height=48, views=2,
                                                  say=lambda *a: print(*a, flush=True))
    assert all(math.isfinite(x) for x in losses)
    assert 0 < int(net.lens[0]) <= net.seen.shape[0]
    # served weights are rounded once more than trained ones: a bfloat16 rounding of
    # weights and of the result, 2^-8 each, of values that the colours' layer brings to
    # the frame
    sizes = net.heads(net.patches(frame))[1][:, 1].abs().max().float() \
        * net.w["out"].detach().abs().sum(0).max()
    assert apart <= 3 * 2.0 ** -8 * float(sizes.detach())

    net.dtype = torch.float32
    loss = (net.train_forward(frame) - target).square().mean()
    grads = dict(zip(net.w, torch.autograd.grad(loss, list(net.w.values()))))
    w = {n: t.detach().double().cpu().requires_grad_() for n, t in net.w.items()}
    plain = _plain(ex, net, frame, w)
    want_loss = (plain - target.double().cpu()).square().mean()
    want = dict(zip(w, torch.autograd.grad(want_loss, list(w.values()))))
    assert abs(float(loss) - float(want_loss)) <= 1e-4 * float(want_loss)
    for n in w:
        off = (grads[n].double().cpu() - want[n]).norm() / want[n].norm()
        print(n, float(off), flush=True)
        # 32-bit operations, a few hundred of them one after another, and what cancels
        # in a softmax's gradient
        assert float(off) <= 2.0 ** -10, n
