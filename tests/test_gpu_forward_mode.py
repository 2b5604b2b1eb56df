"""The refiner's calls inside torch's forward-mode derivatives: they have none there, and
say so instead of dropping an input's tangent."""
import pytest

from paper_2312_11841_amd import mixrt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_tangents_are_refused_rather_than_dropped():
    from torch.autograd import forward_ad
    r = mixrt.Renderer(0, sync_check=True)
    g = torch.Generator().manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=g).cuda()

    x, q, w = draw(2, 30, 16), draw(1, 20, 2, 16), draw(16)
    pos, freq, axis = draw(20, 1), draw(8), torch.zeros(8).byte().cuda()
    table = draw(1, 3, 2)
    places = torch.arange(20).int()[:, None].cuda()
    buckets = torch.zeros((1, 5)).byte().cuda()
    _, stats, kept = r.group_norm_train(x, 4)
    rows = r.checkpoint_pack(x)
    o, saved = r.attention_train(q, q, q)
    calls = {
        "group_norm": (lambda t: r.group_norm(t, 4), x),
        "group_norm gamma": (lambda t: r.group_norm(x, 4, t), w),
        "group_norm_train": (lambda t: r.group_norm_train(t, 4)[0], x),
        "group_norm_backward": (lambda t: r.group_norm_backward(t, kept, stats)[0], x),
        "linear_weight_grad": (lambda t: r.linear_weight_grad(rows, t)[0], x),
        "rotary": (lambda t: r.rotary(t, pos, freq, axis), q[0]),
        "rotary_norm": (lambda t: r.rotary_norm(t, w, pos, freq, axis), q[0]),
        "rotary_norm weight": (lambda t: r.rotary_norm(q[0], t, pos, freq, axis), w),
        "rotary_norm_backward": (lambda t: r.rotary_norm_backward(t, q[0], w, pos, freq,
                                                                  axis)[0], q[0]),
        "attention": (lambda t: r.attention(q, t, q), q),
        "attention table": (lambda t: r.attention(q, q, q, bias=mixrt.RelativeBias(
            t, buckets, places, places)), table),
        "attention_train": (lambda t: r.attention_train(t, q, q)[0], q),
        "attention_backward": (lambda t: r.attention_backward(t, q, q, q, o, saved)[0], q),
    }
    try:
        for name, (call, t) in calls.items():
            want = call(t)
            with forward_ad.dual_level():
                dual = forward_ad.make_dual(t, torch.ones_like(t))
                with pytest.raises(RuntimeError, match="forward mode"):
                    call(dual)
                with torch.no_grad(), pytest.raises(RuntimeError, match="forward mode"):
                    call(dual)
                assert torch.equal(call(t), want), name
            assert torch.equal(call(t), want), name
    finally:
        r.close()
