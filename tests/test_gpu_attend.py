"""The refiner's attention on the GPU against 64-bit statements on the CPU
(tests/attend_ref.py, which derives the bounds): heads normed and turned, attention
to keys of another number, and the learned bias by relative position, with their
gradients."""
import math

import pytest

import attend_ref as ref
from paper_2312_11841_amd import mixrt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def r():
    r = mixrt.Renderer(0, sync_check=True)
    yield r
    r.close()


def say(*a):
    print(*a, flush=True)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _inside(got, want, what):
    want, bound = want
    got = got.double().cpu()
    assert got.shape == want.shape, what
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), what
    over = ((got - want).abs() - bound)[~nan]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))


# --- heads normed and turned ----------------------------------------------------------

# tokens, heads, kv_heads, D, pairs: one element; no pairs; odd widths; part of the
# pairs; pairs that no vector divides; heads of one wave's items and of more; no token
HEADS = [(1, 1, 1, 1, 0), (3, 2, 1, 2, 1), (1, 32, 8, 128, 64), (77, 4, 2, 64, 32),
         (29, 3, 3, 80, 36), (50, 2, 1, 33, 7), (19, 5, 5, 96, 40), (130, 12, 3, 80, 40),
         (7, 1, 1, 1024, 512), (5, 2, 1, 1024, 1), (6, 1, 1, 999, 499), (4, 2, 2, 1023, 12),
         (9, 1, 1, 517, 128), (0, 4, 2, 64, 32), (700, 16, 16, 64, 32)]


def _heads_case(i, dtype, layout):
    T, H, Hk, D, pairs = HEADS[i]
    g = _gen(i)
    x = [torch.randn((T, n, D), generator=g).mul(torch.exp(torch.randn((n, 1), generator=g)))
         .to(dtype) for n in (H, Hk)]
    w = [1 + 0.3 * torch.randn((D,), generator=g) for _ in range(2)]
    if i % 4 == 1:
        w[1] = None
    dy = [0.1 * torch.randn((T, n, D), generator=g).to(dtype) for n in (H, Hk)]
    pos = torch.randint(0, 60, (T, 3), generator=g).float()
    freq = 30.0 ** (-torch.arange(pairs) / max(1, pairs))
    axis = (torch.arange(pairs) % 3).to(torch.uint8)
    return x, w, dy, pos, freq, axis


def _cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(HEADS)), ids=lambda i: str(HEADS[i]))
def test_rotary_norm_and_gradients(r, i, dtype, layout):
    dt = DT[dtype]
    say("rotary_norm", HEADS[i], dtype, layout)
    x, w, dy, pos, freq, axis = _heads_case(i, dt, layout)
    place = (pos.cuda(), freq.cuda(), axis.cuda())
    xs, ws, dys = ([_cuda(t) for t in a] for a in (x, w, dy))
    got = r.rotary_norm(xs, ws, *place, eps=1e-3, layout=layout)
    dx, dw = r.rotary_norm_backward(dys, xs, ws, *place, eps=1e-3, layout=layout)
    for n in range(2):
        _inside(got[n], ref.rotary_norm(x[n], w[n], pos, freq, axis, layout, 1e-3, dt), "out")
        want, bound = ref.rotary_norm_back(dy[n], x[n], w[n], pos, freq, axis, layout, 1e-3, dt)
        _inside(dx[n], (want[0], bound[0]), "dx")
        _inside(dw[n], (want[1], bound[1]), "dw")


# --- attention -----------------------------------------------------------------------

# B, queries, keys, heads, kv_heads, D: one of each; one query to many keys; many to
# one; tiles of 32, 64 and 128 and one past them; widths that are not a chunk's
# multiple; shared heads; more keys than one split; no queries; no keys
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 1, 700, 8, 2, 128), (1, 1, 3000, 4, 4, 64), (1, 300, 1, 2, 2, 32),
          (2, 32, 32, 2, 1, 32), (1, 33, 65, 3, 3, 64), (1, 129, 257, 4, 2, 80),
          (3, 7, 31, 6, 3, 33), (1, 64, 100, 2, 2, 96), (1, 200, 150, 2, 1, 128),
          (2, 5, 1100, 12, 1, 40), (1, 260, 2200, 2, 2, 16), (1, 0, 5, 2, 2, 32),
          (2, 5, 0, 2, 2, 32), (1, 600, 600, 64, 64, 7), (1, 16, 4500, 2, 2, 24),
          (1, 513, 40, 128, 64, 12), (1, 9, 300, 7, 1, 100)]


def _sequences(g, B, Tq, Tk, H, Hk, D, dt, sharp=1.5):
    q = (sharp * torch.randn((B, Tq, H, D), generator=g)).to(dt)
    k, v = (torch.randn((B, Tk, Hk, D), generator=g).to(dt) for _ in range(2))
    dout = (0.1 * torch.randn((B, Tq, H, D), generator=g)).to(dt)
    return q, k, v, dout


def _bias(g, axes, count, reach, B, Tq, Tk, H, own=False):
    table = torch.randn((axes, count, H), generator=g)
    buckets = torch.randint(0, count, (axes, 2 * reach + 1), generator=g).to(torch.uint8)
    q_pos, k_pos = (torch.randint(-20, 20, (*((B,) if own else ()), n, axes), generator=g)
                    .to(torch.int32) for n in (Tq, Tk))
    return table, buckets, q_pos, k_pos


def _on_gpu(bias):
    return None if bias is None else mixrt.RelativeBias(*[t.cuda() for t in bias])


def _check(r, q, k, v, dout, dt, lens=None, bias=None, scale=None, arrays=None):
    """Every call on (arrays or) the sequences against the statement."""
    B, Tq, H, D = q.shape
    cq, ck, cv, cd = [t.cuda() for t in (q, k, v, dout)] if arrays is None else arrays
    kw = dict(lens=_cuda(lens), bias=_on_gpu(bias), scale=scale)
    want = ref.attention(q, k, v, dt, lens, bias, scale)
    _inside(r.attention(cq, ck, cv, **kw), want["o"], "o")
    want = ref.attention(q, k, v, dt, lens, bias, scale, dout)
    o, saved = r.attention_train(cq, ck, cv, **kw)
    _inside(o, want["o"], "o of training")
    grads = r.attention_backward(cd, cq, ck, cv, o, saved, **kw)
    for name, got in zip(("dq", "dk", "dv", "dtable"), grads):
        _inside(got, want[name], name)
    return o, grads


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_and_gradients(r, shape, dtype):
    say("attention", shape, dtype)
    q, k, v, dout = _sequences(_gen(SHAPES.index(shape)), *shape, DT[dtype])
    _check(r, q, k, v, dout, DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_with_bias_and_gradients(r, shape, dtype):
    B, Tq, Tk, H, Hk, D = shape
    i = SHAPES.index(shape)
    axes, count, reach = 1 + i % 3, [1, 5, 16, 32][i % 4], [0, 3, 20, 127][(i // 2) % 4]
    say("attention with bias", shape, dtype, axes, count, reach)
    g = _gen(100 + i)
    q, k, v, dout = _sequences(g, *shape, DT[dtype])
    _check(r, q, k, v, dout, DT[dtype], bias=_bias(g, axes, count, reach, B, Tq, Tk, H, i % 2))
