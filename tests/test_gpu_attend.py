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
          (1, 513, 40, 128, 64, 12), (1, 9, 300, 7, 1, 100),
          # columns of their own for every wave, of each padded width; walks that are
          # split there; two blocks of columns a wave
          (1, 130, 130, 130, 130, 96), (2, 131, 95, 128, 64, 128), (1, 1100, 1090, 16, 16, 40),
          (1, 1050, 60, 32, 32, 32), (1, 300, 1200, 43, 43, 64)]


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


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_bias_of_one_bucket_has_no_gradient(r, dtype):
    """A bias that all keys of a row share does not change its weights: the table's
    gradient is 0 exactly with one bucket, with a reach of 0, and on an axis where all
    tokens have one place; not a NaN's."""
    B, Tq, Tk, H, Hk, D = 2, 70, 300, 4, 2, 32
    g = _gen(77)
    q, k, v, dout = _sequences(g, B, Tq, Tk, H, Hk, D, DT[dtype])
    args = [t.cuda() for t in (q, k, v)]
    for axes, count, reach, level in ((1, 1, 20, None), (2, 7, 0, None), (3, 9, 15, 1)):
        say("one bucket", dtype, axes, count, reach, level)
        bias = _bias(g, axes, count, reach, B, Tq, Tk, H)
        if level is not None:
            bias[2][:, level], bias[3][:, level] = 4, 9
        on = _on_gpu(bias)
        o, saved = r.attention_train(*args, bias=on)
        table = r.attention_backward(dout.cuda(), *args, o, saved, bias=on)[3]
        for a in range(axes):
            assert bool((table[a] == 0).all()) == (level is None or a == level)
        bad = dout.clone()
        bad[1, 3, 2, 0] = math.nan
        table = r.attention_backward(bad.cuda(), *args, o, saved, bias=on)[3].cpu()
        assert all(bool(table[a, :, 2].isnan().any()) for a in range(axes))
        assert not bool(table[:, :, 0].isnan().any())


# --- masks, lengths and values that are not numbers ------------------------------------

@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_lengths_and_what_lies_behind_them(r, dtype, biased):
    """Entries of every length, none, one and out of range among them; keys and values
    behind a length are NaN and infinite, and are not read; nor are their places."""
    dt = DT[dtype]
    lens = [0, 1, 31, 32, 33, 150, 200, 999, -3, 64]
    B, Tq, Tk, H, Hk, D = len(lens), 45, 200, 4, 2, 24
    g = _gen(5)
    q, k, v, dout = _sequences(g, B, Tq, Tk, H, Hk, D, dt)
    for b, n in enumerate(lens):
        k[b, max(0, n):] = math.nan
        v[b, max(0, n):] = math.inf
    bias = _bias(g, 2, 9, 15, B, Tq, Tk, H) if biased else None
    _, grads = _check(r, q, k, v, dout, dt, torch.tensor(lens, dtype=torch.int32), bias)
    for b, n in enumerate(lens):
        for t in grads[1:3]:
            assert float(t[b, max(0, n):].float().abs().sum()) == 0
        if n <= 0:
            assert float(grads[0][b].float().abs().sum()) == 0
        if n == 1:      # one key: its weight is 1 whatever its score
            for t in grads[:2]:
                assert float(t[b].float().abs().sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_buckets_that_are_banned(r, dtype):
    """A bias of -infinity leaves its pairs out; a row with no others is 0, and no
    gradient passes."""
    dt = DT[dtype]
    g = _gen(6)
    B, Tq, Tk, H, D = 2, 70, 90, 2, 32
    q, k, v, dout = _sequences(g, B, Tq, Tk, H, H, D, dt)
    table = torch.randn((1, 3, H), generator=g)
    table[0, 2] = -math.inf
    buckets = torch.tensor([[2, 2, 0, 1, 0, 2, 2]], dtype=torch.uint8)
    q_pos = torch.arange(Tq, dtype=torch.int32)[:, None]
    k_pos = torch.arange(Tk, dtype=torch.int32)[:, None]
    q_pos[10:20] += 1000        # nobody near
    o, grads = _check(r, q, k, v, dout, dt, bias=(table, buckets, q_pos, k_pos))
    assert float(o[:, 10:20].float().abs().sum()) == 0
    assert float(grads[0][:, 10:20].float().abs().sum()) == 0
    assert float(grads[3][0, 2].abs().sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 70, 90, 2, 2, 40), (1, 200, 64, 130, 130, 64)], ids=str)
def test_values_that_are_not_finite(r, shape, dtype):
    """A query with NaN makes its own rows NaN; a value that is infinite its element of
    the rows; a key with NaN its head."""
    dt = DT[dtype]
    B, Tq, Tk, H, Hk, D = shape
    q, k, v, dout = _sequences(_gen(7), *shape, dt, sharp=0.2)
    q[0, 3, 1, 2] = math.nan
    v[0, 5, 0, 4] = math.inf
    k[0, 7, 1, 0] = math.nan
    o = r.attention(q.cuda(), k.cuda(), v.cuda()).cpu().float()
    want = torch.zeros((Tq, H, D), dtype=torch.bool)
    want[:, 1] = True
    assert torch.equal(torch.isnan(o[0]), want)
    assert bool((o[0, :, 0, 4] == math.inf).all())
    o[0, :, 0, 4] = 0
    o[0, :, 1] = 0
    assert bool(torch.isfinite(o).all())


def test_gradients_of_any_size_in_float16(r):
    """dS far below float16's normal numbers, and far above its largest: gradients keep
    their relative accuracy."""
    for size in (2.0 ** -20, 2.0 ** -9, 1.0, 2.0 ** 9):
        g = _gen(8)
        q, k, v, _ = _sequences(g, 1, 60, 500, 2, 2, 32, torch.float16)
        dout = (size * torch.randn(q.shape, generator=g)).clamp(-60000, 60000).half()
        q, k = q * 0.2, k * 2.0 ** -7 if size > 1 else k
        grads = _check(r, q, k, v, dout, torch.float16)[1]
        want = ref.attention(q, k, v, torch.float16, dout=dout)
        if size >= 2.0 ** -9:
            for name, got in zip(("dq", "dk", "dv"), grads):
                exact = want[name][0]
                off = (got.double().cpu() - exact).norm() / exact.norm()
                say(size, name, float(off))
                # each term's rounding and the result's, and what the result's type
                # cannot hold
                room = 2.0 ** -25 * exact.numel() ** 0.5 / float(exact.norm())
                assert float(off) <= 2.0 ** -10 + room, (size, name)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_that_look_at_one_key(r, dtype):
    """Weights of almost 1 on one of two keys: dS cancels to a small part of its terms,
    and the gradients still hold."""
    dt = DT[dtype]
    g = _gen(9)
    q, k, v, dout = _sequences(g, 1, 64, 2, 2, 2, 32, dt)
    k[0, 0], k[0, 1] = 0.6 * torch.ones((2, 32)), -0.6 * torch.ones((2, 32))
    q = (0.5 + 0.1 * torch.randn(q.shape, generator=g)).to(dt)
    _check(r, q, k, v, dout, dt)
    o, saved = r.attention_train(q.cuda(), k.cuda(), v.cuda())
    dq = r.attention_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), o, saved)[0]
    exact = ref.attention(q, k, v, dt, dout=dout)["dq"][0]
    off = float((dq.double().cpu() - exact).norm() / exact.norm())
    # the roundings of dS and of the result (a gradient from rounded weights is off by
    # about a weight's rounding over the smaller weight, 3 to 30 times that)
    assert off <= 2 * ref.HALF_UNIT[dt]


# --- layouts ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_of_every_array(r, dtype):
    """Keys and values as slices of a joint projection at odd offsets, heads before
    tokens, one set of keys for all entries, an output in a wider array."""
    dt = DT[dtype]
    g = _gen(11)
    B, Tq, Tk, H, Hk, D = 3, 37, 70, 4, 2, 20
    q, k, v, dout = _sequences(g, B, Tq, Tk, H, Hk, D, dt)
    k[1:], v[1:] = k[:1], v[:1]
    joint = torch.zeros((1, Tk, 2 * Hk * D + 3), dtype=dt)
    joint[0, :, 1:1 + Hk * D] = k[0].reshape(Tk, -1)
    joint[0, :, 1 + Hk * D:-2] = v[0].reshape(Tk, -1)
    joint = joint.cuda()
    ks = joint[..., 1:1 + Hk * D].reshape(1, Tk, Hk, D).expand(B, -1, -1, -1)
    vs = joint.as_strided((1, Tk, Hk, D), (0, joint.shape[2], D, 1),
                          1 + Hk * D).expand(B, -1, -1, -1)
    assert vs.stride(0) == 0
    qs = q.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    ds = torch.zeros((B, Tq, H, D + 7), dtype=dt, device="cuda")[..., 3:3 + D]
    ds.copy_(dout)
    _check(r, q, k, v, dout, dt, arrays=(qs, ks, vs, ds))
    wide = torch.full((B, Tq, H + 1, D + 5), 7.0, dtype=dt, device="cuda")
    into = wide[:, :, 1:, 2:2 + D]
    got = r.attention(qs, ks, vs, out=into)
    assert got is into and torch.equal(into, r.attention(qs, ks, vs))
    into.fill_(7.0)
    assert bool((wide == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_heads_far_apart(r, dtype):
    """Offsets of more than 2^31 elements between tokens, heads and entries."""
    dt = DT[dtype]
    g = _gen(12)
    far = 2 ** 31 + 24
    buf = torch.zeros((far + 64 * 40,), dtype=dt, device="cuda")
    q, k, v, dout = _sequences(g, 2, 2, 2, 2, 2, 16, dt)
    near = [t.cuda() for t in (q, k, v, dout)]
    want = r.attention(*near[:3])
    o, saved = r.attention_train(*near[:3])
    grads = r.attention_backward(near[3], *near[:3], o, saved)
    for strides in ((far, 64, 16, 1), (64, far, 16, 1), (64, 16, far, 1)):
        for n in range(4):
            x = buf.as_strided((2, 2, 2, 16), strides)
            x.copy_(near[n])
            a = list(near)
            a[n] = x
            if n < 3:
                assert torch.equal(r.attention(*a[:3]), want), (strides, n)
            got = r.attention_backward(a[3], *a[:3], o, saved)
            assert all(torch.equal(x, y) for x, y in zip(got, grads)), (strides, n)
        out = buf.as_strided((2, 2, 2, 16), strides)
        assert torch.equal(r.attention(*near[:3], out=out), want)
    heads = near[0][0]
    w, pos = torch.rand(16, generator=g).cuda(), torch.ones((2, 1), device="cuda")
    freq, axis = torch.rand(8, generator=g).cuda(), torch.zeros(8, device="cuda").byte()
    want = r.rotary_norm(heads, w, pos, freq, axis)
    back = r.rotary_norm_backward(near[3][0], heads, w, pos, freq, axis)
    for strides in ((far, 16, 1), (16, far, 1)):
        x = buf.as_strided((2, 2, 16), strides)
        x.copy_(heads)
        assert torch.equal(r.rotary_norm(x, w, pos, freq, axis), want)
        assert torch.equal(r.rotary_norm(x, w, pos, freq, axis, out=x), want)
        x.copy_(near[3][0])
        got = r.rotary_norm_backward(x, heads, w, pos, freq, axis, out=x)
        assert all(torch.equal(a, b) for a, b in zip(got, back))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_places_in_every_order(r, dtype):
    """Rows of tokens of every width (places that count up, that stay, that mix inside 8
    and 32 rows), places in no order, and places at the ends of 32 bits."""
    dt = DT[dtype]
    g = _gen(13)
    H, D, reach = 2, 16, 9
    table = torch.randn((3, 7, H), generator=g)
    buckets = torch.randint(0, 7, (3, 2 * reach + 1), generator=g).to(torch.uint8)
    for width in (1, 3, 8, 9, 16, 32, 40, 64):
        n = 4 * width + 5 if width > 9 else 70
        at = torch.arange(n)
        pos = torch.stack([at // (2 * width), at // width, at % width], 1).to(torch.int32)
        q, k, v, dout = _sequences(g, 1, n, n, H, H, D, dt)
        say("width", width, dtype)
        _check(r, q, k, v, dout, dt, bias=(table, buckets, pos, pos))
    n = 100
    top = 2 ** 31 - 1
    pos = torch.randint(-12, 12, (n, 3), generator=g)
    pos[:40, 0] = top - 39 + torch.arange(40)       # counts up to the largest
    pos[40:72, 0] = -top - 1 + torch.arange(32)
    pos[:, 1] = torch.where(torch.arange(n) % 2 == 0, top, -top - 1)
    q, k, v, dout = _sequences(g, 1, n, n, H, H, D, dt)
    pos = pos.to(torch.int32)
    _check(r, q, k, v, dout, dt, bias=(table, buckets, pos, pos))


def test_buckets_by_distance():
    """The host's rule: near distances one bucket each, then by their logarithm."""
    b = mixrt.distance_buckets(16, 20, near=4)
    assert b.dtype == torch.uint8 and b.shape == (41,)
    assert b[20 - 3:21].tolist() == [3, 2, 1, 0] and b[21:25].tolist() == [8, 9, 10, 11]
    left, right = b[:21].flip(0).int(), b[21:].int()
    assert int(left.max()) == 7 and int(right.max()) == 15
    assert bool((left.diff() >= 0).all()) and bool((right.diff() >= 0).all())
    for n in range(4, 21):      # 4 (21/4)^((b - 4) / 4) <= n, the last such b
        want = max(c for c in range(4, 8) if 4 * (21 / 4) ** ((c - 4) / 4) <= n + 1e-9)
        assert int(left[n]) == want, n
    assert mixrt.distance_buckets(1, 3).tolist() == [0] * 7
    assert mixrt.distance_buckets(5, 0).tolist() == [0]
    for args in ((0, 3), (33, 3), (4, -1), (4, 128)):
        with pytest.raises(ValueError):
            mixrt.distance_buckets(*args)
    with pytest.raises(ValueError, match="near"):
        mixrt.distance_buckets(8, 3, near=5)


# --- gradients against differences, repeats, streams and graphs --------------------------

def test_gradients_against_differences(r):
    """Central differences of sum(dout * out), of the statement in 64 bits, in random
    directions: the kernels' gradients are the function's."""
    g = _gen(14)
    B, Tq, Tk, H, Hk, D = 2, 9, 23, 4, 2, 12
    q, k, v, dout = _sequences(g, B, Tq, Tk, H, Hk, D, torch.float32, sharp=1.0)
    bias = _bias(g, 2, 5, 6, B, Tq, Tk, H)
    lens = torch.tensor([23, 11], dtype=torch.int32)
    cuda = [t.cuda() for t in (q, k, v)]
    kw = dict(lens=lens.cuda(), bias=_on_gpu(bias))
    o, saved = r.attention_train(*cuda, **kw)
    grads = [t.double().cpu() for t in r.attention_backward(dout.cuda(), *cuda, o, saved, **kw)]
    inputs = [q.double(), k.double(), v.double(), bias[0].double()]

    def value(x):
        got = ref.attention(x[0], x[1], x[2], torch.float32, lens, (x[3], *bias[1:]))["o"][0]
        return float((got * dout.double()).sum())

    for n in range(4):
        way = torch.randn(inputs[n].shape, generator=g).double()
        if n in (1, 2):
            way[1, 11:] = 0
        step = 1e-4
        ends = []
        for sign in (step, -step):
            x = list(inputs)
            x[n] = x[n] + sign * way
            ends.append(value(x))
        want = (ends[0] - ends[1]) / (2 * step)
        got = float((grads[n] * way).sum())
        # the gradient's error in 32 bits, and the differences' of third order
        room = 2.0 ** -14 * float((grads[n].abs() * way.abs()).sum()) + 1e-6
        assert abs(got - want) <= room, (n, got, want)


def test_norm_gradients_against_differences(r):
    g = _gen(15)
    x, dy = (torch.randn((21, 3, 20), generator=g) for _ in range(2))
    w = 1 + 0.3 * torch.randn((20,), generator=g)
    pos = torch.randint(0, 30, (21, 2), generator=g).float()
    freq, axis = torch.rand(7, generator=g), (torch.arange(7) % 2).to(torch.uint8)
    dx, dw = (t.double().cpu() for t in r.rotary_norm_backward(
        dy.cuda(), x.cuda(), w.cuda(), pos.cuda(), freq.cuda(), axis.cuda(), eps=0.05))

    def value(x, w):
        return float((ref.rotary_norm(x, w, pos, freq, axis, "halves", 0.05, torch.float32)[0]
                      * dy.double()).sum())

    step = 1e-4
    for n, grad in enumerate((dx, dw)):
        way = torch.randn(grad.shape, generator=g).double()
        at = [x.double(), w.double()]
        ends = []
        for sign in (step, -step):
            moved = list(at)
            moved[n] = moved[n] + sign * way
            ends.append(value(*moved))
        got = float((grad * way).sum())
        room = 2.0 ** -15 * float((grad.abs() * way.abs()).sum()) + 1e-6
        assert abs(got - (ends[0] - ends[1]) / (2 * step)) <= room


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_heads_of_extreme_size(r, dtype):
    """Squares that leave the range of 32 bits either way, zeros, and values that are
    not finite: each head for itself."""
    dt = DT[dtype]
    g = _gen(16)
    top = 1e38 if dtype != "f16" else 6e4
    low = {"f32": 1e-40, "f16": 6e-8, "bf16": 1e-38}[dtype]
    x = torch.randn((6, 2, 48), generator=g)
    sizes = torch.tensor([top / 8, low, 1.0, 1e-3, low * 50, top / 100])[:, None, None]
    x = (x.clamp(-4, 4) * sizes).to(dt)
    dy = torch.randn((6, 2, 48), generator=g).to(dt)
    w = 1 + 0.3 * torch.randn((48,), generator=g)
    pos = torch.arange(6.0)[:, None]
    freq, axis = torch.rand(24, generator=g), torch.zeros(24, dtype=torch.uint8)
    place = (pos.cuda(), freq.cuda(), axis.cuda())
    for eps in (0.0, 1e-6):
        got = r.rotary_norm(x.cuda(), w.cuda(), *place, eps=eps)
        _inside(got, ref.rotary_norm(x, w, pos, freq, axis, "halves", eps, dt), ("out", eps))
        dx = r.rotary_norm_backward(dy.cuda(), x.cuda(), w.cuda(), *place, eps=eps)[0]
        want, bound = ref.rotary_norm_back(dy, x, w, pos, freq, axis, "halves", eps, dt)
        fits = want[0].abs() < 0.9 * torch.finfo(dt).max      # (others round to infinity)
        off = (dx.double().cpu() - want[0]).abs()
        assert bool((off <= bound[0])[fits].all()), eps
    bad = x.clone()
    bad[2, 0, 5], bad[3, 1, 7] = math.nan, math.inf
    got = r.rotary_norm(bad.cuda(), w.cuda(), *place).cpu()
    clean = r.rotary_norm(x.cuda(), w.cuda(), *place).cpu()
    assert bool(torch.isnan(got[2, 0]).all())
    assert bool(torch.isnan(got[3, 1, [7, 31]]).all())
    for t in (got, clean):
        t[2, 0] = t[3, 1] = 0
    assert torch.equal(got, clean)


def _step(rr, dt=torch.bfloat16):
    """A training step of the calls as they follow each other, and a serving one."""
    g = _gen(17)
    T, S, H, Hk, D = 300, 700, 4, 2, 32
    q = torch.randn((T, H, D), generator=g).to(dt).cuda()
    k = torch.randn((S, Hk, D), generator=g).to(dt).cuda()
    v = torch.randn((1, S, Hk, D), generator=g).to(dt).cuda()
    dout = torch.randn((1, T, H, D), generator=g).to(dt).cuda()
    w = [torch.rand(D, generator=g).cuda() for _ in range(2)]
    freq, axis = torch.rand(16, generator=g).cuda(), (torch.arange(16) % 2).byte().cuda()
    places = [torch.stack([torch.arange(n) // 20, torch.arange(n) % 20], 1) for n in (T, S)]
    pos = [p.float().cuda() for p in places]
    table = torch.randn((2, 8, H), generator=g).cuda()
    buckets = torch.stack([mixrt.distance_buckets(8, 10)] * 2).cuda()
    bias = mixrt.RelativeBias(table, buckets, *[p.int().cuda() for p in places])
    lens = torch.tensor([690], dtype=torch.int32).cuda()
    torch.cuda.synchronize()

    def run():
        qn = rr.rotary_norm(q, w[0], pos[0], freq, axis)
        kn = rr.rotary_norm(k, w[1], pos[1], freq, axis)
        kw = dict(lens=lens, bias=bias)
        served = rr.attention(qn[None], kn[None], v, **kw)
        one = rr.attention(qn[None, :1], kn[None], v)
        o, saved = rr.attention_train(qn[None], kn[None], v, **kw)
        dq, dk, dv, dtable = rr.attention_backward(dout, qn[None], kn[None], v, o, saved, **kw)
        dx, dw = rr.rotary_norm_backward(dq[0], q, w[0], pos[0], freq, axis)
        dy, du = rr.rotary_norm_backward(dk[0], k, w[1], pos[1], freq, axis)
        return [qn, kn, served, one, o, saved.lse, dq, dk, dv, dtable, dx, dw, dy, du]
    return run


def test_the_same_bits_again_and_on_another_stream(r):
    first = _step(r)()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, _step(r)()))
    torch.cuda.synchronize()
    other = mixrt.Renderer(0, stream=torch.cuda.Stream())
    try:
        got = _step(other)()
        other.sync()
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    finally:
        other.close()


def test_two_captured_steps_replay_beside_eager_calls(r):
    """Graphs of one context have scratch of their own; every replay gives the eager
    outputs."""
    stream = torch.cuda.Stream()
    c = mixrt.Renderer(0, stream=stream)
    try:
        steps = [_step(c), _step(c, torch.float16)]
        want = [[t.clone() for t in s()] for s in steps]
        c.sync()
        graphs, outs = [], []
        for s in steps:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(s())
            graphs.append(graph)
        scratch = c._ws[2]
        for rep in range(3):
            scratch.fill_(77)
            for o in outs:
                for t in o:
                    t.zero_()
            torch.cuda.synchronize()
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            assert bool((scratch == 77).all())
            for o, w in zip(outs, want):
                assert all(torch.equal(a, b) for a, b in zip(o, w)), rep
            r.attention(*[torch.ones((1, 40, 1, 16), device="cuda")] * 3)
    finally:
        c.close()


def test_lengths_that_change_between_replays(r):
    """Lengths are read when the call runs: a graph sees new ones."""
    g = _gen(18)
    q, k, v, _ = [t.cuda() for t in _sequences(g, 2, 40, 90, 2, 2, 32, torch.float32)]
    lens = torch.tensor([90, 10], dtype=torch.int32).cuda()
    stream = torch.cuda.Stream()
    c = mixrt.Renderer(0, stream=stream)
    try:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = c.attention(q, k, v, lens=lens)
        for new in ([90, 10], [3, 90], [0, 1]):
            lens.copy_(torch.tensor(new, dtype=torch.int32))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, r.attention(q, k, v, lens=lens)), new
    finally:
        c.close()


# --- what is refused --------------------------------------------------------------------

def test_binding_refuses_wrong_tensors(r):
    q = torch.zeros((2, 5, 4, 16), device="cuda")
    k = torch.zeros((2, 7, 2, 16), device="cuda")
    with pytest.raises(ValueError, match="kv_heads a divisor"):
        r.attention(q, k[:, :, :1].expand(-1, -1, 3, -1), k[:, :, :1].expand(-1, -1, 3, -1))
    with pytest.raises(ValueError, match="expected"):
        r.attention(q, k, k[:, :6])
    with pytest.raises(ValueError, match="one dtype"):
        r.attention(q, k.half(), k.half())
    with pytest.raises(ValueError, match="dtype"):
        r.attention(q.double(), k.double(), k.double())
    with pytest.raises(ValueError, match="expected cuda"):
        r.attention(q, k.cpu(), k)
    with pytest.raises(ValueError, match="neighbours"):
        r.attention(q.transpose(2, 3).contiguous().transpose(2, 3), k, k)
    with pytest.raises(ValueError, match="4 dim|dimensions"):
        r.attention(q[0], k[0], k[0])
    with pytest.raises(ValueError, match="lens"):
        r.attention(q, k, k, lens=torch.tensor([1, 2]).cuda())
    with pytest.raises(ValueError, match="lens"):
        r.attention(q, k, k, lens=torch.tensor([1], dtype=torch.int32).cuda())
    with pytest.raises(TypeError, match="tensor|Tensor"):
        r.attention(q, k, k, lens=[1, 2])
    with pytest.raises(mixrt.MixrtError, match="head_dim"):
        wide = torch.zeros((1, 2, 1, 129), device="cuda")
        r.attention(wide, wide, wide)
    for scale in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(mixrt.MixrtError, match="scale"):
            r.attention(q, k, k, scale=scale)
    with pytest.raises(mixrt.MixrtError, match="overlap"):
        r.attention(q, k, k, out=torch.zeros((2, 1, 4, 16), device="cuda").expand(-1, 5, -1, -1))
    with pytest.raises(mixrt.MixrtError, match="also another"):
        r.attention(q, k, k, out=q)
    with pytest.raises(ValueError, match="out"):
        r.attention(q, k, k, out=q[:1])
    o, saved = r.attention_train(q.half(), k.half(), k.half())
    args = (q.half(), k.half(), k.half(), o)
    with pytest.raises(ValueError, match="dout"):
        r.attention_backward(q, *args, saved)
    with pytest.raises(TypeError, match="AttentionSaved"):
        r.attention_backward(q.half(), *args, saved.lse)
    with pytest.raises(ValueError, match="lse"):
        r.attention_backward(q.half(), *args, mixrt.AttentionSaved(saved.lse[:1], saved.rest))
    with pytest.raises(TypeError, match="rest"):
        r.attention_backward(q.half(), *args, mixrt.AttentionSaved(saved.lse, None))


def test_outputs_that_share_memory_with_inputs(r):
    """An output over a part of an input is refused, one beside the inputs in a joint
    array is not, and gives what an array of its own gives."""
    g = _gen(31)
    buf = torch.randn((2, 9, 4, 16), generator=g).cuda()
    q, k = buf[:, :7], torch.randn((2, 7, 2, 16), generator=g).cuda()
    for out in (buf[:, 1:8], buf[:, 2:]):
        with pytest.raises(mixrt.MixrtError, match="also another"):
            r.attention(q, k, k, out=out)
    # half a head further
    flat = torch.zeros(2 * 7 * 4 * 16 + 8, device="cuda")
    with pytest.raises(mixrt.MixrtError, match="also another"):
        r.attention(flat[:-8].view(2, 7, 4, 16), k, k, out=flat[8:].view(2, 7, 4, 16))
    # heads of one token behind each other: q, out, k, v, in either order of dimensions
    joint = torch.randn((2, 7, 4 + 4 + 2 + 2, 16), generator=g).cuda()
    q, out, k, v = joint.split([4, 4, 2, 2], 2)
    want = r.attention(q, k, v)
    keep = [t.clone() for t in (q, k, v)]
    r.attention(q, k, v, out=out)
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(keep, (q, k, v)))
    wide = torch.randn((2, 4, 7, 64), generator=g).cuda().transpose(1, 2)
    q, out, k, v = wide.split(16, 3)
    want = r.attention(q, k, v)
    r.attention(q, k, v, out=out)
    assert torch.equal(out, want)
    # arrays behind each other in one allocation
    rows = torch.randn((3, 2, 7, 4, 16), generator=g).cuda()
    want = r.attention(rows[0], rows[1], rows[1])
    r.attention(rows[0], rows[1], rows[1], out=rows[2])
    assert torch.equal(rows[2], want)


def test_binding_refuses_a_wrong_bias(r):
    q = torch.zeros((2, 5, 4, 16), device="cuda")
    table, buckets = torch.zeros((2, 3, 4)), torch.zeros((2, 9)).byte()
    pos = torch.zeros((5, 2)).int()
    good = [t.cuda() for t in (table, buckets, pos, pos)]
    r.attention(q, q, q, bias=mixrt.RelativeBias(*good))
    wrong = [(0, table[:, :, :3]), (0, table.double()), (0, table[0]), (1, buckets[:1]),
             (1, buckets[:, :8]), (1, buckets.int()), (2, pos[:4]), (2, pos.long()),
             (3, pos[None].expand(3, -1, -1)), (3, pos[:, :1])]
    for n, t in wrong:
        bad = list(good)
        bad[n] = t.contiguous().cuda()
        with pytest.raises(ValueError, match="bias"):
            r.attention(q, q, q, bias=mixrt.RelativeBias(*bad))
    with pytest.raises(ValueError, match="expected cuda"):
        r.attention(q, q, q, bias=mixrt.RelativeBias(table, *good[1:]))
    for shape, what in (((4, 3, 4), "axes"), ((2, 33, 4), "count")):
        bad = [torch.zeros(shape), torch.zeros((shape[0], 9)).byte(),
               *[torch.zeros((5, shape[0])).int()] * 2]
        with pytest.raises(mixrt.MixrtError, match=what):
            r.attention(q, q, q, bias=mixrt.RelativeBias(*[t.cuda() for t in bad]))
    bad = [good[0], torch.zeros((2, 257)).byte().cuda(), *good[2:]]
    with pytest.raises(mixrt.MixrtError, match="reach"):
        r.attention(q, q, q, bias=mixrt.RelativeBias(*bad))


def test_buckets_out_of_range_are_the_last(r):
    """As the declaration says: no place outside the table is read."""
    g = _gen(19)
    q, k, v, dout = _sequences(g, 1, 40, 50, 2, 2, 16, torch.float32)
    table, buckets, qp, kp = _bias(g, 1, 5, 8, 1, 40, 50, 2)
    wild = torch.where(buckets == 4, 200, buckets.int()).to(torch.uint8)
    cuda = [t.cuda() for t in (q, k, v)]
    results = []
    for b in (buckets, wild):
        kw = dict(bias=_on_gpu((table, b, qp, kp)))
        o, saved = r.attention_train(*cuda, **kw)
        results.append((o, *r.attention_backward(dout.cuda(), *cuda, o, saved, **kw)))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_rotary_norm_refusals(r):
    x = torch.zeros((5, 2, 8), device="cuda")
    pos, freq = torch.zeros((5, 1), device="cuda"), torch.ones(4, device="cuda")
    axis = torch.zeros(4, device="cuda").byte()
    w = torch.ones(8, device="cuda")
    with pytest.raises(ValueError, match="weights"):
        r.rotary_norm(x, w[:7], pos, freq, axis)
    with pytest.raises(ValueError, match="weights"):
        r.rotary_norm(x, w.half(), pos, freq, axis)
    with pytest.raises(ValueError, match="2 arrays and 1 weights"):
        r.rotary_norm((x, x), (w,), pos, freq, axis)
    with pytest.raises(ValueError, match="tokens"):
        r.rotary_norm(x, w, pos[:4], freq, axis)
    with pytest.raises(mixrt.MixrtError, match="eps"):
        r.rotary_norm(x, w, pos, freq, axis, eps=-1.0)
    with pytest.raises(mixrt.MixrtError, match="pairs"):
        r.rotary_norm(x, w, pos, torch.ones(5, device="cuda"), torch.zeros(5).byte().cuda())
    with pytest.raises(mixrt.MixrtError, match="overlap"):
        r.rotary_norm(x, w, pos, freq, axis, out=torch.zeros(8, device="cuda").expand(5, 2, 8))
    with pytest.raises(ValueError, match="grads"):
        r.rotary_norm_backward(x[:4], x, w, pos, freq, axis)
    with pytest.raises(mixrt.MixrtError, match="dx is x"):
        r.rotary_norm_backward(x.clone(), x, w, pos, freq, axis, out=x)
    with pytest.raises(TypeError):
        r.rotary_norm(x, [1.0] * 8, pos, freq, axis)


def test_numbers_that_change_in_place(r):
    """A scale or an epsilon given as a tensor counts by its value."""
    x = torch.randn((1, 20, 2, 16), generator=_gen(20)).cuda()
    scale = torch.tensor(0.5)
    first = r.attention(x, x, x, scale=scale)
    assert torch.equal(first, r.attention(x, x, x, scale=0.5))
    scale.fill_(0.01)
    assert torch.equal(r.attention(x, x, x, scale=scale), r.attention(x, x, x, scale=0.01))
    pos, freq = torch.zeros((20, 1), device="cuda"), torch.ones(8, device="cuda")
    axis, eps = torch.zeros(8, device="cuda").byte(), torch.tensor(1e-3)
    first = r.rotary_norm(x[0], None, pos, freq, axis, eps=eps)
    assert torch.equal(first, r.rotary_norm(x[0], None, pos, freq, axis, eps=float(eps)))
    eps.fill_(2.0)
    assert torch.equal(r.rotary_norm(x[0], None, pos, freq, axis, eps=eps),
                       r.rotary_norm(x[0], None, pos, freq, axis, eps=2.0))


def test_a_gradient_is_refused_rather_than_dropped(r):
    g = _gen(21)
    x = torch.randn((1, 20, 2, 16), generator=g).cuda()
    pos, freq = torch.zeros((20, 1), device="cuda"), torch.ones(8, device="cuda")
    axis, w = torch.zeros(8, device="cuda").byte(), torch.ones(16, device="cuda")
    table = torch.zeros((1, 3, 2), device="cuda")
    places = torch.arange(20, device="cuda").int()[:, None]
    buckets = torch.zeros((1, 5), device="cuda").byte()

    def biased(t):
        return r.attention(x, x, x, bias=mixrt.RelativeBias(t, buckets, places, places))

    o, saved = r.attention_train(x, x, x)
    calls = {
        "q": (lambda a: r.attention(a, x, x), x),
        "v": (lambda a: r.attention(x, x, a), x),
        "table": (biased, table),
        "train": (lambda a: r.attention_train(x, a, x)[0], x),
        "lse": (lambda a: r.attention_train(x, a, x)[1].lse, x),
        "backward": (lambda a: r.attention_backward(a, x, x, x, o, saved)[1], x),
        "rotary_norm": (lambda a: r.rotary_norm(a, w, pos, freq, axis), x[0]),
        "weight": (lambda a: r.rotary_norm(x[0], a, pos, freq, axis), w),
        "rotary_norm_backward": (lambda a: r.rotary_norm_backward(a, x[0], w, pos, freq,
                                                                  axis)[1], x[0]),
    }
    for name, (call, t) in calls.items():
        leaf = t.clone().requires_grad_()
        got = call(leaf)
        assert torch.equal(got.detach(), call(t)), name
        with pytest.raises(RuntimeError, match="no derivative"):
            got.sum().backward()
        with torch.no_grad():
            assert not call(leaf).requires_grad
    leaf = x.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="out="):
        r.attention(leaf, x, x, out=torch.empty_like(x))
    with pytest.raises(RuntimeError, match="out="):
        r.rotary_norm(leaf[0], w, pos, freq, axis, out=torch.empty_like(x[0]))


# --- sums over many keys ------------------------------------------------------------------

def test_many_equal_keys(r):
    """200,000 equal keys: every weight is the same, and sums of equal terms lean one
    way.  A chain is at most 2048 keys (two of them a matrix instruction), so the
    output is off by about half of 1024 roundings and a few joins; a mean of equal
    values is the value."""
    n = 200_000
    q = torch.ones((1, 40, 1, 16), device="cuda")
    k = torch.full((1, 1, 1, 16), 0.1, device="cuda").expand(-1, n, -1, -1)
    v = torch.full((1, 1, 1, 16), 0.7, device="cuda").expand(-1, n, -1, -1)
    o, saved = r.attention_train(q, k, v)
    off = float((o.double() / float(v[0, 0, 0, 0].double()) - 1).abs().max())
    say(f"off by {off / ref.U:.0f} u")
    assert off <= ref.U * (1024 + 300)
    want = (float((q[0, 0, 0].double() * 0.25 * k[0, 0, 0].double()).sum()) + math.log(n)) / \
        math.log(2)
    assert abs(float(saved.lse[0, 0, 0]) - want) <= 1400 * ref.U * abs(want)
