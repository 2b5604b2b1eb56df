"""Limits of the refiner's operators: inputs, sizes and arguments at which a
result could be wrong without an error, each against a 64-bit statement or
against what the call promises."""
import ctypes as C
import math

import pytest

import refine_ref as ref
from paper_2312_11841_amd import mixrt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": mixrt.MIXRT_F32, "f16": mixrt.MIXRT_F16, "bf16": mixrt.MIXRT_BF16}


@pytest.fixture(scope="module")
def r():
    r = mixrt.Renderer(0, sync_check=True)
    yield r
    r.close()


def say(*a):
    print(*a, flush=True)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# --- a NaN of any bit pattern --------------------------------------------------------

NANS = {"f32": (torch.int32, (0x7fffffff, 0xffffffff, 0x7fc00001, 0x7f800001, 0xff8000ff,
                              0x7fc0007f, 0x7fc00080)),
        "f16": (torch.int16, (0x7fff, 0xffff, 0x7e01, 0x7c01, 0xfc7f)),
        "bf16": (torch.int16, (0x7fff, 0xffff, 0x7fc1, 0x7f81, 0xff9f))}


@pytest.mark.parametrize("dtype", list(NANS))
def test_a_nan_of_any_bits_is_kept_as_one(r, dtype):
    """A group that held a NaN has codes 0 and byte 255 and reads back as NaN,
    whatever the NaN's payload and sign are; its weights' gradients are NaN."""
    bits, patterns = NANS[dtype]
    wide = 1 << (32 if bits == torch.int32 else 16)
    n, width = len(patterns), 70
    x = torch.randn((n, width), generator=_gen(1)).to(DT[dtype])
    raw = x.view(bits)
    for i, p in enumerate(patterns):
        raw[i, 3 + 7 * i] = p - wide if p >= wide // 2 else p     # groups 0 and 1
    assert int(torch.isnan(x).sum()) == n
    say("nan", dtype)
    hit = torch.isnan(x)
    groups = torch.stack([hit[:, :32].any(1), hit[:, 32:64].any(1), hit[:, 64:].any(1)], 1)
    held = groups.repeat_interleave(32, 1)[:, :width]
    x = x.cuda()
    by_norm = r.group_norm_train(x.reshape(1, n, width), 7)[2]
    for kept in (r.checkpoint_pack(x), by_norm):
        assert torch.equal(kept.exps.cpu() == 255, groups)
        assert not bool(kept.codes.cpu()[held].any())
        for odt in DT.values():
            assert torch.equal(torch.isnan(r.checkpoint_unpack(kept, dtype=odt)).cpu(), held)
        for outs in (4, 65):       # rows dealt to lanes, and tiles
            dw, _ = r.linear_weight_grad(kept, torch.ones((n, outs), dtype=DT[dtype],
                                                          device="cuda"))
            want = held.any(0)[:, None].expand(width, outs)
            assert torch.equal(torch.isnan(dw).cpu(), want)
            assert bool(torch.isfinite(dw.cpu()[~want]).all())


# --- sums over very many rows ---------------------------------------------------------
#
# m equal terms added one after another in 32 bits are off by at most u m / 2 of
# the sum: the k-th addition rounds k terms.

@pytest.mark.parametrize("dtype", list(DT))
def test_linear_gradient_of_many_equal_rows(r, dtype):
    """A wide layer over 921,600 rows, all of them the same: its rows are one
    part.  At most 1024 additions of a wave go one after another, then its sums
    are moved on."""
    rows, width = 921_600, 2048
    dt = DT[dtype]
    say("equal rows", dtype)
    codes = torch.full((rows, width), 64, dtype=torch.int8, device="cuda")
    exps = torch.full((rows, width // 32), 127 - 6, dtype=torch.uint8, device="cuda")
    dy = torch.full((1, 1), 0.1, dtype=dt, device="cuda")
    each = float(dy.double())
    # (the columns of dy are neighbours in one row that all rows share)
    dy = dy.expand(1, width).contiguous().expand(rows, width)
    dw, db = r.linear_weight_grad(mixrt.Checkpoint(codes, exps, dt), dy)
    want = rows * each
    bound = ref.U * (1024 / 2 + 57 + 16)
    for got in (dw, db):
        off = float((got.double() / want - 1).abs().max())
        say(f"off by {off / ref.U:.0f} u, may be {bound / ref.U:.0f}")
        assert off <= bound


def test_linear_gradient_of_many_rows_and_a_short_gradient(r):
    """Two outs that all rows share, 130 channels: a thread's sum a weight."""
    rows, width = 1 << 24, 130
    codes = torch.full((rows, width), 64, dtype=torch.int8, device="cuda")
    exps = torch.full((rows, 5), 127 - 6, dtype=torch.uint8, device="cuda")
    dy = torch.full((1, 2), 0.1, dtype=torch.float16, device="cuda")
    each = float(dy[0, 0].double())
    dw, db = r.linear_weight_grad(mixrt.Checkpoint(codes, exps, torch.float16),
                                  dy.expand(rows, 2))
    for got in (dw, db):
        off = float((got.double() / (rows * each) - 1).abs().max())
        say(f"off by {off / ref.U:.0f} u")
        # a part in 64 bits, rounded; up to 4096 parts by 32 threads and a tree
        assert off <= ref.U * (128 / 2 + 8)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
def test_linear_gradient_of_long_ragged_parts(r, dtype, shared):
    """Widths that are no multiples of a vector, in parts of several chains;
    with rows of dy that repeat, which are read without vectors past the row."""
    rows, width, outs = 30_011, 1101, 1030
    dt = DT[dtype]
    say("long parts", dtype, shared)
    g = torch.Generator("cuda").manual_seed(3)
    kept = r.checkpoint_pack(torch.randn((rows, width), generator=g, device="cuda").to(dt))
    dy = torch.randn((1 if shared else rows, outs), generator=g, device="cuda").to(dt)
    dy = dy.expand(rows, outs)
    dw, db = r.linear_weight_grad(kept, dy)
    xv, dv = r.checkpoint_unpack(kept).double(), dy.double().contiguous()
    # 1024 additions, the moves to LDS of four waves, the sums of the waves
    scale = ref.U * (1024 + 2 * 16 + 8)
    xt = xv.t().contiguous()
    assert bool(((dw.double() - xt @ dv).abs() <= scale * (xt.abs() @ dv.abs())).all())
    assert bool(((db.double() - dv.sum(0)).abs() <= scale * dv.abs().sum(0)).all())


def test_linear_gradient_of_very_many_narrow_rows(r):
    """2^28 equal rows of one channel and four outs: about 1024 rows a lane,
    then 32 lanes' and blocks' sums in trees and runs."""
    rows = 1 << 28
    codes = torch.full((rows, 1), 64, dtype=torch.int8, device="cuda")
    exps = torch.full((rows, 1), 127 - 6, dtype=torch.uint8, device="cuda")
    dy = torch.full((1, 4), 0.1, device="cuda")
    dw, db = r.linear_weight_grad(mixrt.Checkpoint(codes, exps, torch.float32),
                                  dy.expand(rows, 4))
    want = rows * float(dy[0, 0].double())
    for got in (dw, db):
        off = float((got.double() / want - 1).abs().max())
        say(f"off by {off / ref.U:.0f} u")
        # a lane's rows; 6 steps of a wave, 4 waves, 32 parts a thread, 5 steps
        assert off <= ref.U * ((1024 + 32) / 2 + 6 + 4 + 5)


@pytest.mark.parametrize("dtype", list(DT))
def test_norm_gradient_of_many_equal_rows(r, dtype):
    """128 images of 131,072 equal pixels, wide rows: at most 128 rows of a
    thread are added in 32 bits, then in 64.  (The map is one pixel that
    repeats; dx is not asked for.)"""
    N, P, width, G = 128, 1 << 17, 1024, 8
    dt = DT[dtype]
    say("equal pixels", dtype)
    dy = torch.full((width,), 0.1, dtype=dt, device="cuda")
    x = torch.full((width,), 0.75, dtype=dt, device="cuda")
    stats = torch.tensor([0.25, 1.7], device="cuda").repeat(N, G, 1)
    norm = mixrt.Norm(N, width, P, G, CODE[dtype], 0, 1e-5, 0, 0)
    size = C.c_size_t()
    assert r._L.mixrt_norm_workspace(C.byref(norm), C.byref(size)) == 0
    ws = torch.empty((size.value,), dtype=torch.uint8, device="cuda")
    grads = torch.zeros((2, width), device="cuda")
    one = lambda t: C.byref(mixrt.Map(t.data_ptr(), 0, 0))  # noqa: E731
    r._check(r._L.mixrt_norm_backward(r._h, C.byref(norm), one(dy), one(x), None,
                                      stats.data_ptr(), None, grads[0].data_ptr(),
                                      grads[1].data_ptr(), ws.data_ptr(), size.value))
    r.sync()
    d = float(dy[0].double())
    xh = 0.5 * float(stats[0, 0, 1].double())
    for got, want, terms in ((grads[0], N * P * d * xh, 4), (grads[1], N * P * d, 2)):
        off = float((got.double() / want - 1).abs().max())
        say(f"off by {off / ref.U:.0f} u")
        # 128 rows, up to 8 steps that join a block's rows, the term and its sum
        assert off <= ref.U * (128 / 2 + 8 + terms)


# --- scratch of captured calls ---------------------------------------------------------

def test_a_captured_call_has_scratch_of_its_own(r):
    """A replay may run beside eager calls or another graph of the same
    context: it must not write where they do."""
    g = _gen(2)
    x = torch.randn((1, 30000, 32), generator=g).to(torch.float16).cuda()
    dy = torch.randn((1, 30000, 32), generator=g).to(torch.float16).cuda()
    stream = torch.cuda.Stream()
    c = mixrt.Renderer(0, stream=stream)

    def step():
        y, stats, kept = c.group_norm_train(x, 8, act="silu")
        return (y, *c.group_norm_backward(dy, kept, stats, act="silu"),
                *c.linear_weight_grad(kept, dy.reshape(-1, 32)))

    try:
        torch.cuda.synchronize()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = step()
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
        scratch = c._ws[2]
        for _ in range(3):
            scratch.fill_(77)
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert bool((scratch == 77).all())
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
    finally:
        c.close()
    assert c._ws is None     # given back


def test_a_capture_before_any_eager_call(r):
    """The first call of a context may be a captured one."""
    x = torch.randn((1, 30000, 32), generator=_gen(3)).to(torch.bfloat16).cuda()
    want = r.group_norm(x, 8, act="relu")
    stream = torch.cuda.Stream()
    c = mixrt.Renderer(0, stream=stream)
    try:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = c.group_norm(x, 8, act="relu")
        again = c.group_norm(x, 8, act="relu")
        for _ in range(3):
            out.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(again, want)
    finally:
        c.close()


# --- maps without pixels -----------------------------------------------------------------

@pytest.mark.parametrize("shape", [(3, 0, 1024, 8), (1, 0, 4095, 1), (2, 0, 640, 640),
                                   (70, 0, 8, 2)], ids=str)
def test_maps_without_pixels(r, shape):
    """Wide maps too: statistics of nothing, gradients 0."""
    N, P, width, G = shape
    say("no pixels", shape)
    for dt in DT.values():
        x = torch.empty((N, P, width), dtype=dt, device="cuda")
        y, stats, kept = r.group_norm_train(x, G, eps=0.25)
        assert y.shape == x.shape
        assert torch.equal(stats.cpu(), torch.tensor([0.0, 2.0]).expand(N, G, 2))
        for saved in (kept, x):
            dx, dgamma, dbeta = r.group_norm_backward(x, saved, stats)
            assert dx.shape == x.shape
            assert float(dgamma.abs().sum()) == 0.0 == float(dbeta.abs().sum())


def test_maps_without_pixels_from_c(r):
    """Maps at addresses of their own, of which nothing is read."""
    some = torch.zeros((64,), device="cuda")
    norm = mixrt.Norm(2, 8, 0, 2, mixrt.MIXRT_F32, 1, 0.25, 0, 0)
    stats = torch.zeros((2, 2, 2), device="cuda")
    size = C.c_size_t()
    assert r._L.mixrt_norm_workspace(C.byref(norm), C.byref(size)) == 0
    ws = torch.empty((size.value,), dtype=torch.uint8, device="cuda")
    r._check(r._L.mixrt_norm_forward(
        r._h, C.byref(norm), C.byref(mixrt.Map(some.data_ptr(), 0, 8)),
        C.byref(mixrt.Map(some.data_ptr() + 128, 0, 8)), stats.data_ptr(), None, ws.data_ptr(),
        size.value))
    r.sync()
    assert torch.equal(stats.cpu(), torch.tensor([0.0, 2.0]).expand(2, 2, 2))


# --- arguments that change between calls -----------------------------------------------

def test_an_epsilon_that_changes_in_place(r):
    x = torch.randn((1, 50, 8), generator=_gen(4)).cuda()
    eps = torch.tensor(1e-3)
    first = r.group_norm(x, 2, eps=eps)
    assert torch.equal(first, r.group_norm(x, 2, eps=float(eps)))
    eps.fill_(4.0)
    assert torch.equal(r.group_norm(x, 2, eps=eps), r.group_norm(x, 2, eps=4.0))
    groups = torch.tensor(2)
    first = r.group_norm(x, groups)
    groups.fill_(4)
    assert torch.equal(r.group_norm(x, groups), r.group_norm(x, 4))
    assert not torch.equal(first, r.group_norm(x, 4))
    with pytest.raises(ValueError, match="groups"):
        r.group_norm(x, 2.5)


def test_a_direction_that_changes_in_place(r):
    x = torch.randn((5, 2, 8), generator=_gen(5)).cuda()
    pos, freq = torch.arange(5.0, device="cuda")[:, None], torch.ones(4, device="cuda")
    axis = torch.zeros(4, dtype=torch.uint8, device="cuda")
    way = torch.tensor(False)
    assert torch.equal(r.rotary(x, pos, freq, axis, inverse=way), r.rotary(x, pos, freq, axis))
    way.fill_(True)
    assert torch.equal(r.rotary(x, pos, freq, axis, inverse=way),
                       r.rotary(x, pos, freq, axis, inverse=True))


# --- gradients that a graph asks for ----------------------------------------------------

def test_a_gradient_is_refused_rather_than_dropped(r):
    """The calls have no derivative for torch's graph: a backward pass that
    reaches one says so, and values are as without a graph."""
    g = _gen(6)
    x = torch.randn((1, 50, 8), generator=g).cuda()
    gamma = torch.ones(8, device="cuda")
    q = torch.randn((5, 2, 8), generator=g).cuda()
    pos, freq = torch.arange(5.0, device="cuda")[:, None], torch.ones(4, device="cuda")
    axis = torch.zeros(4, dtype=torch.uint8, device="cuda")
    _, stats, kept = r.group_norm_train(x, 2, gamma)
    calls = {
        "group_norm": (lambda a: r.group_norm(a, 2, gamma), x),
        "group_norm gamma": (lambda a: r.group_norm(x, 2, a), gamma),
        "group_norm_train": (lambda a: r.group_norm_train(a, 2, gamma)[0], x),
        "group_norm_train stats": (lambda a: r.group_norm_train(a, 2, gamma)[1], x),
        "group_norm_backward": (lambda a: r.group_norm_backward(a, kept, stats, gamma)[0], x),
        "group_norm_backward dgamma": (lambda a: r.group_norm_backward(a, kept, stats,
                                                                       gamma)[1], x),
        "linear_weight_grad": (lambda a: r.linear_weight_grad(kept, a)[0], x),
        "rotary": (lambda a: r.rotary(a, pos, freq, axis), q),
        "rotary keys": (lambda a: r.rotary((q, a), pos, freq, axis)[1], q),
    }
    for name, (call, at) in calls.items():
        want = call(at)
        assert not want.requires_grad, name
        leaf = at.clone().requires_grad_()
        with torch.no_grad():
            assert not call(leaf).requires_grad, name
        got = call(leaf)
        assert torch.equal(got, want), name
        other = torch.ones((), device="cuda", requires_grad=True)
        with pytest.raises(RuntimeError, match=name.split()[0]):
            (got * other).sum().backward()
        assert leaf.grad is None, name
        if name in ("group_norm", "rotary"):
            with pytest.raises(RuntimeError, match="out"):
                if name == "rotary":
                    r.rotary(leaf, pos, freq, axis, out=torch.empty_like(q))
                else:
                    r.group_norm(leaf, 2, gamma, out=torch.empty_like(x))


# --- the activations' tails ----------------------------------------------------------------

def _at(r, z, act):
    """(act(z), its slope) by the norm's kernels: with gamma 0, z is beta."""
    z = z.float().cuda()
    width = z.numel()
    x = torch.linspace(-1, 1, width, device="cuda").reshape(1, 1, width)
    gamma = torch.zeros(width, device="cuda")
    y, stats, _ = r.group_norm_train(x, 1, gamma, z, act=act)
    slope = r.group_norm_backward(torch.ones_like(x), x, stats, gamma, z, act=act)[2]
    return y.double().cpu().reshape(-1), slope.double().cpu()


def test_gelu_keeps_its_relative_accuracy_in_the_negative_tail(r):
    """Half of erfc(|z| / sqrt 2) is good to (24 + 2 z^2) u: its exponent z^2 / 2
    carries three roundings, which act on the value z^2 / 2 times each; 2.6 u of
    the polynomial, 9 for its argument, the rest for the operations."""
    z = torch.linspace(-8, 8, 4001).float().double()
    y, slope = _at(r, z, "gelu")
    half = 0.5 * torch.erfc(z.abs() / math.sqrt(2))
    phi = torch.where(z < 0, half, 1 - half)
    density = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    rel = ref.U * (24 + 2 * z * z)
    want = z * phi
    bound = z.abs() * half * rel + 2 * ref.U * want.abs()
    assert bool(((y - want).abs() <= bound).all()), float(((y - want).abs() / bound).max())
    want = phi + z * density
    bound = (half + z.abs() * density) * rel + 2 * ref.U * (phi + want.abs())
    assert bool(((slope - want).abs() <= bound).all()), float(((slope - want).abs() / bound).max())


def test_silu_keeps_its_relative_accuracy_in_the_negative_tail(r):
    """exp(-z) is good to (2 |z| + 4) u, as its argument in bits is a rounded
    product with a rounded constant; four more operations.  The slope
    s (1 + z (1 - s)) is a sum of s and z s (1 - s)."""
    z = torch.linspace(-80, 40, 4001).float().double()
    y, slope = _at(r, z, "silu")
    s = torch.sigmoid(z)
    rel = ref.U * (2 * z.abs() + 12)
    assert bool(((y - z * s).abs() <= (z * s).abs() * rel).all())
    rest = torch.sigmoid(-z)
    want = s + z * s * rest
    # the kernel forms 1 - s as a difference: u of z beside what it leaves
    bound = (s + z.abs() * s * rest) * rel + 4 * ref.U * z.abs() * s
    assert bool(((slope - want).abs() <= bound).all()), float(((slope - want).abs() / bound).max())


# --- activations of extreme size ---------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e24, 1e-24, 1e34, 1e-34])
def test_gradient_of_activations_of_extreme_size(r, size, dtype):
    """1 / deviation squared leaves the range of 32 bits; dx does not."""
    g = _gen(7)
    shapes = [(1, 64, 8, 2), (2, 20000, 16, 2)]
    for N, P, width, G in shapes:
        x0 = torch.randn((N, P, width), generator=g)
        x = (x0 * size).to(DT[dtype]).cuda()
        dy = (x0 + 0.1 * torch.randn((N, P, width), generator=g)).to(DT[dtype]).cuda()
        _, stats, _ = r.group_norm_train(x, G, eps=0.0, act="silu")
        gamma, beta = torch.ones(width), torch.zeros(width)
        for kind in ("none", "silu"):
            dx, dgamma, dbeta = r.group_norm_backward(dy, x, stats, act=kind)
            want, bound = ref.norm_back(dy.cpu(), x.cpu(), stats.cpu(), gamma, beta, kind,
                                        DT[dtype])
            for name, got in (("dx", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
                over = (got.double().cpu() - want[name]).abs() - bound[name]
                assert float(over.max()) <= 0, (size, kind, name, P)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_activations_of_values_that_are_not_finite(r, act):
    """A NaN stays one in the value and in the slope; plus infinity is its own
    value where the activation is not a step."""
    z = torch.tensor([math.nan, math.inf, 1e30, -1e30, 0.0])
    y, slope = _at(r, z, act)
    assert math.isnan(y[0]) and (act == "none" or math.isnan(slope[0]))
    assert y[1] == math.inf
    assert y[2] == float(z[2].double()) and y[4] == 0.0
    assert float(y[3]) == (float(z[3].double()) if act == "none" else 0.0)
    if act != "none":
        assert slope[2] == 1.0 and slope[3] == 0.0
        assert slope[4] == (0.0 if act == "relu" else 0.5)
