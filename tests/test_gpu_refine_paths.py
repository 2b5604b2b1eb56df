"""Group norm's launch paths for large maps (refine_paths.py says which shape
takes which) against the 64-bit statement: forward, forward that keeps x, and
the gradients from the kept form and from x, with relu among the activations;
and the outputs that a caller of the C ABI may leave out."""
import ctypes as C

import pytest

import refine_ref as ref
from paper_2312_11841_amd import mixrt
from refine_paths import PATHS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SHAPES = list(PATHS)


@pytest.fixture(scope="module")
def r():
    r = mixrt.Renderer(0, sync_check=True)
    yield r
    r.close()


def say(*a):
    print(*a, flush=True)


def _inside(got, want, bound, what):
    assert got.shape == want.shape, what
    over = float(((got.double() - want).abs() - bound).max())
    assert over <= 0, (what, over)      # (a NaN is not)


def _draw(shape, dtype, seed):
    N, P, width, G = shape
    g = torch.Generator("cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # images of different levels and spreads, so that one's sums are not another's
    x = randn(N, P, width) * (0.5 + torch.rand((N, 1, 1), generator=g, device="cuda"))
    x += 0.5 * randn(N, 1, width)
    gamma, beta = 1 + 0.3 * randn(width), 0.3 * randn(width)
    dy = 0.1 * randn(N, P, width) + 0.01 * randn(N, 1, width)
    return x.to(DT[dtype]), gamma, beta, dy.to(DT[dtype])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_paths(r, shape, dtype):
    N, P, width, G = shape
    i = SHAPES.index(shape)
    kind = ["silu", "none", "gelu"][i % 3]
    say("path", shape, dtype, kind)
    x, gamma, beta, dy = _draw(shape, dtype, i)
    dt = DT[dtype]
    for act in (kind, "relu"):
        y = r.group_norm(x, G, gamma, beta, eps=1e-4, act=act)
        want, bound, mean, rstd = ref.norm(x, G, gamma, beta, 1e-4, act, dt)
        _inside(y, want, bound, "y " + act)
        yt, stats, kept = r.group_norm_train(x, G, gamma, beta, eps=1e-4, act=act)
        _inside(yt, want, bound, "y, kept " + act)
        del want, bound
    # (bounds as for the small shapes: a mean is rounded once, a variance is a
    # difference of 64-bit sums)
    scale = float(x.double().abs().max()) + 1
    _inside(stats[..., 0], mean, torch.full_like(mean, 4 * ref.U * scale), "mean")
    _inside(stats[..., 1], rstd, 8 * ref.U * rstd * (1 + (rstd * 1e-2) ** 2), "rstd")
    # some rows of every image, its first and last ones among them
    step = max(1, P // max(1, 24 // N))
    rows = sorted({n * P + p for n in range(N) for p in (0, *range(step, P, step), P - 1)})[:60]
    codes, exps, _ = ref.keep(x.reshape(-1, width)[rows].cpu())
    assert torch.equal(kept.codes[rows].cpu(), codes)
    assert torch.equal(kept.exps[rows].cpu(), exps)

    values = r.checkpoint_unpack(kept).reshape(N, P, width)
    for act in (kind, "relu"):
        for saved, at in ((kept, values), (x, x)):
            d = dy
            if act == "relu":     # either side of its jump gives the same
                m, q = (ref.wide(stats[..., e].double(), P, width) for e in (0, 1))
                z = (at.double() - m) * q * gamma.double() + beta.double()
                d = torch.where(z.abs() < 1e-4, torch.zeros_like(dy), dy)
                del m, q, z
            grads = r.group_norm_backward(d, saved, stats, gamma, beta, act=act)
            want, bound = ref.norm_back(d, at, stats, gamma, beta, act, dt)
            for name, got in zip(("dx", "dgamma", "dbeta"), grads):
                _inside(got, want[name], bound[name], (act, name, saved is x))
            del want, bound


# (fold; large with one, several and many images)
@pytest.mark.parametrize("shape", [(2, 3000, 24, 3), (1, 20000, 64, 8), (3, 20000, 64, 8),
                                   (70, 6000, 24, 8)], ids=str)
def test_outputs_left_out(r, shape):
    """dx, dgamma and dbeta may each be NULL; the others come out as with all."""
    N, P, width, G = shape
    x, gamma, beta, dy = _draw(shape, "bf16", 5)
    _, stats, kept = r.group_norm_train(x, G, gamma, beta, act="silu")
    want = r.group_norm_backward(dy, kept, stats, gamma, beta, act="silu")
    norm = mixrt.Norm(N, width, P, G, mixrt.MIXRT_BF16, mixrt.ACTS["silu"], 1e-5,
                      gamma.data_ptr(), beta.data_ptr())
    size = C.c_size_t()
    assert r._L.mixrt_norm_workspace(C.byref(norm), C.byref(size)) == 0
    ws = torch.empty((size.value,), dtype=torch.uint8, device="cuda")
    dense = lambda t: C.byref(mixrt.Map(t.data_ptr(), P * width, width))  # noqa: E731
    for given in range(8):
        say("given", shape, f"{given:03b}")
        outs = [torch.full_like(w, 7.0) for w in want]
        has = [bool(given & 1 << i) for i in range(3)]
        r._check(r._L.mixrt_norm_backward(
            r._h, C.byref(norm), dense(dy), None, C.byref(kept.descriptor(0)), stats.data_ptr(),
            dense(outs[0]) if has[0] else None, outs[1].data_ptr() if has[1] else None,
            outs[2].data_ptr() if has[2] else None, ws.data_ptr(), size.value))
        r.sync()
        for h, got, w in zip(has, outs, want):
            if not h:
                assert bool((got == 7.0).all())
            else:
                # without dx the images' sums may be added in another order, in
                # 64 bits: the rounding to 32 may turn out the other way
                off = (got.double() - w.double()).abs()
                assert bool((off <= 2 * ref.U * w.double().abs() + 1e-12).all())


def test_no_images_give_no_gradient(r):
    x = torch.empty((0, 5, 24), device="cuda")
    _, stats, kept = r.group_norm_train(x, 3)
    for saved in (x, kept):
        _, dgamma, dbeta = r.group_norm_backward(x, saved, stats)
        assert float(dgamma.abs().sum()) == 0.0 == float(dbeta.abs().sum())
