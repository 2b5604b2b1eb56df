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
