"""The refiner's operators without a GPU: struct layouts, every refusal of the
C ABI (checked before any device work, on a context that no device backs),
the pure-host workspace sizes, and the 64-bit statements themselves."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

import refine_ref as ref
from paper_2312_11841_amd import mixrt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # an aligned address that is never read
torch = pytest.importorskip("torch")


def test_struct_layouts():
    structs = {"mixrt_norm": mixrt.Norm, "mixrt_map": mixrt.Map, "mixrt_kept": mixrt.Kept,
               "mixrt_rotary": mixrt.Rotary, "mixrt_heads": mixrt.Heads}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "mixrt.h"', "int main(void){"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        for fname, _ in py._fields_:
            lines.append(f'printf("{cname} {fname} %zu\\n", offsetof({cname}, {fname}));')
    consts = {"MIXRT_BF16": mixrt.MIXRT_BF16, "MIXRT_KEPT_GROUP": mixrt.KEPT_GROUP,
              **{f"MIXRT_ACT_{k.upper()}": v for k, v in mixrt.ACTS.items()},
              **{f"MIXRT_ROTARY_{k.upper()}": v for k, v in mixrt.ROTARY_LAYOUTS.items()}}
    for name in consts:
        lines.append(f'printf("const {name} %d\\n", (int){name});')
    lines.append("return 0;}")
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "l.c"), os.path.join(d, "l")
        open(src, "w").write("\n".join(lines))
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
        out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout
    got = {tuple(l.split()[:2]): int(l.split()[2]) for l in out.splitlines()}
    for cname, py in structs.items():
        assert got[(cname, "size")] == C.sizeof(py)
        for fname, _ in py._fields_:
            assert got[(cname, fname)] == getattr(py, fname).offset, (cname, fname)
    for name, v in consts.items():
        assert got[("const", name)] == v, name


def _norm(**kw):
    d = dict(images=2, channels=16, pixels=100, groups=4, dtype=mixrt.MIXRT_F16, act=2, eps=1e-5,
             gamma=FAKE, beta=FAKE)
    return mixrt.Norm(**{**d, **kw})


def _workspace(norm):
    size = C.c_size_t()
    return mixrt.lib().mixrt_norm_workspace(C.byref(norm), C.byref(size)), size.value


@pytest.mark.parametrize("kw,status", [
    (dict(images=-1), -1), (dict(images=65536), -4), (dict(channels=0), -1),
    (dict(channels=4100, groups=1), -4), (dict(pixels=-1), -1), (dict(pixels=2 ** 40), -4),
    (dict(groups=0), -1), (dict(groups=3), -1), (dict(dtype=mixrt.MIXRT_U8), -4),
    (dict(dtype=9), -4), (dict(act=4), -4), (dict(act=-1), -4), (dict(eps=-1e-9), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(gamma=FAKE + 2), -1),
    (dict(beta=FAKE + 1), -1)])
def test_norm_refusals(kw, status):
    rc, size = _workspace(_norm(**kw))
    assert rc == status and size == 0
    assert mixrt.lib().mixrt_thread_error()


def test_workspaces_are_bounded():
    """Scratch stays small beside the arrays, at the extremes too."""
    for N, P, Ch, G in ((1, 1, 1, 1), (0, 10, 8, 2), (8, 1920 * 1080, 16, 4), (1, 2 ** 27, 4096, 32),
                        (65535, 64, 64, 8), (1, 10 ** 6, 4096, 4096)):
        for dt in (0, 1, 3):
            rc, size = _workspace(_norm(images=N, pixels=P, channels=Ch, groups=G, dtype=dt))
            assert rc == 0 and size % 16 == 0
            assert size <= (1 << 16) + max(1 << 28, N * P * Ch // 2), (N, P, Ch, G, size)
    for rows, ch, outs in ((0, 1, 1), (1, 4096, 4096), (2 ** 30, 64, 64), (3600, 512, 1536)):
        size = C.c_size_t()
        k = mixrt.Kept(rows, ch, mixrt.MIXRT_F16, 0, 0)
        assert mixrt.lib().mixrt_linear_grad_workspace(C.byref(k), outs, C.byref(size)) == 0
        assert size.value <= 1 << 28


@pytest.mark.parametrize("kw,outs,status", [
    (dict(rows=-1), 8, -1), (dict(channels=0), 8, -1), (dict(channels=5000), 8, -4),
    (dict(rows=2 ** 40), 8, -4), (dict(dtype=mixrt.MIXRT_U8), 8, -4), ({}, 0, -1), ({}, 4097, -4)])
def test_linear_refusals(kw, outs, status):
    k = mixrt.Kept(**{**dict(rows=10, channels=16, dtype=1, codes=FAKE, exps=FAKE), **kw})
    size = C.c_size_t(7)
    assert mixrt.lib().mixrt_linear_grad_workspace(C.byref(k), outs, C.byref(size)) == status
    assert size.value == 0


def test_calls_without_a_context_or_with_null():
    L = mixrt.lib()
    n, m = _norm(), mixrt.Map(FAKE, 1600, 16)
    k = mixrt.Kept(10, 16, 1, FAKE, FAKE)
    rot, h = mixrt.Rotary(), mixrt.Heads()
    ref_ = C.byref
    assert L.mixrt_norm_forward(None, ref_(n), ref_(m), ref_(m), None, None, FAKE, 1 << 30) == -1
    assert b"ctx" in L.mixrt_thread_error()
    assert L.mixrt_norm_backward(None, ref_(n), ref_(m), ref_(m), None, FAKE, ref_(m), None, None,
                                 FAKE, 1 << 30) == -1
    assert L.mixrt_kept_pack(None, ref_(k), FAKE, 16) == -1
    assert L.mixrt_kept_unpack(None, ref_(k), 1, FAKE, 16) == -1
    assert L.mixrt_linear_grad(None, ref_(k), 8, FAKE, 8, FAKE, None, FAKE, 1 << 30) == -1
    assert L.mixrt_rotary_apply(None, ref_(rot), ref_(h), 1) == -1
    assert L.mixrt_norm_workspace(None, ref_(C.c_size_t())) == -1
    assert L.mixrt_norm_workspace(ref_(n), None) == -1
    assert L.mixrt_linear_grad_workspace(None, 8, ref_(C.c_size_t())) == -1


# --- the statements themselves ----------------------------------------------------------

def test_keep_examples():
    x = torch.zeros((1, 40))
    x[0, :3] = torch.tensor([1.0, -0.5, 127.0 / 64])
    x[0, 33] = 3.0
    codes, exps, values = ref.keep(x)
    assert exps.tolist() == [[127 - 6, 127 - 5]]        # 127/64 needs code 127 at 2^-6
    assert codes[0, :3].tolist() == [64, -32, 127] and codes[0, 33] == 96
    assert torch.equal(values, x.double())
    top = torch.full((1, 2), 65504.0, dtype=torch.float16)
    codes, exps, values = ref.keep(top)
    assert codes.tolist() == [[63, 63]] and exps.tolist() == [[137]]
    assert values[0, 0] == 64512.0


def test_norm_statement_against_autograd():
    g = torch.Generator().manual_seed(0)
    x = torch.randn((2, 30, 12), generator=g).double().requires_grad_()
    gamma = torch.randn((12,), generator=g).double().requires_grad_()
    beta = torch.randn((12,), generator=g).double().requires_grad_()
    dy = torch.randn((2, 30, 12), generator=g).double()
    for kind in ("none", "silu", "gelu"):
        y, _, mean, rstd = ref.norm(x, 3, gamma, beta, 1e-3, kind, torch.float32)
        lib = torch.nn.functional.group_norm(x.transpose(1, 2), 3, gamma, beta, 1e-3)
        lib = {"none": lambda t: t, "silu": torch.nn.functional.silu,
               "gelu": torch.nn.functional.gelu}[kind](lib).transpose(1, 2)
        assert torch.allclose(y, lib, atol=1e-12)
        grads = torch.autograd.grad((y * dy).sum(), (x, gamma, beta))
        got, _ = ref.norm_back(dy, x.detach(), torch.stack([mean, rstd], -1).detach(),
                               gamma.detach(), beta.detach(), kind, torch.float32)
        for a, b in zip(grads, (got["dx"], got["dgamma"], got["dbeta"])):
            assert torch.allclose(a, b, atol=1e-11)


@pytest.mark.parametrize("source", ["mixrt_norm", "mixrt_norm_back", "mixrt_kept",
                                    "mixrt_rotary"])
def test_kernels_use_no_scratch(source):
    """No register spills, and no scratch memory that the HIP runtime would
    allocate at a kernel's first launch (which a captured call could not)."""
    from paper_2312_11841_amd import build
    from test_abi_host import _kernel_private_segments
    obj = os.path.join(build.OBJ_DIR, source + ".o")
    if not os.path.exists(obj):
        pytest.skip("library objects not built")
    sizes = _kernel_private_segments(obj)
    assert sizes, source
    assert {k: v for k, v in sizes.items() if v} == {}
