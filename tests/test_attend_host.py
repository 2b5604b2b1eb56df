"""The refiner's attention without a GPU: struct layouts, the refusals that need no
context, workspace sizes, the 64-bit statements, and that no kernel has a scratch
segment."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest

import attend_ref as ref
from paper_2312_11841_amd import mixrt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # an aligned address that is never read
torch = pytest.importorskip("torch")


def test_struct_layouts():
    structs = {"mixrt_normed_heads": mixrt.NormedHeads, "mixrt_attention": mixrt.Attention,
               "mixrt_relative_bias": mixrt.RelativeBiasDesc, "mixrt_sequence": mixrt.Sequence}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "mixrt.h"', "int main(void){"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        for fname, _ in py._fields_:
            lines.append(f'printf("{cname} {fname} %zu\\n", offsetof({cname}, {fname}));')
    consts = {"MIXRT_MAX_ATTENTION_DIM": mixrt.MAX_ATTENTION_DIM,
              "MIXRT_MAX_BIAS_AXES": mixrt.MAX_BIAS_AXES,
              "MIXRT_MAX_BIAS_BUCKETS": mixrt.MAX_BIAS_BUCKETS,
              "MIXRT_MAX_BIAS_REACH": mixrt.MAX_BIAS_REACH}
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


def _att(**kw):
    d = dict(batch=2, heads=8, kv_heads=2, head_dim=64, dtype=mixrt.MIXRT_BF16, scale=0.125,
             queries=100, keys=300, lens=FAKE)
    return mixrt.Attention(**{**d, **kw})


def _bias(**kw):
    d = dict(axes=2, count=8, reach=16, table=FAKE, buckets=FAKE, q_pos=FAKE, k_pos=FAKE,
             q_pos_stride=0, k_pos_stride=0)
    return mixrt.RelativeBiasDesc(**{**d, **kw})


def _size(att, bias=None, backward=0):
    size = C.c_size_t(7)
    rc = mixrt.lib().mixrt_attention_workspace(
        C.byref(att), None if bias is None else C.byref(bias), backward, C.byref(size))
    return rc, size.value


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), -1), (dict(batch=65536), -4), (dict(heads=0), -1), (dict(kv_heads=0), -1),
    (dict(kv_heads=3), -1), (dict(heads=65536, kv_heads=65536), -4), (dict(head_dim=0), -1),
    (dict(head_dim=129), -4), (dict(dtype=mixrt.MIXRT_U8), -4), (dict(dtype=7), -4),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1),
    (dict(scale=math.inf), -1), (dict(queries=-1), -1), (dict(keys=-1), -1),
    (dict(queries=2 ** 30), -4), (dict(keys=2 ** 30), -4), (dict(queries=2 ** 27), -4),
    (dict(lens=FAKE + 2), -1),
    (dict(batch=1, heads=1, kv_heads=1, queries=2 ** 29, keys=2 ** 29), -4)])
def test_attention_refusals(kw, status):
    rc, size = _size(_att(**kw))
    assert rc == status and size == 0
    assert mixrt.lib().mixrt_thread_error()


@pytest.mark.parametrize("kw,status", [
    (dict(axes=0), -4), (dict(axes=4), -4), (dict(count=0), -4), (dict(count=33), -4),
    (dict(reach=-1), -4), (dict(reach=128), -4)])
def test_bias_refusals(kw, status):
    rc, size = _size(_att(), _bias(**kw))
    assert rc == status and size == 0


def test_workspaces():
    """None where a call is one launch, and bounded beside the arrays."""
    for dt in (0, 1, 3):
        assert _size(_att(dtype=dt, queries=1, keys=100)) == (0, 0)
        for B, H, Hk, D, Tq, Tk in ((1, 1, 1, 1, 1, 1), (0, 1, 1, 8, 5, 5), (1, 32, 8, 128, 1, 14400),
                                    (2, 12, 3, 64, 3600, 7200), (1, 8, 8, 64, 3600, 2 ** 20),
                                    (1, 2, 2, 16, 0, 9), (1, 2, 2, 16, 9, 0),
                                    (64, 64, 64, 64, 4096, 64)):
            att = _att(batch=B, heads=H, kv_heads=Hk, head_dim=D, queries=Tq, keys=Tk, dtype=dt)
            rows, keys = B * H * Tq, B * Hk * Tk
            for back in (0, 1):
                rc, size = _size(att, _bias(axes=3, count=32), back)
                assert rc == 0 and size % 16 == 0
                parts = 16 + Tk // 2048 + H // Hk * Tq // 2048 if Tq > 16 else 512
                room = 8 * (D + 1) * max(rows, keys) * parts + (1 << 20)
                room += 4 * 96 * B * H * (Tq // 32 + 1) * parts if back else 0
                assert size <= room, (att.batch, att.queries, att.keys, back, size)


def _rot(**kw):
    d = dict(tokens=50, axes=3, pairs=8, layout=0, inverse=0, pos=FAKE, freq=FAKE, axis=FAKE)
    return mixrt.Rotary(**{**d, **kw})


def _normed(**kw):
    d = dict(heads=4, head_dim=32, dtype=1, weight=FAKE, x=FAKE, dy=FAKE, out=FAKE, dweight=FAKE)
    return mixrt.NormedHeads(**{**d, **kw})


@pytest.mark.parametrize("rot,heads,n,status", [
    (dict(tokens=-1), {}, 1, -1), (dict(tokens=2 ** 31), {}, 1, -4), (dict(axes=0), {}, 1, -4),
    (dict(axes=9), {}, 1, -4), (dict(layout=2), {}, 1, -4), (dict(pairs=-1), {}, 1, -1),
    (dict(pairs=17), {}, 1, -1), (dict(pairs=2 ** 30), {}, 1, -1), ({}, dict(heads=-1), 1, -4),
    ({}, dict(heads=65536), 1, -4), ({}, dict(head_dim=0), 1, -4),
    ({}, dict(head_dim=1025), 1, -4), ({}, dict(dtype=2), 1, -4), ({}, {}, 0, -1),
    ({}, {}, 3, -1)])
def test_rotary_norm_refusals(rot, heads, n, status):
    size = C.c_size_t(7)
    arr = (mixrt.NormedHeads * 3)(*[_normed(**heads)] * 3)
    assert mixrt.lib().mixrt_rotary_norm_workspace(C.byref(_rot(**rot)), arr, n,
                                                   C.byref(size)) == status
    assert size.value == 0


def test_rotary_norm_workspaces():
    for tokens, heads, dim, pairs in ((0, 4, 32, 8), (1, 32, 128, 64), (3600, 12, 80, 36),
                                      (10 ** 7, 16, 64, 32), (5, 1, 1024, 1), (9, 0, 8, 4)):
        size = C.c_size_t()
        arr = (mixrt.NormedHeads * 2)(*[_normed(heads=heads, head_dim=dim)] * 2)
        assert mixrt.lib().mixrt_rotary_norm_workspace(
            C.byref(_rot(tokens=tokens, pairs=pairs)), arr, 2, C.byref(size)) == 0
        assert size.value % 16 == 0 and size.value <= (1 << 24) + tokens * heads * dim // 16


def test_calls_without_a_context_or_with_null():
    L = mixrt.lib()
    att, b, s, ref_ = _att(), _bias(), mixrt.Sequence(FAKE, 1, 1, 1), C.byref
    four = [ref_(s)] * 4
    assert L.mixrt_attention_forward(None, ref_(att), None, *four, None, None, FAKE, 1) == -1
    assert b"ctx" in L.mixrt_thread_error()
    assert L.mixrt_attention_backward(None, ref_(att), ref_(b), *four, ref_(s), FAKE, FAKE,
                                      *four[:3], None, FAKE, 1) == -1
    assert L.mixrt_attention_workspace(None, None, 0, ref_(C.c_size_t())) == -1
    assert L.mixrt_attention_workspace(ref_(att), None, 0, None) == -1
    rot, h = _rot(), _normed()
    assert L.mixrt_rotary_norm_apply(None, ref_(rot), 1e-6, ref_(h), 1) == -1
    assert L.mixrt_rotary_norm_backward(None, ref_(rot), 1e-6, ref_(h), 1, FAKE, 1) == -1
    assert L.mixrt_rotary_norm_workspace(None, ref_(h), 1, ref_(C.c_size_t())) == -1
    assert L.mixrt_rotary_norm_workspace(ref_(rot), None, 1, ref_(C.c_size_t())) == -1
    assert L.mixrt_rotary_norm_workspace(ref_(rot), ref_(h), 1, None) == -1


# --- the statements themselves ----------------------------------------------------------

def test_attention_statement_against_autograd():
    g = torch.Generator().manual_seed(0)
    B, Tq, Tk, H, Hk, D = 2, 7, 11, 4, 2, 6
    q = torch.randn((B, Tq, H, D), generator=g).double().requires_grad_()
    k, v = (torch.randn((B, Tk, Hk, D), generator=g).double().requires_grad_() for _ in range(2))
    table = torch.randn((2, 5, H), generator=g).double().requires_grad_()
    buckets = torch.randint(0, 5, (2, 7), generator=g)
    qp, kp = torch.randint(-4, 4, (Tq, 2), generator=g), torch.randint(-4, 4, (Tk, 2), generator=g)
    dout = torch.randn((B, Tq, H, D), generator=g).double()
    lens = torch.tensor([11, 4])
    s = torch.einsum("bihd,bjhd->bhij", q, k.repeat_interleave(2, 2)) / math.sqrt(D)
    for a in range(2):
        d = (kp[None, :, a] - qp[:, None, a]).clamp(-3, 3) + 3
        s = s + table[a][buckets[a][d]].permute(2, 0, 1)
    s = s.masked_fill((torch.arange(Tk) >= lens[:, None])[:, None, None], -math.inf)
    o = torch.einsum("bhij,bjhd->bihd", torch.softmax(s, -1), v.repeat_interleave(2, 2))
    want = torch.autograd.grad((o * dout).sum(), (q, k, v, table))
    got = ref.attention(q.detach(), k.detach(), v.detach(), torch.float32, lens,
                        (table.detach(), buckets, qp, kp), dout=dout)
    assert torch.allclose(got["o"][0], o, atol=1e-12)
    for name, w in zip(("dq", "dk", "dv", "dtable"), want):
        assert torch.allclose(got[name][0], w, atol=1e-11), name
    for value, bound in got.values():
        assert bool((bound >= 0).all()) and float(bound.max()) < 1e-2


def test_rotary_norm_statement_against_autograd():
    g = torch.Generator().manual_seed(1)
    for layout in ("halves", "pairs"):
        x = torch.randn((9, 3, 14), generator=g).double().requires_grad_()
        w = torch.randn((14,), generator=g).double().requires_grad_()
        dy = torch.randn((9, 3, 14), generator=g).double()
        pos, freq = torch.randint(0, 9, (9, 2), generator=g).float(), torch.rand(5, generator=g)
        axis = (torch.arange(5) % 2).to(torch.uint8)
        y, _ = ref.rotary_norm(x, w, pos, freq, axis, layout, 0.1, torch.float32)
        want = torch.autograd.grad((y * dy).sum(), (x, w))
        got, _ = ref.rotary_norm_back(dy, x.detach(), w.detach(), pos, freq, axis, layout, 0.1,
                                      torch.float32)
        for a, b in zip(want, got):
            assert torch.allclose(a, b, atol=1e-11)


@pytest.mark.parametrize("source", ["mixrt_rotary_norm", "mixrt_attend_f32", "mixrt_attend_f16",
                                    "mixrt_attend_bf16"])
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
