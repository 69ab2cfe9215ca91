"""The row operators' C ABI without a GPU: struct layouts, sizes of workspaces, and what the calls refuse before they
launch anything."""
import ctypes as C
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_05255_amd import build as gsbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20   # a non-NULL address; never read by the checks
BIG = 1 << 40


@pytest.fixture(scope="module")
def gs():
    if not os.path.exists(gsbuild.LIB):
        gsbuild.build()
    from paper_2609_05255_amd import gsraster
    return gsraster


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no host C compiler")
def test_struct_layouts(gs, tmp_path):
    mirrors = {"gs_linear": gs.Linear, "gs_grad_tensor": gs.GradTensor}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "gsraster.h"', "int main(void) {"]
    for name, cls in mirrors.items():
        lines.append('printf("%s size %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s %s %%zu\\n", offsetof(%s, %s));' % (name, f, name, f) for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;", "}"]))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")],
                   check=True)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout
    for line in out.splitlines():
        name, field, value = line.split()
        cls = mirrors[name]
        assert int(value) == (C.sizeof(cls) if field == "size" else getattr(cls, field).offset), (name, field)


def test_type_and_activation_numbers(gs):
    text = open(os.path.join(ROOT, "include", "gsraster.h")).read()
    for name, value in (("GS_F32", 0), ("GS_F16", 1), ("GS_BF16", 2)):
        assert "%s = %d" % (name, value) in text
    for name, value in gs.ACTIVATIONS.items():
        assert "GS_ACT_%s = %d" % (name.upper(), value) in text


def norm_fwd(gs, type_=0, rows=8, dim=16, x=FAKE, ldx=16, eps=1e-5, y=FAKE, ldy=16):
    return gs.lib().gs_layer_norm_fwd(type_, rows, dim, x, ldx, None, None, eps, y, ldy, None, None, None)


def norm_bwd(gs, type_=0, rows=8, dim=16, dy=FAKE, x=FAKE, mean=FAKE, rstd=FAKE, add=None, dx=FAKE, ld=16, ws=FAKE,
             ws_bytes=BIG):
    return gs.lib().gs_layer_norm_bwd(type_, rows, dim, dy, ld, x, ld, None, mean, rstd, add, ld, dx, ld, None, None, ws,
                                      ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(type_=3), dict(type_=-1), dict(rows=-1), dict(rows=1 << 31), dict(dim=0),
                                 dict(dim=(1 << 20) + 1, ldx=1 << 21, ldy=1 << 21), dict(x=None), dict(y=None),
                                 dict(ldx=15), dict(ldy=15), dict(eps=-1.0), dict(eps=math.nan), dict(x=FAKE + 2),
                                 dict(type_=1, y=FAKE + 1), dict(ldx=1 << 31)])
def test_layer_norm_forward_refuses(gs, bad):
    assert norm_fwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad
    assert gs.lib().gs_last_error()


@pytest.mark.parametrize("bad", [dict(type_=7), dict(rows=-1), dict(dim=0), dict(dy=None), dict(x=None), dict(mean=None),
                                 dict(rstd=None), dict(dx=None), dict(ld=15), dict(add=FAKE + 1), dict(ws=None),
                                 dict(ws=FAKE + 16)])
def test_layer_norm_backward_refuses(gs, bad):
    assert norm_bwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad


def test_layer_norm_workspace(gs):
    out = C.c_size_t(0)
    assert gs.lib().gs_layer_norm_workspace_size(0, 1000, 64, C.byref(out)) == gs.GS_OK and out.value > 0
    assert norm_bwd(gs, rows=1000, dim=64, ld=64, ws_bytes=out.value - 1) == gs.GS_ERR_CAPACITY
    assert b"workspace" in gs.lib().gs_last_error()
    for args in ((5, 8, 8), (0, -1, 8), (0, 8, 0)):
        assert gs.lib().gs_layer_norm_workspace_size(*args, C.byref(out)) == gs.GS_ERR_INVALID_ARG
    assert gs.lib().gs_layer_norm_workspace_size(0, 8, 8, None) == gs.GS_ERR_INVALID_ARG


def layer(gs, type_=0, act=0, rows=100, n_in=16, n_out=8, x=FAKE, w=FAKE, bias=None, ldx=16, ldw=16):
    return gs.Linear(type_, act, rows, n_in, n_out, x, w, bias, ldx, ldw)


BAD_LAYERS = [dict(type_=3), dict(act=6), dict(act=-1), dict(rows=-1), dict(rows=1 << 31), dict(n_in=0), dict(n_out=0),
              dict(n_in=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(n_out=(1 << 20) + 1), dict(x=None), dict(w=None),
              dict(ldx=15), dict(ldw=15), dict(x=FAKE + 1), dict(w=FAKE + 2)]


@pytest.mark.parametrize("bad", BAD_LAYERS)
def test_linear_refuses_layers(gs, bad):
    L, p = gs.lib(), layer(gs, **bad)
    assert L.gs_linear_fwd(C.byref(p), None, 0, FAKE, 8, None, 0, FAKE, BIG, None) == gs.GS_ERR_INVALID_ARG
    assert L.gs_linear_bwd(C.byref(p), FAKE, 8, FAKE, 8, FAKE, 16, FAKE, 16, 0, FAKE, FAKE, BIG,
                           None) == gs.GS_ERR_INVALID_ARG


def test_linear_refuses_operands(gs):
    L, p = gs.lib(), layer(gs, act=2)
    ref = C.byref(p)
    bad = gs.GS_ERR_INVALID_ARG
    assert L.gs_linear_fwd(None, None, 0, FAKE, 8, None, 0, FAKE, BIG, None) == bad
    for y, ldy, r, ldr, z, ldz in ((None, 8, None, 0, None, 0), (FAKE, 7, None, 0, None, 0), (FAKE, 8, FAKE, 7, None, 0),
                                   (FAKE, 8, FAKE + 1, 8, None, 0), (FAKE, 8, None, 0, FAKE, 7)):
        assert L.gs_linear_fwd(ref, r, ldr, y, ldy, z, ldz, FAKE, BIG, None) == bad
    for dy, z, dx, ldx, dw, ldw, dt in ((None, FAKE, FAKE, 16, FAKE, 16, 0), (FAKE, None, FAKE, 16, FAKE, 16, 0),
                                        (FAKE, FAKE, FAKE, 15, FAKE, 16, 0), (FAKE, FAKE, FAKE, 16, FAKE, 15, 0),
                                        (FAKE, FAKE, FAKE, 16, FAKE, 16, 1), (FAKE, FAKE, FAKE, 16, FAKE, 16, 5),
                                        (FAKE, FAKE, FAKE, 16, FAKE + 2, 16, 0)):
        assert L.gs_linear_bwd(ref, dy, 8, z, 8, dx, ldx, dw, ldw, dt, None, FAKE, BIG, None) == bad
    assert L.gs_linear_bwd(ref, FAKE, 8, FAKE, 8, FAKE, 16, FAKE, 16, 0, None, FAKE, 16, None) == gs.GS_ERR_CAPACITY
    assert L.gs_linear_bwd(ref, FAKE, 8, FAKE, 8, FAKE, 16, FAKE, 16, 0, None, None, BIG, None) == bad
    assert L.gs_linear_bwd(ref, FAKE, 8, FAKE, 8, FAKE, 16, FAKE, 16, 0, None, FAKE + 8, BIG, None) == bad
    huge = layer(gs, rows=(1 << 31) - 1, n_out=1 << 20)
    assert L.gs_linear_fwd(C.byref(huge), None, 0, FAKE, 1 << 20, None, 0, FAKE, BIG, None) == gs.GS_ERR_UNSUPPORTED


def test_linear_workspace(gs):
    out, L = C.c_size_t(0), gs.lib()
    sizes = {}
    for dw_type in (-1, 0, 1):
        assert L.gs_linear_workspace_size(1, 2, 1000, 64, 48, dw_type, C.byref(out)) == gs.GS_OK
        sizes[dw_type] = out.value
    # the backward keeps dz, for an fp32 weight gradient in two planes
    assert sizes[1] >= 1000 * 48 * 2 and sizes[0] >= 2 * 1000 * 48 * 2 and sizes[-1] < sizes[1]
    for args in ((3, 0, 1, 1, 1, 0), (0, 9, 1, 1, 1, 0), (0, 0, -1, 1, 1, 0), (0, 0, 1, 0, 1, 0), (0, 0, 1, 1, 0, 0),
                 (0, 0, 1, 1, 1, 2), (1, 0, 1, 1, 1, -2)):
        assert L.gs_linear_workspace_size(*args, C.byref(out)) == gs.GS_ERR_INVALID_ARG, args
    assert L.gs_linear_workspace_size(0, 0, 1, 1, 1, 0, None) == gs.GS_ERR_INVALID_ARG


def test_grad_norm_refuses(gs):
    L, bad = gs.lib(), gs.GS_ERR_INVALID_ARG

    def call(tensors, max_norm=1.0, result=FAKE, ws=FAKE, ws_bytes=BIG, count=None, f="gs_grad_norm"):
        arr = (gs.GradTensor * max(1, len(tensors)))(*[gs.GradTensor(*t) for t in tensors])
        return getattr(L, f)(arr, len(tensors) if count is None else count, max_norm, result, ws, ws_bytes, None)

    good = (FAKE, None, 1 << 20, 0)
    for f in ("gs_grad_norm", "gs_grad_clip"):
        assert call([good], max_norm=-1.0, f=f) == bad
        assert call([good], max_norm=math.nan, f=f) == bad
        assert call([good], result=None, f=f) == bad
        assert call([good], result=FAKE + 2, f=f) == bad
        assert call([good], count=-1, f=f) == bad
        assert call([good], ws=None, f=f) == bad
        assert call([good], ws=FAKE + 8, f=f) == bad
        assert call([good], ws_bytes=8, f=f) == gs.GS_ERR_CAPACITY
        for t in ((None, None, 5, 0), (FAKE, None, -1, 0), (FAKE, None, 1 << 40, 0), (FAKE, None, 5, 3),
                  (FAKE + 2, None, 5, 0), (FAKE + 1, None, 5, 1), (FAKE, FAKE + 2, 5, 1)):
            assert call([good, t], f=f) == bad, t
        assert getattr(L, f)(None, 1, 1.0, FAKE, FAKE, BIG, None) == bad
    out = C.c_size_t(0)
    assert L.gs_grad_workspace_size(None, 0, C.byref(out)) == gs.GS_OK and out.value == 0
    assert L.gs_grad_workspace_size(None, 0, None) == bad and L.gs_grad_workspace_size(None, 2, C.byref(out)) == bad


def test_binding_refuses(gs):
    # the binding's own checks come before the library's: shapes, types, layout and the device
    x, w = torch.zeros(4, 6), torch.zeros(5, 6)
    with pytest.raises(ValueError, match="not on the GPU"):
        gs.gs_linear_fwd(x, w, None, torch.zeros(4, 5))
    with pytest.raises(ValueError, match="matrix"):
        gs.gs_layer_norm_fwd(torch.zeros(4), None, None, 1e-5, torch.zeros(4))
    with pytest.raises(ValueError, match="element type"):
        gs.gs_layer_norm_workspace_size(torch.zeros(2, 2, dtype=torch.float64))
    with pytest.raises(ValueError, match="activation"):
        gs.gs_linear_workspace_size(x, w, "swish")
    with pytest.raises(ValueError, match="contiguous"):
        gs.GradSet([torch.zeros(4, 4).t()[:2]])
    with pytest.raises(ValueError, match="entry"):
        gs.GradSet([], out=[None])
    with pytest.raises(ValueError, match="grad_scale"):
        gs.gs_adam_step([], 0.9, 1e-8, 1, grad_scale=torch.ones(1))


def test_binding_refuses_workspaces(gs):
    # a host array, which a kernel could not write
    for bad in (torch.zeros(512, dtype=torch.uint8), torch.zeros(64, 8, dtype=torch.uint8)[:, :4]):
        with pytest.raises(ValueError, match="workspace"):
            gs._space(bad)
    assert gs._space(None) == (None, 0)
