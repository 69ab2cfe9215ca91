"""The C ABI of codebooks and mixtures without a GPU: struct layouts, limits, sizes of workspaces, and what the calls refuse
before they launch anything."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_05255_amd import build as gsbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20   # a non-NULL address; never read by the checks
BIG = 1 << 40
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def gs():
    if not os.path.exists(gsbuild.LIB):
        gsbuild.build()
    from paper_2609_05255_amd import gsraster
    return gsraster


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no host C compiler")
def test_struct_layouts(gs, tmp_path):
    mirrors = {"gs_row_order": gs.RowOrderArrays, "gs_experts": gs.Experts}
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


def order(gs, count=12, groups=4, order=FAKE, sorted=FAKE, place=FAKE, offsets=FAKE):
    return gs.RowOrderArrays(count, groups, order, sorted, place, offsets)


ORDERS = [dict(count=-1), dict(count=1 << 31), dict(groups=0), dict(groups=(1 << 31) - 1), dict(order=None),
          dict(offsets=None), dict(order=FAKE + 2), dict(sorted=FAKE + 1), dict(place=FAKE + 3), dict(offsets=FAKE + 2)]


def sort_rows(gs, group_of=FAKE, ws=FAKE, ws_bytes=BIG, **kw):
    return gs.lib().gs_sort_rows(group_of, C.byref(order(gs, **kw)), ws, ws_bytes, None)


@pytest.mark.parametrize("bad", ORDERS + [dict(group_of=None), dict(group_of=FAKE + 1), dict(count=100_000, ws=None),
                                          dict(count=100_000, ws=FAKE + 16)])
def test_sort_rows_refuses(gs, bad):
    assert sort_rows(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad
    assert gs.lib().gs_last_error()


def test_sort_rows_refuses_small_workspaces(gs):
    out = C.c_size_t(0)
    assert gs.lib().gs_sort_rows(FAKE, None, None, 0, None) == gs.GS_ERR_INVALID_ARG
    for count, groups in ((100_000, 4), (9000, 70_000), (3_000_000, 65_536), (5, 20_000)):
        assert gs.lib().gs_sort_rows_workspace_size(count, groups, C.byref(out)) == gs.GS_OK and out.value > 0
        assert sort_rows(gs, count=count, groups=groups, ws_bytes=out.value - 1) == gs.GS_ERR_CAPACITY
    assert gs.lib().gs_sort_rows_workspace_size(8192, 16_384, C.byref(out)) == gs.GS_OK and out.value == 0
    for count, groups in ((-1, 4), (1 << 31, 4), (5, 0), (5, (1 << 31) - 1)):
        assert gs.lib().gs_sort_rows_workspace_size(count, groups, C.byref(out)) == gs.GS_ERR_INVALID_ARG
    assert gs.lib().gs_sort_rows_workspace_size(5, 4, None) == gs.GS_ERR_INVALID_ARG


def embedding_fwd(gs, type_=F32, rows=8, dim=16, entries=5, table=FAKE, ldt=16, index=FAKE, y=FAKE, ldy=16):
    return gs.lib().gs_embedding_fwd(type_, rows, dim, entries, table, ldt, index, 1.0, y, ldy, None)


@pytest.mark.parametrize("bad", [dict(type_=3), dict(rows=-1), dict(rows=1 << 31), dict(dim=0),
                                 dict(dim=(1 << 20) + 1, ldt=1 << 21, ldy=1 << 21), dict(entries=0),
                                 dict(entries=(1 << 31) - 1), dict(table=None), dict(index=None), dict(y=None),
                                 dict(ldt=15), dict(ldy=15), dict(index=FAKE + 2), dict(table=FAKE + 2),
                                 dict(type_=F16, y=FAKE + 1)])
def test_embedding_forward_refuses(gs, bad):
    assert embedding_fwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad


def embedding_bwd(gs, type_=F16, dim=16, dy=FAKE, lddy=16, dtable=FAKE, lddt=16, dtable_type=F32, ws=FAKE, ws_bytes=BIG,
                  **kw):
    return gs.lib().gs_embedding_bwd(type_, dim, dy, lddy, C.byref(order(gs, **kw)), 1.0, dtable, lddt, dtable_type, ws,
                                     ws_bytes, None)


@pytest.mark.parametrize("bad", ORDERS + [dict(sorted=None), dict(type_=9), dict(dim=0), dict(dy=None), dict(lddy=15),
                                          dict(dtable=None), dict(lddt=15), dict(dtable_type=BF16), dict(dtable=FAKE + 2),
                                          dict(ws=None), dict(ws=FAKE + 64)])
def test_embedding_backward_refuses(gs, bad):
    assert embedding_bwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad


def test_embedding_workspace(gs):
    out = C.c_size_t(0)
    for type_, rows, dim in ((F32, 1, 1), (F16, 3_000_000, 64), (BF16, 50_001, 333), (F32, (1 << 31) - 1, 8)):
        assert gs.lib().gs_embedding_workspace_size(type_, rows, dim, C.byref(out)) == gs.GS_OK
        assert 0 < out.value < 1 << 33
    assert gs.lib().gs_embedding_workspace_size(F16, 12, 16, C.byref(out)) == gs.GS_OK
    assert embedding_bwd(gs, ws_bytes=out.value - 1) == gs.GS_ERR_CAPACITY
    assert gs.lib().gs_embedding_workspace_size(F16, 0, 16, C.byref(out)) == gs.GS_OK and out.value == 0
    assert gs.lib().gs_embedding_workspace_size(5, 12, 16, C.byref(out)) == gs.GS_ERR_INVALID_ARG


def route(gs, backward, type_=F16, rows=8, experts=6, k=2, logits=FAKE, ld=6, expert=FAKE, weight=FAKE, dweight=FAKE,
          dlogits=FAKE, normalise=0):
    if backward:
        return gs.lib().gs_route_bwd(type_, rows, experts, k, dweight, logits, ld, expert, weight, normalise, dlogits, ld,
                                     None)
    return gs.lib().gs_route_fwd(type_, rows, experts, k, logits, ld, normalise, expert, weight, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("bad", [dict(type_=4), dict(rows=-1), dict(rows=1 << 30), dict(experts=0, ld=1),
                                 dict(experts=1025, ld=1025), dict(k=0), dict(k=7), dict(k=17, experts=100, ld=100),
                                 dict(logits=None), dict(ld=5), dict(expert=None), dict(weight=None),
                                 dict(expert=FAKE + 2), dict(weight=FAKE + 1), dict(logits=FAKE + 1)])
def test_route_refuses(gs, bad, backward):
    assert route(gs, backward, **bad) == gs.GS_ERR_INVALID_ARG, bad


@pytest.mark.parametrize("bad", [dict(dweight=None), dict(dweight=FAKE + 2), dict(dlogits=None), dict(dlogits=FAKE + 1)])
def test_route_backward_refuses(gs, bad):
    assert route(gs, True, **bad) == gs.GS_ERR_INVALID_ARG, bad


def move(gs, name, type_=F16, rows=6, dim=8, a=FAKE, lda=8, b=FAKE, ldb=8, c=FAKE, ldc=8, weight=FAKE, dweight=FAKE, **kw):
    o, lib = C.byref(order(gs, **kw)), gs.lib()
    if name == "dispatch_fwd":
        return lib.gs_dispatch_fwd(type_, rows, dim, a, lda, o, b, ldb, None)
    if name == "dispatch_bwd":
        return lib.gs_dispatch_bwd(type_, rows, dim, a, lda, o, c, ldc, b, ldb, None)
    if name == "combine_fwd":
        return lib.gs_combine_fwd(type_, rows, dim, a, lda, o, weight, c, ldc, b, ldb, None)
    return lib.gs_combine_bwd(type_, rows, dim, a, lda, c, ldc, o, weight, b, ldb, dweight, None)


MOVES = ["dispatch_fwd", "dispatch_bwd", "combine_fwd", "combine_bwd"]


@pytest.mark.parametrize("name", MOVES)
@pytest.mark.parametrize("bad", ORDERS + [dict(type_=7), dict(rows=-1), dict(rows=5), dict(rows=0), dict(rows=24), dict(dim=0),
                                          dict(a=None), dict(b=None), dict(lda=7), dict(ldb=7), dict(a=FAKE + 1),
                                          dict(count=17 * 6)])
def test_moves_refuse(gs, name, bad):
    assert move(gs, name, **bad) == gs.GS_ERR_INVALID_ARG, bad


@pytest.mark.parametrize("name", MOVES[1:])
@pytest.mark.parametrize("bad", [dict(place=None), dict(ldc=7), dict(c=FAKE + 1)])
def test_moves_back_refuse(gs, name, bad):
    assert move(gs, name, **bad) == gs.GS_ERR_INVALID_ARG, bad


@pytest.mark.parametrize("name", MOVES[2:])
@pytest.mark.parametrize("bad", [dict(weight=None), dict(weight=FAKE + 2)])
def test_combinations_refuse(gs, name, bad):
    assert move(gs, name, **bad) == gs.GS_ERR_INVALID_ARG, bad
    assert move(gs, "combine_bwd", dweight=None) == gs.GS_ERR_INVALID_ARG
    assert move(gs, "combine_bwd", c=None) == gs.GS_ERR_INVALID_ARG


def layer(gs, type_=F16, act=0, rows=40, n_in=16, n_out=24, x=FAKE, w=FAKE, bias=None, ldx=16, ldw=16, experts=4,
          w_stride=24 * 16, offsets=FAKE):
    return gs.Experts(gs.Linear(type_, act, rows, n_in, n_out, x, w, bias, ldx, ldw), experts, w_stride, offsets)


LAYERS = [dict(type_=5), dict(act=6), dict(act=-1), dict(rows=-1), dict(n_in=0), dict(n_out=0), dict(x=None), dict(w=None),
          dict(ldx=15), dict(ldw=15), dict(experts=0), dict(experts=1025), dict(w_stride=-1), dict(offsets=None),
          dict(offsets=FAKE + 2), dict(x=FAKE + 1), dict(w=FAKE + 1)]


def experts_fwd(gs, y=FAKE, ldy=24, z=None, ldz=24, ws=FAKE, ws_bytes=BIG, **kw):
    return gs.lib().gs_experts_fwd(C.byref(layer(gs, **kw)), y, ldy, z, ldz, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", LAYERS + [dict(y=None), dict(ldy=23), dict(z=FAKE, ldz=23), dict(y=FAKE + 1)])
def test_experts_forward_refuses(gs, bad):
    assert experts_fwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad
    assert gs.lib().gs_experts_fwd(None, FAKE, 24, None, 0, None, 0, None) == gs.GS_ERR_INVALID_ARG


def experts_bwd(gs, dy=FAKE, lddy=24, z=FAKE, ldz=24, dx=FAKE, lddx=16, dw=FAKE, lddw=16, dw_stride=24 * 16, dw_type=F32,
                db=FAKE, ws=FAKE, ws_bytes=BIG, **kw):
    return gs.lib().gs_experts_bwd(C.byref(layer(gs, **{"act": 3, **kw})), dy, lddy, z, ldz, dx, lddx, dw, lddw, dw_stride,
                                   dw_type, db, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", LAYERS + [dict(dy=None), dict(lddy=23), dict(z=None), dict(ldz=23), dict(lddx=15),
                                          dict(lddw=15), dict(dw_stride=24 * 16 - 1), dict(dw_type=BF16), dict(db=FAKE + 2),
                                          dict(dw=FAKE + 2), dict(ws=None), dict(ws=FAKE + 32)])
def test_experts_backward_refuses(gs, bad):
    assert experts_bwd(gs, **bad) == gs.GS_ERR_INVALID_ARG, bad


def test_experts_unsupported_sizes(gs):
    big = dict(rows=(1 << 31) - 1, n_in=1 << 20, n_out=1 << 20, ldx=1 << 20, ldw=1 << 20, w_stride=1 << 40)
    assert experts_fwd(gs, ldy=1 << 20, **big) == gs.GS_ERR_UNSUPPORTED
    many = dict(rows=100, experts=1024, n_in=1 << 18, n_out=1 << 18, ldx=1 << 18, ldw=1 << 18, w_stride=1 << 36)
    assert experts_fwd(gs, ldy=1 << 18, **many) == gs.GS_ERR_UNSUPPORTED


SIZES = [(40, 4, 16, 24), (1, 1, 1, 1), (33, 5, 200, 130), (1_000_000, 16, 64, 128), (16_384, 8, 2048, 2048),
         (5003, 7, 333, 215), (3000, 1000, 160, 130), (0, 3, 264, 144), (200_000, 64, 300, 900), (700, 3, 1, 700)]


@pytest.mark.parametrize("rows,experts,n_in,n_out", SIZES)
@pytest.mark.parametrize("type_", [F32, F16, BF16])
def test_experts_workspace_is_enough_for_every_call(gs, rows, experts, n_in, n_out, type_):
    """The size that is told does for whatever alignment the operands have, for either type of dw and for a backward
    without it: calls with one byte less than what they need are refused, so the need is found by bisection."""
    def need(call):
        low, high = 0, 1 << 42
        while low < high:
            mid = (low + high) // 2
            # (an unaligned workspace is refused after its size: nothing is launched)
            if call(mid) == gs.GS_ERR_CAPACITY:
                low = mid + 1
            else:
                high = mid
        return low

    out = C.c_size_t(0)
    for act in (0, 1, 3):
        told = {}
        for dw_type in (-1, type_, F32):
            assert gs.lib().gs_experts_workspace_size(type_, act, rows, experts, n_in, n_out, dw_type, C.byref(out)) == gs.GS_OK
            told[dw_type] = out.value
        assert told[-1] <= told[type_] <= told[F32]
        for pad in (0, 1):
            kw = dict(type_=type_, act=act, rows=rows, n_in=n_in, n_out=n_out, ldx=n_in + pad, ldw=n_in + pad,
                      experts=experts, w_stride=n_out * (n_in + pad), x=FAKE + 4 * pad, w=FAKE + 4 * pad)
            if rows and pad:   # (aligned weights may need none, and a call that needs none is not refused)
                assert need(lambda b: experts_fwd(gs, ldy=n_out, ws=FAKE + 16, ws_bytes=b, **kw) if told[-1] else 0) <= told[-1]
            for dw, dw_type in ((None, F32), (FAKE, type_), (FAKE, F32)):
                got = need(lambda b: experts_bwd(gs, lddy=n_out + pad, ldz=n_out, lddx=n_in, dw=dw, lddw=n_in,
                                                 dw_stride=n_out * n_in, dw_type=dw_type, ws=FAKE + 16, ws_bytes=b, **kw))
                assert got <= told[type_ if dw is None else dw_type], (act, pad, dw, dw_type)


def test_names_and_constants(gs):
    text = open(os.path.join(ROOT, "include", "gsraster.h")).read()
    assert "#define GS_MAX_EXPERTS 1024" in text and "#define GS_MAX_CHOICES 16" in text
    assert [gs.lib().gs_kernel_name(i).decode() for i in range(len(gs.KERNEL_NAMES))] == gs.KERNEL_NAMES
    assert "experts_bwd" in gs.KERNEL_NAMES and "sort_rows" in gs.KERNEL_NAMES


def test_binding_refuses_host_tensors(gs, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        gs.gs_embedding_fwd(x, torch.zeros(3, dtype=torch.int32), 1.0, torch.zeros(3, 8))
    with pytest.raises(ValueError):
        gs.gs_route_fwd(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(ValueError):
        gs.gs_experts_fwd(x, torch.zeros(3, dtype=torch.int32), torch.zeros(2, 5, 8), None, torch.zeros(4, 5))
