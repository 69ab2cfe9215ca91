"""Which workspaces a linear backward accepts, without a GPU: gs_linear_bwd's size check comes before that of the
workspace's alignment, so a call with an unaligned workspace ends at the one or the other and never launches."""
import ctypes as C
import os

import pytest

from paper_2609_05255_amd import build as gsbuild

FAKE = 1 << 20   # a non-NULL address; never read by the checks
F32, F16, BF16 = 0, 1, 2
NONE, RELU, GELU = 0, 1, 2
# (rows, inputs, outputs): few rows, the narrow form, tiles, split sums, widths that are not whole vectors
LAYERS = [(1, 4096, 4096), (30, 200, 150), (1000, 64, 48), (5000, 256, 256), (2763, 2922, 71), (5581, 1426, 66),
          (300, 1031, 77), (100_000, 200, 600), (4096, 4096, 4096)]


@pytest.fixture(scope="module")
def gs():
    if not os.path.exists(gsbuild.LIB):
        gsbuild.build()
    from paper_2609_05255_amd import gsraster
    return gsraster


def size(gs, type_, act, layer, dw_type):
    out = C.c_size_t(0)
    assert gs.lib().gs_linear_workspace_size(type_, act, *layer, dw_type, C.byref(out)) == gs.GS_OK
    return out.value


def accepts(gs, type_, act, layer, dw, dw_type, ws_bytes, odd):
    """Whether ws_bytes are enough for a backward; odd: operands off their vectors' alignment."""
    rows, n_in, n_out = layer
    at = FAKE + (4 if odd else 0)
    p = gs.Linear(type_, act, rows, n_in, n_out, at, FAKE, None, n_in, n_in)
    status = gs.lib().gs_linear_bwd(C.byref(p), at, n_out, at, n_out, FAKE, n_in, FAKE if dw else None, n_in, dw_type,
                                    FAKE, FAKE + 8, ws_bytes, None)
    assert status in (gs.GS_ERR_CAPACITY, gs.GS_ERR_INVALID_ARG)
    text = gs.lib().gs_last_error()
    assert (b"needed" if status == gs.GS_ERR_CAPACITY else b"aligned") in text
    return status == gs.GS_ERR_INVALID_ARG


@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("act", [NONE, RELU, GELU])
@pytest.mark.parametrize("type_", [F32, F16, BF16])
@pytest.mark.parametrize("odd", [False, True])
def test_without_a_weight_gradient(gs, type_, act, layer, odd):
    # a workspace sized for either type of dw also does for a call that leaves dw out, whatever dw_type that names
    for sized_for in {F32, type_}:
        have = size(gs, type_, act, layer, sized_for)
        for dw_type in {F32, type_}:
            assert accepts(gs, type_, act, layer, False, dw_type, have, odd), (sized_for, dw_type)
        assert accepts(gs, type_, act, layer, True, sized_for, have, odd)
