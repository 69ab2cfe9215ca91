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


# with gelu in binary16 the product of the first plane alone is split further than that of both: 2763 x 2922 -> 71 and
# 5581 x 1426 -> 66 needed more for a binary16 dw than for an fp32 one
@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("act", [NONE, RELU, GELU])
@pytest.mark.parametrize("type_", [F16, BF16])
@pytest.mark.parametrize("odd", [False, True])
def test_the_size_for_an_fp32_weight_gradient_does_for_both_types(gs, type_, act, layer, odd):
    assert size(gs, type_, act, layer, F32) >= size(gs, type_, act, layer, type_)
    assert accepts(gs, type_, act, layer, True, type_, size(gs, type_, act, layer, F32), odd)


def test_general_layers_keep_dz_in_planes(gs):
    # beyond the narrow form's 128 columns the workspace holds dz, once more for each further plane of an fp32 dw
    plane = 1000 * 200 * 2
    for type_, planes in ((F16, 2), (BF16, 3)):
        for act, kept in ((GELU, planes), (RELU, 1)):
            assert size(gs, type_, act, (1000, 256, 200), F32) >= kept * plane + 256 * 200 * 2
        one, more = (size(gs, type_, GELU, (1000, 256, 200), t) for t in (type_, F32))
        assert one >= plane + 256 * 200 * 2 and more - one >= (planes - 1) * plane - 256 * 200 * 4
    # the narrow form keeps none: parts of dW and db alone, alike for either type of dw
    assert size(gs, F16, GELU, (1000, 64, 48), F32) == size(gs, F16, GELU, (1000, 64, 48), F16)


def test_weights_too_large_to_transpose_are_refused(gs):
    # 2^18 x 2^18: the launch that transposes W for dx would have 2^32 work items; without dx there is none
    n = 1 << 18
    p = gs.Linear(BF16, NONE, 1, n, n, FAKE, FAKE, None, n, n)

    def call(dx):
        return gs.lib().gs_linear_bwd(C.byref(p), FAKE, n, None, 0, dx, n, None, n, F32, FAKE, FAKE + 8, 1 << 50, None)

    assert call(FAKE) == gs.GS_ERR_UNSUPPORTED
    assert call(None) == gs.GS_ERR_INVALID_ARG and b"aligned" in gs.lib().gs_last_error()


@pytest.mark.parametrize("layer", LAYERS + [(1_100_000, 30, 63), (3_000_000, 64, 128)])
@pytest.mark.parametrize("type_", [F32, F16, BF16])
def test_the_forward_needs_the_same_for_any_activation(gs, type_, layer):
    assert len({size(gs, type_, act, layer, -1) for act in range(6)}) == 1
