"""What the layer calls refuse, and the workspaces they ask for (no GPU needed: arguments are looked at before a context)."""
import ctypes

import pytest

from paper_2605_29986_b200 import binding as cz
from test_head_host import BIG, GOOD, status


def layer(weight=GOOD, in_=64, out=40, activation=cz.ACT_SILU, bias=GOOD, bias_dtype=cz.F32, row_stride=None):
    return cz.cfgzip_layer(weight, in_, out, activation, bias, bias_dtype, row_stride)


def forward(l, **change):
    a = dict(ctx=None, layer=l, x=GOOD, x_stride=64, rows=3, residual=GOOD, residual_stride=40, y=GOOD, y_stride=40, slope=GOOD,
             slope_stride=40, workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_layer_forward, **a)


def backward(l, **change):
    a = dict(ctx=None, layer=l, x=GOOD, x_stride=64, rows=3, slope=GOOD, slope_stride=40, d_y=GOOD, d_y_stride=40, add=GOOD, add_stride=64,
             d_x=GOOD, d_x_stride=64, d_weight=GOOD, d_weight_dtype=cz.BF16, d_weight_stride=64, d_bias=GOOD, accumulate=0, workspace=GOOD,
             workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_layer_backward, **a)


@pytest.mark.parametrize("change,want", [
    (None, cz.E_ARG),
    (dict(weight=None), cz.E_ARG),
    (dict(in_=0), cz.E_ARG),
    (dict(out=-8), cz.E_ARG),
    (dict(in_=60, row_stride=64), cz.E_ARG),  # 8 to a vector
    (dict(out=36), cz.E_ARG),
    (dict(in_=65544), cz.E_RANGE),
    (dict(out=65544), cz.E_RANGE),
    (dict(activation=-1), cz.E_ARG),
    (dict(activation=5), cz.E_ARG),
    (dict(bias_dtype=cz.MXFP4), cz.E_ARG),
    (dict(row_stride=56), cz.E_ARG),
    (dict(row_stride=68), cz.E_ALIGN),
    (dict(weight=GOOD + 8), cz.E_ALIGN),
    (dict(bias=GOOD + 4), cz.E_ALIGN),
])
def test_both_refuse_a_layer_that_is_none(change, want):
    l = None if change is None else layer(**change)
    assert forward(l) == want and backward(l) == want


def test_arguments_of_the_layer():
    l = layer()
    assert forward(l) == cz.E_ARG  # nothing wrong but the context
    assert forward(layer(bias=None, bias_dtype=7), rows=0) == cz.E_ARG
    for change in (dict(rows=-1), dict(x=None), dict(y=None), dict(x_stride=56), dict(y_stride=32), dict(residual_stride=32),
                   dict(slope_stride=32)):
        assert forward(l, **change) == cz.E_ARG, change
    assert forward(l, rows=(1 << 24) + 1) == cz.E_RANGE
    for change in (dict(x=GOOD + 2), dict(x_stride=68), dict(y=GOOD + 8), dict(y_stride=44), dict(residual=GOOD + 2), dict(slope_stride=42)):
        assert forward(l, **change) == cz.E_ALIGN, change


def test_arguments_of_its_gradient():
    l = layer()
    assert backward(l) == cz.E_ARG  # the context
    for change in (dict(rows=-1), dict(x=None), dict(slope=None), dict(d_y=None), dict(d_x=None, d_weight=None, d_bias=None),
                   dict(d_weight_dtype=2), dict(d_weight_stride=56), dict(d_x_stride=56), dict(add_stride=56), dict(d_y_stride=32),
                   dict(slope_stride=32), dict(workspace=None)):
        assert backward(l, **change) == cz.E_ARG, change
    assert backward(l, rows=(1 << 24) + 1) == cz.E_RANGE
    for change in (dict(x=GOOD + 2), dict(slope=GOOD + 2), dict(d_y_stride=44), dict(add=GOOD + 4), dict(d_x=GOOD + 8), dict(d_weight=GOOD + 8),
                   dict(d_weight_dtype=cz.F32, d_weight_stride=66), dict(d_bias=GOOD + 2)):
        assert backward(l, **change) == cz.E_ALIGN, change
    assert backward(l, workspace_bytes=cz.cfgzip_layer_workspace(l, cz.LAYER_BACKWARD, 3) - 1) == cz.E_NOMEM


def test_workspaces_of_the_layer():
    for in_, out in ((8, 8), (64, 40), (512, 512), (1024, 2048), (8192, 4096)):
        for activation in (cz.ACT_NONE, cz.ACT_SILU):
            l = layer(in_=in_, out=out, activation=activation)
            for op in (cz.LAYER_FORWARD, cz.LAYER_BACKWARD):
                sizes = [cz.cfgzip_layer_workspace(l, op, n) for n in list(range(0, 3000)) + list(range(3000, 1 << 20, 50021))]
                assert all(a <= b for a, b in zip(sizes, sizes[1:])), (in_, out, op)
                assert status(cz.cfgzip_layer_workspace, l, op, -1) == cz.E_ARG
                assert status(cz.cfgzip_layer_workspace, l, op, (1 << 24) + 1) == cz.E_RANGE
    assert status(cz.cfgzip_layer_workspace, layer(), 2, 1) == cz.E_ARG
    assert status(cz.cfgzip_layer_workspace, layer(in_=60), 0, 1) == cz.E_ARG
    assert cz.load_library().cfgzip_layer_workspace(ctypes.byref(layer()), 0, 1, None) == cz.E_ARG
