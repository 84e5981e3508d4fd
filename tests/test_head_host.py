"""What the head calls refuse, and the workspaces they ask for (no GPU needed: arguments are looked at before a context)."""
import ctypes

import pytest

from paper_2605_29986_b200 import binding as cz

GOOD = 4096  # an address on 16 bytes; nothing here is ever read through it
BIG = 1 << 40


def head(weight=GOOD, dtype=cz.BF16, V=100, H=64, row_stride=None, scales=None, scale_stride=None, reserved=0):
    if dtype == cz.MXFP4 and scales is None:
        scales, scale_stride = GOOD, 16
    h = cz.cfgzip_head(weight, dtype, V, H, row_stride, scales, scale_stride)
    h.reserved = reserved
    return h


BAD_HEADS = [
    (None, cz.E_ARG),
    (dict(weight=None), cz.E_ARG),
    (dict(V=0), cz.E_ARG),
    (dict(V=-1), cz.E_ARG),
    (dict(H=0), cz.E_ARG),
    (dict(H=63), cz.E_ARG),                       # 8 to a vector
    (dict(H=65544, row_stride=65544), cz.E_RANGE),
    (dict(V=(1 << 30) + 1), cz.E_RANGE),
    (dict(dtype=cz.F32), cz.E_ARG),
    (dict(dtype=7), cz.E_ARG),
    (dict(reserved=1), cz.E_ARG),
    (dict(row_stride=56), cz.E_ARG),
    (dict(row_stride=68), cz.E_ALIGN),
    (dict(weight=GOOD + 8), cz.E_ALIGN),
    (dict(dtype=cz.MXFP4, H=72, row_stride=64), cz.E_ARG),   # 32 to a scale
    (dict(dtype=cz.MXFP4, row_stride=16), cz.E_ARG),
    (dict(dtype=cz.MXFP4, row_stride=40), cz.E_ALIGN),
    (dict(dtype=cz.MXFP4, H=1024, scales=GOOD, scale_stride=16), cz.E_ARG),
    (dict(dtype=cz.MXFP4, scales=GOOD, scale_stride=20), cz.E_ALIGN),
    (dict(dtype=cz.MXFP4, scales=GOOD + 4, scale_stride=16), cz.E_ALIGN),
]


def status(call, *args, **given):
    with pytest.raises(cz.CfgzipError) as e:
        call(*args, **given)
    return e.value.status


def step(h, **change):
    a = dict(ctx=None, part0=0, row_part=None, class_mask=GOOD, class_stride_words=1, head=h, hidden=GOOD, hidden_stride=64, B=3,
             vocab_mask=None, vocab_stride_words=0, logits=None, logits_dtype=0, logits_stride=0, argmax=GOOD, rep=None,
             logp_argmax=None, lse=None, workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_head_step, **a)


def loss(h, **change):
    a = dict(ctx=None, head=h, hidden=GOOD, hidden_stride=64, N=3, vocab_mask=None, vocab_stride_words=0, targets=GOOD, loss=GOOD,
             lse=None, workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_head_loss, **a)


def backward(h, **change):
    a = dict(ctx=None, head=h, hidden=GOOD, hidden_stride=64, N=3, vocab_mask=None, vocab_stride_words=0, targets=GOOD, lse=GOOD,
             d_loss=GOOD, d_hidden=GOOD, d_hidden_stride=64, d_weight=GOOD, d_weight_dtype=cz.BF16, d_weight_stride=64, accumulate=0,
             workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_head_loss_backward, **a)


@pytest.mark.parametrize("change,want", BAD_HEADS)
def test_every_call_refuses_a_head_that_is_none(change, want):
    h = None if change is None else head(**change)
    assert step(h) == want
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.BF16, 1 << 20, h) == want
    assert status(cz.cfgzip_head_dequantize, None, h, GOOD, 1 << 20) == want
    if change is None or change.get("dtype") != cz.MXFP4:  # (those take no 4-bit head at all)
        assert loss(h) == want and backward(h) == want


def test_arguments_of_the_step():
    h = head()
    assert step(h) == cz.E_ARG  # nothing wrong but the context
    for change in (dict(B=-1), dict(argmax=None), dict(class_mask=None), dict(class_stride_words=0), dict(hidden=None), dict(workspace=None),
                   dict(hidden_stride=56), dict(vocab_mask=GOOD, vocab_stride_words=3), dict(logits=GOOD, logits_stride=99),
                   dict(logits=GOOD, logits_stride=100, logits_dtype=2)):
        assert step(h, **change) == cz.E_ARG, change
    assert step(h, B=(1 << 30) + 1) == cz.E_RANGE
    for change in (dict(hidden=GOOD + 2), dict(hidden_stride=68)):
        assert step(h, **change) == cz.E_ALIGN, change
    for h in (head(), head(dtype=cz.MXFP4)):
        need = cz.cfgzip_head_workspace(h, cz.HEAD_STEP, 3)
        assert step(h, workspace_bytes=need - 1) == cz.E_NOMEM and step(h, workspace_bytes=need) == cz.E_ARG


def test_arguments_of_the_loss_and_its_gradient():
    h = head()
    assert loss(h) == cz.E_ARG and backward(h) == cz.E_ARG  # the context
    assert loss(head(dtype=cz.MXFP4)) == cz.E_ARG and backward(head(dtype=cz.MXFP4)) == cz.E_ARG
    for change in (dict(N=-1), dict(targets=None), dict(hidden=None), dict(workspace=None), dict(hidden_stride=56),
                   dict(vocab_mask=GOOD, vocab_stride_words=3)):
        assert loss(h, **change) == cz.E_ARG and backward(h, **change) == cz.E_ARG, change
    assert loss(h, loss=None) == cz.E_ARG
    assert loss(h, N=(1 << 30) + 1) == cz.E_RANGE and backward(h, N=(1 << 30) + 1) == cz.E_RANGE
    for change in (dict(lse=None), dict(d_loss=None), dict(d_hidden=None, d_weight=None), dict(d_hidden_stride=56), dict(d_weight_stride=56),
                   dict(d_weight_dtype=2)):
        assert backward(h, **change) == cz.E_ARG, change
    for change in (dict(hidden=GOOD + 2), dict(hidden_stride=68)):
        assert loss(h, **change) == cz.E_ALIGN and backward(h, **change) == cz.E_ALIGN, change
    for change in (dict(d_hidden=GOOD + 8), dict(d_hidden_stride=68), dict(d_weight=GOOD + 8), dict(d_weight_stride=68),
                   dict(d_weight_dtype=cz.F32, d_weight_stride=66)):
        assert backward(h, **change) == cz.E_ALIGN, change
    assert loss(h, workspace_bytes=cz.cfgzip_head_workspace(h, cz.HEAD_LOSS, 3) - 1) == cz.E_NOMEM
    assert backward(h, workspace_bytes=cz.cfgzip_head_workspace(h, cz.HEAD_LOSS_BACKWARD, 3) - 1) == cz.E_NOMEM


def test_arguments_of_quantising():
    h = head(dtype=cz.MXFP4)
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.BF16, 64, h) == cz.E_ARG  # the context
    assert status(cz.cfgzip_head_quantize, None, None, cz.BF16, 64, h) == cz.E_ARG
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.MXFP4, 64, h) == cz.E_ARG
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.BF16, 56, h) == cz.E_ARG
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.BF16, 64, head()) == cz.E_ARG
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.BF16, 68, h) == cz.E_ALIGN
    assert status(cz.cfgzip_head_quantize, None, GOOD, cz.F32, 66, h) == cz.E_ALIGN
    assert status(cz.cfgzip_head_dequantize, None, h, None, 64) == cz.E_ARG
    assert status(cz.cfgzip_head_dequantize, None, h, GOOD, 56) == cz.E_ARG
    assert status(cz.cfgzip_head_dequantize, None, head(), GOOD, 64) == cz.E_ARG
    assert status(cz.cfgzip_head_dequantize, None, h, GOOD + 8, 64) == cz.E_ALIGN


def test_workspaces():
    h = head(V=50021, H=1024)
    for op in (cz.HEAD_STEP, cz.HEAD_LOSS, cz.HEAD_LOSS_BACKWARD):
        sizes = [cz.cfgzip_head_workspace(h, op, n) for n in (0, 1, 32, 127, 128, 129, 1000, 8192, 100000)]
        assert sizes == sorted(sizes) and sizes[0] >= 0, op
        assert status(cz.cfgzip_head_workspace, h, op, -1) == cz.E_ARG
    assert status(cz.cfgzip_head_workspace, h, 3, 1) == cz.E_ARG
    assert status(cz.cfgzip_head_workspace, head(H=63), cz.HEAD_STEP, 1) == cz.E_ARG
    assert status(cz.cfgzip_head_workspace, head(dtype=cz.MXFP4), cz.HEAD_LOSS, 1) == cz.E_ARG
    assert cz.load_library().cfgzip_head_workspace(ctypes.byref(h), 0, 1, None) == cz.E_ARG
    # enough for `rows` rows is enough for fewer, however those are cut
    for V, H in ((1, 8), (300, 64), (18901, 256), (50021, 1024), (128256, 4096), (1 << 20, 65536)):
        for dtype in (cz.BF16, cz.MXFP4)[:1 if H % 32 else 2]:
            h = head(V=V, H=H, dtype=dtype)
            for op in (cz.HEAD_STEP, cz.HEAD_LOSS, cz.HEAD_LOSS_BACKWARD)[:1 if dtype == cz.MXFP4 else 3]:
                sizes = [cz.cfgzip_head_workspace(h, op, n) for n in list(range(1, 6000)) + list(range(6000, 1 << 20, 50021))]
                assert all(a <= b for a, b in zip(sizes, sizes[1:])), (V, H, dtype, op)
    assert status(cz.cfgzip_head_workspace, head(), cz.HEAD_STEP, (1 << 30) + 1) == cz.E_RANGE
    # the loss keeps no logits, and the gradient no more than a piece of them, however many tokens there are
    assert cz.cfgzip_head_workspace(head(V=128256, H=4096), cz.HEAD_LOSS, 8192) < 128256 * 8192 // 8
    big = cz.cfgzip_head_workspace(head(V=128256, H=4096), cz.HEAD_LOSS_BACKWARD, 65536)
    assert big < (256 << 20) + 16 * 65536 * 4096 * 4 + (1 << 20)
    # the memory is not part of the description: a head without any will do here
    assert cz.cfgzip_head_workspace(cz.cfgzip_head(None, cz.BF16, 100, 64), cz.HEAD_STEP, 4) > 0
