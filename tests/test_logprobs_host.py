"""What the log probability calls refuse (no GPU needed: arguments are looked at before a context)."""
import pytest

from paper_2605_29986_b200 import binding as cz
from test_head_host import BAD_HEADS, BIG, GOOD, head, status


def forward(**change):
    a = dict(ctx=None, logits=GOOD, dtype=cz.BF16, row_stride_elems=100, N=3, V=100, vocab_mask=None, vocab_stride_words=0, tokens=GOOD,
             inv_temperature=1.0, n_top=5, logp=GOOD, entropy=GOOD, lse=GOOD, top_tokens=GOOD, top_logp=GOOD)
    a.update(change)
    return status(cz.cfgzip_token_logprobs, **a)


def backward(**change):
    a = dict(ctx=None, logits=GOOD, dtype=cz.BF16, row_stride_elems=100, N=3, V=100, vocab_mask=None, vocab_stride_words=0, tokens=GOOD,
             inv_temperature=1.0, lse=GOOD, entropy=GOOD, d_logp=GOOD, d_entropy=GOOD, d_logits=2 * GOOD, d_stride_elems=100)
    a.update(change)
    return status(cz.cfgzip_token_logprobs_backward, **a)


BOTH = [
    (dict(), cz.E_ARG),  # nothing wrong but the context
    (dict(N=0), cz.E_ARG),
    (dict(N=-1), cz.E_ARG),
    (dict(V=0), cz.E_ARG),
    (dict(logits=None), cz.E_ARG),
    (dict(dtype=cz.MXFP4), cz.E_ARG),
    (dict(row_stride_elems=99), cz.E_ARG),
    (dict(vocab_mask=GOOD, vocab_stride_words=3), cz.E_ARG),
    (dict(inv_temperature=0.0), cz.E_ARG),
    (dict(inv_temperature=-1.0), cz.E_ARG),
    (dict(inv_temperature=1e-7), cz.E_ARG),
    (dict(inv_temperature=float("nan")), cz.E_ARG),
    (dict(inv_temperature=float("inf")), cz.E_ARG),
    (dict(inv_temperature=2e6), cz.E_ARG),
    (dict(V=(1 << 21) + 1, row_stride_elems=1 << 22, d_stride_elems=1 << 22), cz.E_RANGE),
    (dict(N=(1 << 30) + 1), cz.E_RANGE),
    (dict(logits=GOOD + 1), cz.E_ALIGN),
    (dict(logits=GOOD + 2, dtype=cz.F32), cz.E_ALIGN),
]


@pytest.mark.parametrize("change,want", BOTH)
def test_what_both_refuse(change, want):
    assert backward(**change) == want
    change.pop("d_stride_elems", None)
    assert forward(**change) == want


def test_arguments_of_the_log_probabilities():
    for change in (dict(n_top=-1), dict(n_top=33), dict(logp=None), dict(tokens=None), dict(top_tokens=None), dict(top_logp=None)):
        assert forward(**change) == cz.E_ARG, change


def test_arguments_of_their_gradient():
    for change in (dict(lse=None), dict(entropy=None), dict(d_logp=None, d_entropy=None), dict(tokens=None), dict(d_logits=None),
                   dict(d_logits=GOOD), dict(d_stride_elems=99)):
        assert backward(**change) == cz.E_ARG, change
    assert backward(d_logits=GOOD + 1) == cz.E_ALIGN
    assert backward(d_logits=GOOD + 2, dtype=cz.F32) == cz.E_ALIGN
    assert backward(N=(1 << 30), V=1 << 21, row_stride_elems=1 << 21, d_stride_elems=1 << 21, ctx=None) == cz.E_ARG


# ---- from hidden states -----------------------------------------------------------------------------------------------------
def head_forward(h, **change):
    a = dict(ctx=None, head=h, hidden=GOOD, hidden_stride=64, N=3, vocab_mask=None, vocab_stride_words=0, tokens=GOOD, logp=GOOD,
             entropy=None, lse=None, workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_head_logprobs, **a)


def head_backward(h, **change):
    a = dict(ctx=None, head=h, hidden=GOOD, hidden_stride=64, N=3, vocab_mask=None, vocab_stride_words=0, tokens=GOOD, lse=GOOD,
             entropy=GOOD, d_logp=GOOD, d_entropy=GOOD, d_hidden=GOOD, d_hidden_stride=64, d_weight=GOOD, d_weight_dtype=cz.BF16,
             d_weight_stride=64, accumulate=0, workspace=GOOD, workspace_bytes=BIG)
    a.update(change)
    return status(cz.cfgzip_head_logprobs_backward, **a)


@pytest.mark.parametrize("change,want", [b for b in BAD_HEADS if b[0] is None or b[0].get("dtype") != cz.MXFP4])
def test_both_refuse_a_head_that_is_none(change, want):
    h = None if change is None else head(**change)
    assert head_forward(h) == want and head_backward(h) == want


def test_arguments_from_hidden_states():
    h = head()
    assert head_forward(h) == cz.E_ARG and head_backward(h) == cz.E_ARG  # the context
    assert head_forward(head(dtype=cz.MXFP4)) == cz.E_ARG and head_backward(head(dtype=cz.MXFP4)) == cz.E_ARG
    for change in (dict(N=-1), dict(tokens=None), dict(hidden=None), dict(workspace=None), dict(hidden_stride=56),
                   dict(vocab_mask=GOOD, vocab_stride_words=3)):
        assert head_forward(h, **change) == cz.E_ARG and head_backward(h, **change) == cz.E_ARG, change
    assert head_forward(h, logp=None) == cz.E_ARG
    for change in (dict(lse=None), dict(entropy=None), dict(d_logp=None, d_entropy=None), dict(d_hidden=None, d_weight=None),
                   dict(d_weight_dtype=2), dict(d_hidden_stride=56), dict(d_weight_stride=56)):
        assert head_backward(h, **change) == cz.E_ARG, change
    assert head_forward(h, N=(1 << 30) + 1) == cz.E_RANGE and head_backward(h, N=(1 << 30) + 1) == cz.E_RANGE
    for change in (dict(hidden=GOOD + 2), dict(hidden_stride=68)):
        assert head_forward(h, **change) == cz.E_ALIGN and head_backward(h, **change) == cz.E_ALIGN, change
    for change in (dict(d_hidden=GOOD + 8), dict(d_weight=GOOD + 8), dict(d_weight_dtype=cz.F32, d_weight_stride=66)):
        assert head_backward(h, **change) == cz.E_ALIGN, change
    assert head_forward(h, workspace_bytes=cz.cfgzip_head_workspace(h, cz.HEAD_LOGPROBS, 3) - 1) == cz.E_NOMEM
    assert head_backward(h, workspace_bytes=cz.cfgzip_head_workspace(h, cz.HEAD_LOGPROBS_BACKWARD, 3) - 1) == cz.E_NOMEM


def test_workspaces_from_hidden_states():
    for V, H in ((1, 8), (300, 64), (18901, 256), (128256, 4096)):
        h = head(V=V, H=H)
        for op in (cz.HEAD_LOGPROBS, cz.HEAD_LOGPROBS_BACKWARD):
            sizes = [cz.cfgzip_head_workspace(h, op, n) for n in list(range(0, 3000)) + list(range(3000, 1 << 20, 50021))]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), (V, H, op)
            assert status(cz.cfgzip_head_workspace, h, op, -1) == cz.E_ARG
    assert status(cz.cfgzip_head_workspace, head(dtype=cz.MXFP4), cz.HEAD_LOGPROBS, 1) == cz.E_ARG
    assert status(cz.cfgzip_head_workspace, head(), 6, 1) == cz.E_ARG
