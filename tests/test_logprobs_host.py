"""What the log probability calls on logits refuse (no GPU needed: arguments are looked at before a context)."""
import pytest

from paper_2605_29986_b200 import binding as cz
from test_head_host import GOOD, status


def forward(**change):
    a = dict(ctx=None, logits=GOOD, dtype=cz.BF16, row_stride_elems=100, N=3, V=100, vocab_mask=None, vocab_stride_words=0, tokens=GOOD,
             inv_temperature=1.0, n_top=5, logp=GOOD, entropy=GOOD, lse=GOOD, top_tokens=GOOD, top_logp=GOOD)
    a.update(change)
    return status(cz.cfgzip_token_logprobs, **a)


def backward(**change):
    a = dict(ctx=None, logits=GOOD, dtype=cz.BF16, row_stride_elems=100, N=3, V=100, vocab_mask=None, vocab_stride_words=0, tokens=GOOD,
             inv_temperature=1.0, lse=GOOD, entropy=GOOD, d_logp=GOOD, d_entropy=GOOD, d_logits=GOOD, d_stride_elems=100)
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
                   dict(d_stride_elems=99)):
        assert backward(**change) == cz.E_ARG, change
    assert backward(d_logits=GOOD + 1) == cz.E_ALIGN
    assert backward(d_logits=GOOD + 2, dtype=cz.F32) == cz.E_ALIGN
    assert backward(N=(1 << 30), V=1 << 21, row_stride_elems=1 << 21, d_stride_elems=1 << 21, ctx=None) == cz.E_ARG
