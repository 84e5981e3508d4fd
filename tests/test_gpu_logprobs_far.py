"""Log probabilities of rows whose logits are far from zero: fill values beside ordinary logits, rows of nothing else, either sign."""
import pytest
import torch

from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from test_gpu_logprobs import Rows, backward, check_gradient

pytestmark = pytest.mark.gpu
INF = float("inf")
FILLS = (-1e9, -1e10, -1e12, -1e20, -1e28)
TYPES = [torch.bfloat16, torch.float32]


def check(rows, out, n_top):
    """As Rows.check, with log probabilities held to what differences of logits allow: nothing of the size of the logits themselves."""
    rows.check(out, n_top)
    z = rows.scores()
    top = z.amax(dim=1, keepdim=True)
    some = (top > -INF).squeeze(1)
    x = (z - torch.where(top > -INF, top, 0.0)) * 1.0
    log_s = torch.logsumexp(x, dim=1)
    entropy = torch.special.entr(torch.softmax(x, dim=1)).sum(dim=1)
    of_sum = (rows.V / 512 + 48) * 2.0 ** -23 * (1 + (log_s - entropy).abs())
    t = rows.tokens.long()
    want = x.gather(1, t.clamp(0, rows.V - 1).unsqueeze(1)).squeeze(1) - log_s
    ok = some & (t >= 0) & (t < rows.V) & (want > -INF)
    assert ((out["logp"] - want).abs() <= of_sum + want.abs() * 2.0 ** -22)[ok].all()
    listed = (out["top_tokens"] >= 0) & some.unsqueeze(1)
    want = x.gather(1, out["top_tokens"].long().clamp(min=0)) - log_s.unsqueeze(1)
    assert ((out["top_logp"] - want).abs() <= of_sum.unsqueeze(1) + want.abs() * 2.0 ** -22)[listed].all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [1.0, 0.3, 0.15, 0.1])
@pytest.mark.parametrize("N,V", [(10, 9001), (10, 40000), (700, 20003), (1300, 9000)])
def test_fill_values_beside_ordinary_logits(N, V, t, dtype):
    # allowed tokens that the program in front has set to a large negative number, whole runs of them
    with Ctx([]) as ctx:
        for density in (None, 0.5):
            rows = Rows(N, V, dtype, density=density, t=t)
            for k, fill in enumerate(FILLS):
                rows.logits[k::5, 300 * k:300 * k + V // 2] = fill
                rows.tokens[k::10] = 300 * k + 7  # (some of the given tokens are among them)
            out = rows.run(ctx, 5)
            check(rows, out, 5)
            check_gradient(rows, backward(ctx, rows, out), out["lse"], out["entropy"], *rows.d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [1.0, 0.3, 0.15])
@pytest.mark.parametrize("N,V", [(12, 9001), (12, 40000), (700, 20003), (1300, 9000)])
def test_rows_of_nothing_but_far_logits(N, V, t, dtype):
    # equal ones, a few that are larger or smaller, and of either sign
    with Ctx([]) as ctx:
        for density in (None, 0.5):
            rows = Rows(N, V, dtype, density=density, t=t)
            for k, fill in enumerate(FILLS + tuple(-f for f in FILLS)):
                rows.logits[k::12] = fill
                if k % 2:
                    rows.logits[k::12, 5::1000] = fill * (1.5 if fill > 0 else 0.75)
            rows.logits[10::12] = -1e10
            rows.logits[10::12, V // 2:] = -1e28
            rows.logits[10::12, 17] = 1e10
            rows.logits[11::12] = 1e20
            rows.logits[11::12, ::3] = 1.25e20
            out = rows.run(ctx, 5)
            check(rows, out, 5)
            # (lse holds no more of such a row than its largest logit: its gradient is finite, and 0 where nothing comes back)
            assert backward(ctx, rows, out).isfinite().all()
            zero = torch.zeros(N, device="cuda")
            assert (backward(ctx, rows, out, zero, zero) == 0).all()


@pytest.mark.parametrize("offset", [1.16e7, -1.16e7, 3e7, -3e7, 2e8, -2e8])
def test_rows_about_where_references_change(offset):
    # f32 logits a few steps of theirs apart, on both sides of 2^24 powers of two
    for N, V in ((6, 8003), (6, 60000), (700, 5000)):
        with Ctx([]) as ctx:
            for density in (None, 0.4):
                rows = Rows(N, V, torch.float32, offset=offset, deviation=abs(offset) * 2.0 ** -9, density=density)
                rows.logits[1] = offset + torch.randint(-8, 9, (V,), generator=rows.gen, device="cuda") * max(1.0, abs(offset) * 2.0 ** -23)
                rows.logits[2] = (torch.linspace(-1, 1, V, device="cuda") * abs(offset) * 1.5).round()
                rows.logits[3] = rows.logits[2].flip(0)
                check(rows, rows.run(ctx, 10), 10)


def test_logits_of_thousands_at_the_lowest_temperature():
    with Ctx([]) as ctx:
        for dtype in TYPES:
            for density in (None, 0.5):
                rows = Rows(8, 9001, dtype, density=density, t=1e-6, deviation=3000.0)
                rows.logits[1] = 3000.0
                rows.logits[2, :5000] = -3000.0
                check(rows, rows.run(ctx, 5), 5)


def test_the_largest_numbers():
    with Ctx([]) as ctx:
        for dtype in TYPES:
            rows = Rows(4, 9001, dtype)
            rows.logits[0, ::2] = torch.finfo(dtype).max
            rows.logits[1, 77] = torch.finfo(dtype).max
            rows.logits[2] = torch.finfo(dtype).max
            rows.logits[2, ::2] = torch.finfo(dtype).min
            rows.logits[3] = torch.finfo(dtype).min
            rows.logits[3, 9000] = torch.finfo(dtype).max / 4
            out = rows.run(ctx, 5)
            assert out["lse"].isfinite().all() and out["entropy"].isfinite().all()
            z = rows.scores()
            z = torch.where(z < -1e29, -INF, z)
            lse = torch.logsumexp(z, dim=1)
            assert ((out["lse"] - lse).abs() <= lse.abs() * 2.0 ** -22).all()
            entropy = torch.special.entr(torch.softmax(z, dim=1)).sum(dim=1)
            assert ((out["entropy"] - entropy).abs() <= (9001 / 512 + 48) * 2.0 ** -23 * (8 + entropy)).all()
