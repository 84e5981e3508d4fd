"""Nearly certain tokens in rows of every kind, and their gradient against the logits' own in 64 bits."""
import math

import pytest
import torch

from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from test_gpu_logprobs import CODE, Rows, backward

pytestmark = pytest.mark.gpu
# rows by clusters of blocks, and by one block of 8, 4 and 2 warps
SHAPES = [(6, 2000), (6, 50000), (300, 20003), (900, 20003), (1300, 9000)]


def sure(N, V, dtype, density):
    rows = Rows(N, V, dtype, density=density)
    rows.logits.copy_(torch.empty((N, V), device="cuda").normal_(generator=rows.gen))
    rows.logits[:, 77] = torch.tensor([16.0, 18.0, 20.0, 22.0, 24.0, 26.0], device="cuda").repeat((N + 5) // 6)[:N].to(dtype)
    rows.tokens[:] = 77
    if density is not None:
        rows.allowed[:, 77] = True
        rows.allow(rows.allowed)
    z = rows.scores()
    x = z - z[:, 77:78]
    x[:, 77] = -math.inf
    return rows, z, x, torch.exp(x).sum(dim=1)


def additions(N, V, dtype, density):
    """To a thread's sum of the certain one: half a step of a number up to sqrt(2) each. A row has two warps at least; a thread's pair of
    sums takes eight logits at a time, f32 rows under masks two."""
    return math.ceil(V / 512) * (4 if dtype == torch.float32 and density is not None else 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("density", [None, 0.5])
@pytest.mark.parametrize("N,V", SHAPES)
def test_nearly_certain_tokens(N, V, density, dtype):
    rows, z, x, rest = sure(N, V, dtype, density)
    with Ctx([]) as ctx:
        out = rows.run(ctx, 2)
    # the others' terms: t of 45 at most rounded once and a scale good to 2^-24 (45 * 2^-23 ln 2), an exponential good to 2^-22, additions:
    # below 2^-17 together; of the entropy's terms t counts once more
    of_one = additions(N, V, dtype, density) * 2.0 ** -24
    want = -torch.log1p(rest)
    assert ((out["logp"] - want).abs() <= 2.0 ** -17 * want.abs() + of_one).all()
    assert (out["top_tokens"][:, 0] == 77).all() and torch.equal(out["top_logp"][:, 0], out["logp"])
    want = torch.log1p(rest) - (torch.exp(x) * x).nan_to_num(0.0).sum(dim=1) / (1.0 + rest)
    assert ((out["entropy"] - want).abs() <= 2.0 ** -16 * want + 2 * of_one).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("density", [None, 0.5])
@pytest.mark.parametrize("N,V", SHAPES)
def test_gradient_of_nearly_certain_tokens(N, V, density, dtype):
    """Against the logits' own normaliser in 64 bits: 1 - p of 1e-2 to 1e-8 is off by what a normaliser in 32 bits is rounded by, half a step
    of a number of 16 to 26, and by what the sum in it is off by."""
    rows, z, x, rest = sure(N, V, dtype, density)
    with Ctx([]) as ctx:
        out = rows.run(ctx)
        one = torch.ones(N, device="cuda")
        got = backward(ctx, rows, out, d_logp=one).double()
    lse = torch.logsumexp(z, dim=1)
    p = torch.exp(z - lse.unsqueeze(1))
    off = (lse * 2.0 ** -24 * 1.01 + rest * 2.0 ** -17 + additions(N, V, dtype, density) * 2.0 ** -24).unsqueeze(1)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    want, tol = -p, p * (off + 2.0 ** -20 + (z - lse.unsqueeze(1)).abs().nan_to_num(0.0, 0.0, 0.0) * 2.0 ** -21) + p * half
    want[:, 77] = rest / (1.0 + rest)
    tol[:, 77] = (off + want[:, 77:78] * (half + 2.0 ** -20)).squeeze(1)
    if density is not None:
        want = torch.where(rows.allowed, want, 0.0)
    assert ((got - want).abs() <= tol + 1e-36).all()
    # what comes back of a row is what goes: the sum over its tokens is what lse and the results were rounded by
    assert (got.sum(dim=1).abs() <= tol.sum(dim=1)).all()
