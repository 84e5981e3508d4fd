"""How near the head calls come to the same formulas in 64 bits where little of a result is left over: differences of nearly equal
numbers, long sums, weights far apart in size. Bounds count roundings; what tensor memory cuts off is counted by the addition."""
import numpy as np
import pytest
import torch

from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from _head_util import pack

pytestmark = pytest.mark.gpu
INF = float("inf")


def words(n):
    return (n + 31) // 32


def workspace(head, op, rows):
    return torch.full((cz.cfgzip_head_workspace(head, op, rows),), 0xFF, dtype=torch.uint8, device="cuda")


# ---- the gradient on targets that the model is sure of --------------------------------------------------------------------
@pytest.mark.parametrize("V,H,N", [(300, 1024, 40), (300, 4096, 33), (300, 16384, 300), (5003, 4096, 70), (14001, 4096, 20),
                                   (18901, 2056, 513)])
def test_gradient_of_sure_targets(V, H, N):
    g = torch.Generator(device="cuda")
    g.manual_seed(V + H + N)
    weight = torch.empty((V, H), device="cuda").normal_(0.0, H ** -0.5, generator=g).to(torch.bfloat16)
    targets = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    t, rows = targets.long(), torch.arange(N, device="cuda")
    # scores of the targets 1 to 10 above all others together; a coordinate of its own for every row, by which g is read from d_weight
    sure = np.log(V) + torch.linspace(1.0, 10.0, N, device="cuda").unsqueeze(1)
    x = sure * weight[t].float() + torch.empty((N, H), device="cuda").normal_(0.0, 0.3, generator=g)
    x[:, :N] = 2.0 * torch.eye(N, device="cuda")
    hidden = x.to(torch.bfloat16)
    mask = torch.rand((N, V), generator=g, device="cuda") < 0.5
    alone = rows % 4 == 0  # rows that allow the target and nothing else
    mask[alone] = False
    mask[rows, t] = True
    packed = pack(mask)
    d_loss = torch.rand(N, generator=g, device="cuda") + 0.5
    head = cz.cfgzip_head(weight, cz.BF16, V, H)
    loss, lse = torch.full((N,), 99.0, device="cuda"), torch.full((N,), 99.0, device="cuda")
    d_hidden = torch.full((N, H), 99.0, dtype=torch.bfloat16, device="cuda")
    d_weight = torch.full((V, H), 99.0, device="cuda")
    st = torch.cuda.current_stream()
    with Ctx([]) as ctx:
        ws = workspace(head, cz.HEAD_LOSS, N)
        cz.cfgzip_head_loss(ctx.h, head, hidden, H, N, packed, words(V), targets, loss, lse, ws, ws.numel(), st)
        ws = workspace(head, cz.HEAD_LOSS_BACKWARD, N)
        cz.cfgzip_head_loss_backward(ctx.h, head, hidden, H, N, packed, words(V), targets, lse, d_loss, d_hidden, H, d_weight, cz.F32, H,
                                     0, ws, ws.numel(), st)
        torch.cuda.synchronize()
    got = d_weight[:, :N].T.double() / 2.0  # (other rows have a zero there: products with 2, exact)
    assert (loss[alone] == 0).all()
    assert (got[alone] == 0).all() and (d_hidden[alone] == 0).all()
    z = (hidden.double() @ weight.double().T).masked_fill(~mask, -INF)
    want_lse = torch.logsumexp(z, dim=1, keepdim=True)
    d = d_loss.double().unsqueeze(1)
    p = torch.exp(z - want_lse)
    others = 1.0 - torch.exp(z[rows, t] - want_lse[:, 0])  # (at most 0.3)
    want = d * p
    want[rows, t] = d[:, 0] * torch.expm1(z[rows, t] - want_lse[:, 0])
    # a score, and with it lse, may be 2^-15 off (a millionth of some 20), which is p 2^-15 where nothing cancels
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -14)
    # The target: its score is the one in lse. What is left are lse's own roundings, half a step of the result and of at most 64
    # additions to a sum of about 1 (32 to a chain, the chains, the tiles), and the scores and exponentials of the others.
    tol[rows, t] = want[rows, t].abs() * 2.0 ** -8 + d[:, 0] * (want_lse[:, 0].abs() * 2.0 ** -24 + 64 * 2.0 ** -24 + others * 2.0 ** -13)
    off = (got - want).abs()
    assert (off <= tol)[~alone].all(), (off / tol.clamp(min=1e-30))[~alone].max().item()
