"""How near the head calls come to the same formulas in 64 bits where little of a result is left over: differences of nearly equal
numbers, long sums, weights far apart in size. Bounds count roundings; what tensor memory cuts off is counted by the addition."""
import numpy as np
import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from _head_util import mx_values, pack

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


# ---- sums over many tokens ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("N", [2048, 16000, 65536, 200003])
def test_weight_gradient_summed_over_many_tokens(N):
    V, H = 64, 72
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    weight = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")  # all scores 0: p = 1 / V, a power of two
    x = torch.rand((N, H), generator=g, device="cuda").to(torch.bfloat16)
    d_loss = (torch.rand(N, generator=g, device="cuda") + 0.5).to(torch.bfloat16).float()
    targets = torch.zeros(N, dtype=torch.int32, device="cuda")
    lse = torch.full((N,), float(np.log(V)), device="cuda")
    d_weight = torch.full((V, H), 3.0, device="cuda")
    head = cz.cfgzip_head(weight, cz.BF16, V, H)
    with Ctx([]) as ctx:
        ws = workspace(head, cz.HEAD_LOSS_BACKWARD, N)
        for accumulate in (0, 1):
            cz.cfgzip_head_loss_backward(ctx.h, head, x, H, N, None, 0, targets, lse, d_loss, None, 0, d_weight, cz.F32, H, accumulate,
                                         ws, ws.numel(), torch.cuda.current_stream())
            torch.cuda.synchronize()
            # g = d / V, rounded to bf16, is d / V: an exponential 2^-21 off is far from the next bf16 number
            want = (1 + accumulate) * (d_loss.double() @ x.double()) / V
            # 128 additions to tensor memory of 16 products each at a time, each cut off by less than 2^-23 of a sum that grows evenly, so
            # half of that of the last on average; then a rounding for every such portion, and two at the end
            tol = 64 * 2.0 ** -23 + (N / 2048 + 2) * 2.0 ** -24
            off = ((d_weight.double() - want) / want)[1:]
            assert off.abs().max() <= tol, off.abs().max().item()
            # the row of the targets: g = d (1 / V - 1), 63 / 64 of d, which bf16 holds to 2^-8
            assert ((d_weight[0].double() / want + V - 1).abs() <= (V - 1) * (2.0 ** -8 + tol)).all()


# ---- scores of the decode step, of long rows and large batches ------------------------------------------------------------
def one_class(V):
    return synth.Partition(V=V, K=1, c=np.zeros(V, np.int32), r=np.zeros(1, np.int32), sizes=np.array([V]))


def positive_head(kind, V, H, gen):
    """Weights above 0, so that nothing cancels and what is cut off of a sum is cut off of the score."""
    if kind == "bf16":
        weight = torch.rand((V, H), generator=gen, device="cuda").to(torch.bfloat16)
        return cz.cfgzip_head(weight, cz.BF16, V, H), weight.double()
    packed = (torch.randint(0, 256, (V, H // 2), generator=gen, device="cuda", dtype=torch.int32) & 0x77).to(torch.uint8)
    scales = torch.randint(120, 125, (V, (H // 32 + 15) // 16 * 16), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
    head = cz.cfgzip_head(packed, cz.MXFP4, V, H, H // 2, scales, scales.shape[1])
    return head, mx_values(packed, scales, H).cuda()


LONG = [(kind, H, B, 20000 if H in (4096, 4128) else 300)  # (blocks with 128 tokens and more, and with a few)
        for kind in ("bf16", "mxfp4") for H in (1024, 4096, 4128, 8192, 16384, 65536) for B in (1, 16, 32, 48, 64, 128)
        if kind == "bf16" or B <= 64]
# 300 tokens to a block and more, and more than a block lists at a time
LONG += [("bf16", 8192, 16, 50000), ("bf16", 8192, 32, 50000), ("bf16", 8192, 70, 50000), ("bf16", 4096, 96, 50000),
         ("mxfp4", 8192, 40, 50000), ("mxfp4", 8192, 12, 50000), ("mxfp4", 1312, 33, 310000), ("bf16", 2056, 100, 310000)]


@pytest.mark.parametrize("kind,H,B,V", LONG)
def test_scores_of_long_rows(kind, H, B, V):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(H + B)
    head, weight = positive_head(kind, V, H, gen)
    hidden = torch.rand((B, H), generator=gen, device="cuda").to(torch.bfloat16)
    logits = torch.full((B, V), 99.0, device="cuda")
    argmax = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    with Ctx([one_class(V)]) as ctx:
        ws = workspace(head, cz.HEAD_STEP, B)
        class_mask = torch.ones((B, 1), dtype=torch.int32, device="cuda")
        cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, class_mask, 1, head, hidden, H, B, None, 0, logits, cz.F32, V, argmax, None, None,
                            None, ws, ws.numel(), torch.cuda.current_stream())
        torch.cuda.synchronize()
    z = hidden.double() @ weight.T
    off = (logits.double() - z) / z
    # A piece of 1024 elements (4-bit heads: 2048) is 64 additions to tensor memory of 16 products each, cut off by less than 2^-23 of a
    # sum that grows evenly, so half of that of the last on average. Then a rounding for every piece, and two for 4-bit heads' powers.
    cut = 1 if kind == "bf16" else 2
    tol = cut * 32 * 2.0 ** -23 + (H / 1024 + 3) * 2.0 ** -24
    assert off.abs().max() <= tol, (off.abs().max().item(), off.mean().item())
    assert off.mean().abs() <= cut * 16 * 2.0 ** -23, off.mean().item()  # half a unit on average is cut off, roundings are even


# ---- 4-bit weights and hidden states of very different sizes --------------------------------------------------------------
def four_bit_step(codes, scales, hidden):
    """Scores from a 4-bit head of these codes and scale bytes, and the same in 64 bits."""
    V, H = codes.shape
    packed = (codes[:, ::2] | (codes[:, 1::2] << 4)).to(torch.uint8)
    packed = torch.nn.functional.pad(packed, (0, -(H // 2) % 16)).contiguous()
    scales = torch.nn.functional.pad(scales.to(torch.uint8), (0, -(H // 32) % 16)).contiguous()
    head = cz.cfgzip_head(packed, cz.MXFP4, V, H, packed.shape[1], scales, scales.shape[1])
    B = hidden.shape[0]
    logits = torch.full((B, V), 99.0, device="cuda")
    argmax = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    with Ctx([one_class(V)]) as ctx:
        ws = workspace(head, cz.HEAD_STEP, B)
        class_mask = torch.ones((B, 1), dtype=torch.int32, device="cuda")
        cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, class_mask, 1, head, hidden, H, B, None, 0, logits, cz.F32, V, argmax, None, None,
                            None, ws, ws.numel(), torch.cuda.current_stream())
        torch.cuda.synchronize()
    weight = mx_values(packed, scales, H).cuda()
    return logits.double(), weight


@pytest.mark.parametrize("zeros", [False, True])  # the block with the largest scale holds weights, or only zeros
@pytest.mark.parametrize("H,V", [(128, 120), (1056, 400)])
def test_four_bit_blocks_far_below_the_largest_of_their_row(H, V, zeros):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(H)
    codes = torch.randint(0, 16, (V, H), generator=gen, device="cuda", dtype=torch.int32)
    below = torch.arange(V, device="cuda", dtype=torch.int32) % 40
    scales = torch.full((V, H // 32), 150, dtype=torch.int32, device="cuda")
    scales[:, 1:] -= below.unsqueeze(1)
    if zeros:
        codes[:, :32] = 0
    hidden = torch.empty((3, H), device="cuda").normal_(0.0, 2.0, generator=gen)
    hidden[:2, :32] = 0.0  # what is left of these rows is the small blocks' alone
    hidden = hidden.to(torch.bfloat16)
    got, weight = four_bit_step(codes, scales, hidden)
    x = hidden.double().abs()
    tol = H * 2.0 ** -24 * (x @ weight.abs().T)
    # scales more than 2^36 below the largest: a weight is off by up to 6 times 2^-38 of that
    tol += (below > 36) * 6 * 2.0 ** -38 * 2.0 ** (150 - 127) * x[:, 32:].sum(dim=1, keepdim=True)
    assert ((got - hidden.double() @ weight.T).abs() <= tol).all()


@pytest.mark.parametrize("hidden_power,scale", [(124, 5), (110, 1), (-100, 230), (-120, 247), (0, 127), (60, 60)])
def test_four_bit_scores_of_powers_far_apart(hidden_power, scale):
    V, H = 140, 1024
    gen = torch.Generator(device="cuda")
    gen.manual_seed(scale)
    codes = torch.randint(1, 8, (V, H), generator=gen, device="cuda", dtype=torch.int32)  # (all above 0: nothing cancels)
    scales = torch.full((V, H // 32), scale, dtype=torch.int32, device="cuda")
    hidden = ((1.0 + torch.rand((20, H), generator=gen, device="cuda")).double() * 2.0 ** hidden_power).to(torch.bfloat16)
    got, weight = four_bit_step(codes, scales, hidden)
    want = hidden.double() @ weight.T
    assert (want < 2.0 ** 127).all() and (want > 2.0 ** -120).all()  # finite, and above the numbers that lose bits
    assert ((got - want).abs() <= H * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("H", [1024, 4096, 16384, 65536])
@pytest.mark.parametrize("N", [40, 150])
def test_normalisers_of_long_rows(H, N):
    """The loss, and the step of more than 128 rows: sums in pieces of 512."""
    V = 300
    gen = torch.Generator(device="cuda")
    gen.manual_seed(H + N)
    head, weight = positive_head("bf16", V, H, gen)
    hidden = (torch.rand((N, H), generator=gen, device="cuda") * 2.0 ** -6).to(torch.bfloat16)
    targets = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    loss, lse, step_lse = (torch.full((N,), 99.0, device="cuda") for _ in range(3))
    argmax = torch.full((N,), -7, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream()
    with Ctx([one_class(V)]) as ctx:
        ws = workspace(head, cz.HEAD_LOSS, N)
        cz.cfgzip_head_loss(ctx.h, head, hidden, H, N, None, 0, targets, loss, lse, ws, ws.numel(), st)
        ws = workspace(head, cz.HEAD_STEP, N)
        class_mask = torch.ones((N, 1), dtype=torch.int32, device="cuda")
        cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, class_mask, 1, head, hidden, H, N, None, 0, None, cz.F32, V, argmax, None, None,
                            step_lse, ws, ws.numel(), st)
        torch.cuda.synchronize()
    z = hidden.double() @ weight.T
    want, top = torch.logsumexp(z, dim=1), z.amax(dim=1)
    of_target = z[torch.arange(N, device="cuda"), targets.long()]
    # A piece of 512 is 32 additions to tensor memory, cut off by less than 2^-23 of a sum that grows evenly, half of that of the last on
    # average; then a rounding for every piece. (Steps of up to 128 rows: twice as long.) To lse a sum of V exponentials of relative
    # accuracy 2^-20 and two roundings are added, to the loss the target's score as well.
    pieces = 1 if N > 128 else 2
    score = 16 * 2.0 ** -23 + H / 512 * 2.0 ** -24
    rest = 2.0 ** -20 + 2.0 ** -23 * top
    assert ((lse.double() - want).abs() <= score * top + rest).all()
    assert ((step_lse.double() - want).abs() <= pieces * score * top + rest).all()
    assert ((loss.double() - (want - of_target)).abs() <= score * (top + of_target) + rest).all()
