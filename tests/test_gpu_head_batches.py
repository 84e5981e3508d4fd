"""The head calls on batches of mixed partitions that allow little, on workspaces made for more rows, and gradients of several pieces."""
import copy

import numpy as np
import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx, dev
from _head_util import Case, class_masks, unpack
from test_gpu_head import check_step, close, gradient, loss_inputs, run_backward, run_loss, run_step

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("B", [1, 64, 128, 200])
@pytest.mark.parametrize("head", ["bf16", "mxfp4"])
def test_rows_of_several_partitions_that_allow_little(B, head):
    V, H = 30011, 320
    parts = [synth.zipf_partition(V, K, 1.1, seed=K) for K in (3000, 700, 1501)]
    case = Case(V, H, B, head, seed=B)
    which = np.random.RandomState(B).randint(0, 3, B)
    cm = dev(class_masks(3000, B, 0.001, (6, B)))
    mask = torch.zeros((B, V), dtype=torch.bool, device="cuda")
    reps = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    bits = unpack(cm, 3000)
    for b in range(B):
        p = parts[which[b]]
        mask[b] = bits[b][torch.from_numpy(p.c).long().cuda()]
        reps[b] = torch.from_numpy(p.r[p.c]).cuda()
    assert mask.any(dim=0).float().mean() < 0.75
    with Ctx(parts) as ctx:
        ids = dev(np.array(ctx.ids, dtype=np.int32)[which])
        for logits in (None, torch.bfloat16):
            check_step(case, run_step(ctx, case, cm, B, row_part=ids, logits=logits), mask, reps)


def test_fewer_rows_on_a_workspace_made_for_more():
    V, H, K, most = 20011, 320, 300, 300
    p = synth.zipf_partition(V, K, 1.1, seed=3)
    c, trep = torch.from_numpy(p.c).long().cuda(), torch.from_numpy(p.r[p.c]).cuda()
    for head in ("bf16", "mxfp4"):
        case = Case(V, H, most, head, seed=5)
        cm = dev(class_masks(K, most, 0.2, (4, 1)))
        mask = unpack(cm, K)[:, c]
        ws = case.workspace(cz.HEAD_STEP, most)
        with Ctx([p]) as ctx:
            for B in (300, 150, 129, 128, 65, 33, 17, 1, 257):  # (each finds what the one before has left)
                few = copy.copy(case)
                few.z, few.z_tol = case.z[:B], case.z_tol[:B]
                check_step(few, run_step(ctx, case, cm[:B], B, workspace=ws, logits=torch.float32 if B < 130 else None), mask[:B], trep)


def test_fewer_tokens_on_a_workspace_made_for_more():
    V, H, most = 9001, 136, 700
    case, mask, packed, targets = loss_inputs(V, H, most, 0.4, 0, seed=6)
    d_loss = torch.rand(most, generator=case.gen, device="cuda")
    g, g_tol = gradient(case, mask, targets, d_loss)
    want_lse = torch.logsumexp(case.z.masked_fill(~mask, -INF), dim=1)
    tol = case.lse_tol(mask)
    spaces = [case.workspace(op, most) for op in (cz.HEAD_LOSS, cz.HEAD_LOSS_BACKWARD)]
    st = torch.cuda.current_stream()
    with Ctx([]) as ctx:
        for N in (700, 257, 256, 100, 9, 640):
            loss, lse = torch.full((N,), 99.0, device="cuda"), torch.full((N,), 99.0, device="cuda")
            cz.cfgzip_head_loss(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], targets, loss, lse, spaces[0],
                                spaces[0].numel(), st)
            d_hidden = torch.full((N, H), 77.0, dtype=torch.bfloat16, device="cuda")
            d_weight = torch.full((V, H), 77.0, device="cuda")
            cz.cfgzip_head_loss_backward(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], targets, lse, d_loss, d_hidden, H,
                                         d_weight, cz.F32, H, 0, spaces[1], spaces[1].numel(), st)
            torch.cuda.synchronize()
            some = mask[:N].any(dim=1)
            assert ((lse.double() - want_lse[:N]).abs() <= tol[:N])[some].all() and (lse[~some] == -INF).all()
            assert close(d_hidden, g[:N] @ case.w64, g[:N], g_tol[:N], case.w64, V)
            assert close(d_weight, g[:N].T @ case.x64[:N], g[:N].T, g_tol[:N].T, case.x64[:N], N)


@pytest.mark.parametrize("V,H,N", [(27001, 328, 5003), (40009, 264, 4000)])
def test_gradient_in_several_pieces_and_cuts(V, H, N):
    case, mask, packed, targets = loss_inputs(V, H, N, 0.5, 0, seed=3)
    assert 2 * N * V > 256 << 20  # (more than one piece of the vocabulary)
    d_loss = torch.rand(N, generator=case.gen, device="cuda") / N
    g, g_tol = gradient(case, mask, targets, d_loss)
    with Ctx([]) as ctx:
        _, lse = run_loss(ctx, case, packed, targets)
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        d_weight = torch.full((V, H), 0.5, dtype=torch.float32, device="cuda")
        before = d_weight.clone()
        run_backward(ctx, case, packed, targets, lse, d_loss, d_hidden, d_weight, accumulate=1)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
        assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N, before)
