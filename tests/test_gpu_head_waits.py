"""What the head's products do when one of their bounded waits runs out: a flag, copies and products waited for, and out. A hook reports
waits as run out while the copies asked for so far, all in bounds, land as ever: nothing hangs and nothing is left in flight."""
import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx, dev
from _head_util import Case, class_masks, unpack
from test_gpu_head import check_step, loss_inputs, run_loss, run_step

pytestmark = pytest.mark.gpu


def status(ctx):
    return cz.load_library().cfgzip_poll_status(ctx.h, None, None, None, None)


def expire(ctx, on):
    cz.cfgzip_set_tuning(ctx.h, "test_expire_waits", int(on))


@pytest.mark.parametrize("V,H,B,density,head", [
    (20000, 512, 20, 0.9, "bf16"), (20000, 4096, 40, 0.9, "bf16"), (20000, 512, 20, 0.003, "bf16"), (5003, 320, 150, 0.3, "bf16"),
    (20000, 512, 20, 0.9, "mxfp4"), (20000, 4096, 64, 0.9, "mxfp4"), (20000, 4096, 20, 0.003, "mxfp4"), (400003, 32, 2, 0.9, "mxfp4")])
def test_step_whose_waits_run_out(V, H, B, density, head):
    K = 300
    case = Case(V, H, B, head, seed=V + B)
    p = synth.zipf_partition(V, K, 1.1, seed=3)
    cm = dev(class_masks(K, B, density, (9, V, B)))
    c, trep = torch.from_numpy(p.c).long().cuda(), torch.from_numpy(p.r[p.c]).cuda()
    mask = unpack(cm, K)[:, c]
    with Ctx([p]) as ctx:
        for _ in range(2):
            cz.cfgzip_poll_status(ctx.h)
            check_step(case, run_step(ctx, case, cm, B), mask, trep)
            expire(ctx, True)
            run_step(ctx, case, cm, B)  # results are undefined
            assert status(ctx) == cz.E_CUDA
            expire(ctx, False)
        check_step(case, run_step(ctx, case, cm, B), mask, trep)
        assert status(ctx) == cz.OK


@pytest.mark.parametrize("V,H,N", [(5003, 256, 300), (700, 1032, 130)])
def test_loss_and_gradient_whose_waits_run_out(V, H, N):
    case, _, packed, targets = loss_inputs(V, H, N, 0.5, 0)
    d_loss = torch.rand(N, generator=case.gen, device="cuda")
    d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
    d_weight = torch.zeros((V, H), device="cuda")
    ws = case.workspace(cz.HEAD_LOSS_BACKWARD)

    def both(ctx):
        loss, lse = run_loss(ctx, case, packed, targets)
        expired = status(ctx)
        for dtype in (cz.BF16, cz.F32):
            cz.cfgzip_head_loss_backward(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], targets, lse, d_loss, d_hidden, H,
                                         d_weight if dtype == cz.F32 else torch.zeros_like(d_weight, dtype=torch.bfloat16), dtype, H, 0,
                                         ws, ws.numel(), torch.cuda.current_stream())
        torch.cuda.synchronize()
        return (loss, lse, d_hidden.clone(), d_weight.clone()), expired, status(ctx)

    with Ctx([]) as ctx:
        status(ctx)
        first, *states = both(ctx)
        assert states == [cz.OK, cz.OK]
        expire(ctx, True)
        _, *states = both(ctx)
        assert states == [cz.E_CUDA, cz.E_CUDA]
        expire(ctx, False)
        again, *states = both(ctx)
        assert states == [cz.OK, cz.OK]
        assert all(torch.equal(a, b) for a, b in zip(first, again))
