"""Log probabilities and entropies from hidden states and their gradient, against the formulas in 64 bits."""
import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx, dev
from _head_util import Case, class_masks, pack, unpack
from test_gpu_head import LOSSES, close, loss_inputs, run_loss, words

pytestmark = pytest.mark.gpu
INF = float("inf")


def run(ctx, case, packed, tokens, stream=None, workspace=None):
    N = case.rows
    logp, entropy, lse = (torch.full((N,), 99.0, device="cuda") for _ in range(3))
    ws = case.workspace(cz.HEAD_LOGPROBS) if workspace is None else workspace
    cz.cfgzip_head_logprobs(ctx.h, case.head, case.hidden, case.hidden.stride(0), N, packed, packed.shape[1] if packed is not None else 0,
                            tokens, logp, entropy, lse, ws, ws.numel(), stream or torch.cuda.current_stream())
    return logp, entropy, lse


def run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, d_hidden, d_weight, accumulate=0, workspace=None, stream=None):
    ws = case.workspace(cz.HEAD_LOGPROBS_BACKWARD) if workspace is None else workspace
    cz.cfgzip_head_logprobs_backward(ctx.h, case.head, case.hidden, case.hidden.stride(0), case.rows, packed,
                                     packed.shape[1] if packed is not None else 0, tokens, lse, entropy, d_logp, d_entropy, d_hidden,
                                     d_hidden.stride(0) if d_hidden is not None else 0, d_weight,
                                     cz.F32 if d_weight is not None and d_weight.dtype == torch.float32 else cz.BF16,
                                     d_weight.stride(0) if d_weight is not None else 0, accumulate, ws, ws.numel(),
                                     stream or torch.cuda.current_stream())


def statistics(case, mask):
    """lse and entropy in 64 bits and how far they may be off: by the errors of the scores (the entropy by p |log p + entropy| of them,
    2 entropy + 1 at the most), by sums with 32 additions to a chain, some 30 where chains and tiles meet and one more for every 64 half
    tiles, and by what log s and the mean difference are rounded by."""
    z = case.z.masked_fill(~mask, -INF)
    lse = torch.logsumexp(z, dim=1)
    entropy = torch.special.entr(torch.softmax(z, dim=1)).sum(dim=1).nan_to_num(nan=0.0)
    log_s = (lse - z.amax(dim=1)).nan_to_num(nan=0.0)
    z_tol = torch.where(mask, case.z_tol, 0.0).amax(dim=1)
    steps = (64 + case.V / 5000) * 2.0 ** -23
    return z, lse, entropy, z_tol * (2 * entropy + 1) + steps * (8 + log_s + 2 * (log_s - entropy).abs())


@pytest.mark.parametrize("V,H,N,density,pad", LOSSES)
def test_log_probabilities(V, H, N, density, pad):
    case, mask, packed, tokens = loss_inputs(V, H, N, density, pad, seed=7)
    with Ctx([]) as ctx:
        cz.cfgzip_poll_status(ctx.h)
        logp, entropy, lse = run(ctx, case, packed, tokens)
        assert cz.cfgzip_poll_status(ctx.h) == (0, int((tokens >= V).sum()), 0)
        loss, want_lse = run_loss(ctx, case, packed, tokens)
    # as the loss has them, up to the order of its sums
    finite = loss.isfinite()
    assert ((logp + loss).abs() <= want_lse.abs() * 2.0 ** -22 + loss.abs() * 2.0 ** -22 + 2.0 ** -18)[finite].all()
    assert (logp[~finite] == -INF).all()
    z, want, want_entropy, tol = statistics(case, mask)
    none = ~mask.any(dim=1)
    assert (lse[none] == -INF).all() and (entropy[none] == 0).all()
    assert ((lse - want).abs() <= case.lse_tol(mask))[~none].all()
    assert ((entropy - want_entropy).abs() <= tol)[~none].all()
    t, rows = tokens.long().clamp(0, V - 1), torch.arange(N, device="cuda")
    ignored, lost = tokens < 0, (tokens >= V) | ~mask[rows, t]
    assert (logp[ignored] == 0).all() and (logp[lost & ~ignored] == -INF).all()
    rest = ~ignored & ~lost
    tol = case.lse_tol(mask) + case.z_tol[rows, t] + (want.abs() + z[rows, t].abs()) * 2.0 ** -23
    assert ((logp - (z[rows, t] - want)).abs() <= tol)[rest].all()


def gradient(case, mask, tokens, d_logp, d_entropy):
    """g in 64 bits and how far the bf16 one may be off."""
    V, N = case.V, case.rows
    rows, t = torch.arange(N, device="cuda"), tokens.long().clamp(0, V - 1)
    has = (tokens >= 0) & (tokens < V) & mask[rows, t]
    z, lse, entropy, entropy_tol = statistics(case, mask)
    p = torch.exp(z - lse.unsqueeze(1)).nan_to_num(nan=0.0)
    x = torch.where(p > 0, z - lse.unsqueeze(1), 0.0)
    d = torch.where(has, d_logp.double(), 0.0).unsqueeze(1) if d_logp is not None else torch.zeros_like(p[:, :1])
    e = d_entropy.double().unsqueeze(1) if d_entropy is not None else torch.zeros_like(d)
    one = torch.zeros_like(p)
    one[rows, t] = 1.0
    of_entropy = e * p * (x + entropy.unsqueeze(1))
    g = torch.where(mask, d * (one - p) - of_entropy, 0.0)
    off = case.z_tol + case.lse_tol(mask).nan_to_num(0.0, 0.0).unsqueeze(1) + 2.0 ** -20
    size = p * (d.abs() + e.abs() * (x.abs() + entropy.unsqueeze(1) + 1))
    g_tol = g.abs() * 2.0 ** -8 + size * off * 1.1 + e.abs() * p * entropy_tol.unsqueeze(1) + d.abs() * one * 2.0 ** -23
    return g, torch.where(mask, g_tol, 0.0)


@pytest.mark.parametrize("V,H,N,density,pad", LOSSES)
def test_gradient(V, H, N, density, pad):
    case, mask, packed, tokens = loss_inputs(V, H, N, density, pad, seed=8)
    d_logp = torch.randn(N, generator=case.gen, device="cuda")
    d_entropy = torch.randn(N, generator=case.gen, device="cuda")
    if N > 9:
        d_logp[8], d_entropy[9] = 0.0, 0.0
    with Ctx([]) as ctx:
        _, entropy, lse = run(ctx, case, packed, tokens)
        for of_logp, of_entropy, dtype, accumulate in ((d_logp, d_entropy, torch.bfloat16, 0), (d_logp, d_entropy, torch.float32, 1),
                                                       (d_logp, None, torch.float32, 0), (None, d_entropy, torch.float32, 0)):
            g, g_tol = gradient(case, mask, tokens, of_logp, of_entropy)
            d_hidden = torch.full((N, H + 8), 77.0, dtype=torch.bfloat16, device="cuda")
            d_weight = torch.full((V, H + 8), 77.0, dtype=dtype, device="cuda")
            before = None
            if accumulate:
                before = torch.randn((V, H), generator=case.gen, device="cuda").to(dtype)
                d_weight[:, :H] = before
            run_gradient(ctx, case, packed, tokens if of_logp is not None else None, lse, entropy if of_entropy is not None else None, of_logp,
                         of_entropy, d_hidden[:, :H], d_weight[:, :H], accumulate)
            assert (d_hidden[:, H:] == 77.0).all() and (d_weight[:, H:] == 77.0).all()
            assert close(d_hidden[:, :H], g @ case.w64, g, g_tol, case.w64, V)
            assert close(d_weight[:, :H], g.T @ case.x64, g.T, g_tol.T, case.x64, N, before)
        # either one alone is the same
        g, g_tol = gradient(case, mask, tokens, d_logp, d_entropy)
        alone = torch.full((N, H), 77.0, dtype=torch.bfloat16, device="cuda"), torch.zeros((V, H), device="cuda")
        both = torch.zeros_like(alone[0]), torch.zeros_like(alone[1])
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, alone[0], None)
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, None, alone[1])
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, *both)
        assert torch.equal(alone[0], both[0]) and torch.equal(alone[1], both[1])


@pytest.mark.parametrize("V,H,N", [(300, 64, 1), (5003, 256, 9), (2000, 1032, 300), (40, 64, 1000), (27001, 64, 5003)])
def test_what_the_targets_were_rounded_by_is_not_lost(V, H, N):
    """Weights and hidden states that tell the terms of a gradient apart: what a target's g loses in bf16 comes back in 32 bits (several rows
    may have the same target)."""
    case, mask, packed, tokens = loss_inputs(V, H, N, None, 0, seed=11)
    d_logp = torch.rand(N, generator=case.gen, device="cuda") + 0.5
    with Ctx([]) as ctx:
        _, _, lse = run(ctx, case, packed, tokens)
        d_weight = torch.zeros((V, H), device="cuda")
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        run_gradient(ctx, case, packed, tokens, lse, None, d_logp, None, d_hidden, d_weight)
        g, g_tol = gradient(case, mask, tokens, d_logp, None)
        rows, t = torch.arange(N, device="cuda"), tokens.long().clamp(0, V - 1)
        has = (tokens >= 0) & (tokens < V)
        # (the tolerance of a target's g, without its rounding to bf16: twice a rounding in 32 bits)
        at = rows[has], t[has]
        g_tol[at] -= g[at].abs() * (2.0 ** -8 - 2.0 ** -23)
        assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)


def test_gradient_in_several_pieces_of_the_vocabulary():
    V, H, N = 27001, 64, 5003
    case, mask, packed, tokens = loss_inputs(V, H, N, 0.5, 0, seed=9)
    d_logp, d_entropy = (torch.randn(N, generator=case.gen, device="cuda") / N for _ in range(2))
    g, g_tol = gradient(case, mask, tokens, d_logp, d_entropy)
    with Ctx([]) as ctx:
        _, entropy, lse = run(ctx, case, packed, tokens)
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        d_weight = torch.zeros((V, H), device="cuda")
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, d_hidden, d_weight)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
        assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N)


def test_gradient_is_that_of_the_results():
    """Against differences in 64 bits: a step along the gradient changes the sum by its squared length, to first order."""
    V, H, N = 600, 64, 40
    case, mask, packed, tokens = loss_inputs(V, H, N, 0.5, 0, seed=5)
    tokens[tokens >= V] = -1
    mask[torch.arange(N), tokens.long().clamp(min=0)] = True
    packed = pack(mask)
    a, b = torch.rand(N, generator=case.gen, device="cuda") + 0.5, torch.rand(N, generator=case.gen, device="cuda") + 0.5
    with Ctx([]) as ctx:
        _, entropy, lse = run(ctx, case, packed, tokens)
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        d_weight = torch.zeros((V, H), device="cuda")
        run_gradient(ctx, case, packed, tokens, lse, entropy, a, b, d_hidden, d_weight)

    def value(x, w):
        z = (x @ w.T).masked_fill(~mask, -INF)
        logp = z - torch.logsumexp(z, dim=1, keepdim=True)
        t = tokens.long()
        of = torch.where(t >= 0, logp[torch.arange(N), t.clamp(min=0)], 0.0)
        return (a * of + b * torch.special.entr(torch.exp(logp)).sum(dim=1)).sum()

    eps = 1e-5  # (second order: eps times the curvature, below 1e-3 of the slope)
    for x, w in ((d_hidden.double(), 0.0), (0.0, d_weight.double())):
        slope = ((value(case.x64 + eps * x, case.w64 + eps * w) - value(case.x64 - eps * x, case.w64 - eps * w)) / (2 * eps)).item()
        length = ((x if torch.is_tensor(x) else w) ** 2).sum().item()
        # every element of the gradient is within 2^-8 (g) + 2^-8 (result) of its size: the products agree to 2 % at the worst
        assert abs(slope - length) <= 0.02 * length


def test_the_two_ways_to_log_probabilities_agree():
    """As they are used: decode steps from hidden states under the grammar leave masked logits, which are scored; the same hidden states are
    scored without logits, and an update is made of either gradient."""
    V, H, B, K = 5003, 256, 24, 60
    case = Case(V, H, B, seed=31)
    p = synth.zipf_partition(V, K, 1.1, seed=22)
    cm = dev(class_masks(K, B, 0.4, (9, 3)))
    st = torch.cuda.current_stream()
    with Ctx([p]) as ctx:
        vm = torch.zeros((B, words(V)), dtype=torch.int32, device="cuda")
        logits = torch.zeros((B, V), device="cuda")
        token = torch.zeros(B, dtype=torch.int32, device="cuda")
        ws = case.workspace(cz.HEAD_STEP)
        step_logp, step_lse = torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda")
        cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, cm, cm.shape[1], case.head, case.hidden, H, B, vm, words(V), logits, cz.F32, V, token,
                            None, step_logp, step_lse, ws, ws.numel(), st)
        logp, entropy, lse, of_top = (torch.zeros(B, device="cuda") for _ in range(4))
        top = torch.zeros(B, dtype=torch.int32, device="cuda")
        cz.cfgzip_token_logprobs(ctx.h, logits, cz.F32, V, B, V, None, 0, token, 1.0, 1, logp, entropy, lse, top, of_top, st)
        assert torch.equal(top, token) and torch.equal(of_top, logp)
        of_step = case.z_tol.amax() + 2.0 ** -17  # (scores of two kernels, sums in another order)
        assert (logp - step_logp).abs().max() <= of_step and (lse - step_lse).abs().max() <= of_step
        logp2, entropy2, lse2 = run(ctx, case, vm, token)
        assert (logp2 - logp).abs().max() <= of_step and (lse2 - lse).abs().max() <= of_step
        _, _, want_entropy, tol = statistics(case, unpack(vm, V))
        assert ((entropy - want_entropy).abs() <= tol).all() and ((entropy2 - want_entropy).abs() <= tol).all()
        d_logp, d_entropy = torch.rand(B, device="cuda") - 0.5, torch.full((B,), 0.1, device="cuda")
        g, g_tol = gradient(case, unpack(vm, V), token, d_logp, d_entropy)
        d_hidden = torch.zeros((B, H), dtype=torch.bfloat16, device="cuda")
        run_gradient(ctx, case, vm, token, lse2, entropy2, d_logp, d_entropy, d_hidden, None)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
        d_logits = torch.zeros_like(logits)
        cz.cfgzip_token_logprobs_backward(ctx.h, logits, cz.F32, V, B, V, None, 0, token, 1.0, lse, entropy, d_logp, d_entropy, d_logits, V,
                                          st)
        assert ((d_logits - g).abs() <= g_tol).all()


def test_captured_and_two_at_once_and_a_workspace_made_for_more():
    cases = [loss_inputs(V, 128, N, 0.3, 0, seed=4) for V, N in ((5003, 300), (9001, 40))]
    st = [torch.cuda.Stream() for _ in cases]
    with Ctx([]) as one, Ctx([]) as two:
        want, graphs, results, kept = [], [], [], []
        for ctx, side, (case, mask, packed, tokens) in zip((one, two), st, cases):
            N, V, H = case.rows, case.V, case.H
            d = torch.randn(N, generator=case.gen, device="cuda")
            ws = case.workspace(cz.HEAD_LOGPROBS, 2 * N), case.workspace(cz.HEAD_LOGPROBS_BACKWARD, 2 * N)
            o = tuple(torch.zeros(N, device="cuda") for _ in range(3))
            d_hidden, d_weight = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, H), device="cuda")

            def both(stream):
                cz.cfgzip_head_logprobs(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], tokens, *o, ws[0], ws[0].numel(), stream)
                run_gradient(ctx, case, packed, tokens, o[2], o[1], d, d, d_hidden, d_weight, workspace=ws[1], stream=stream)

            side.wait_stream(torch.cuda.current_stream())
            both(side)
            side.synchronize()
            want.append([t.clone() for t in (*o, d_hidden, d_weight)])
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                both(side)
            graphs.append(graph)
            results.append((*o, d_hidden, d_weight))
            kept.append((ws, d))
        for _ in range(3):
            for r in results:
                for t in r:
                    t.zero_()
            torch.cuda.synchronize()
            for graph, side in zip(graphs, st):
                with torch.cuda.stream(side):
                    graph.replay()
            torch.cuda.synchronize()
            for r, w in zip(results, want):
                assert all(torch.equal(a, b) for a, b in zip(r, w))


def test_no_rows_and_waits_that_run_out():
    case, mask, packed, tokens = loss_inputs(5003, 256, 300, 0.5, 0)
    d_weight = torch.full((5003, 264), 77.0, dtype=torch.bfloat16, device="cuda")
    d = torch.randn(300, generator=case.gen, device="cuda")
    d_hidden = torch.zeros((300, 256), dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.current_stream()
    with Ctx([]) as ctx:
        cz.cfgzip_head_logprobs(ctx.h, case.head, None, 0, 0, None, 0, None, None, None, None, None, 0, st)
        for accumulate in (1, 0):
            cz.cfgzip_head_logprobs_backward(ctx.h, case.head, None, 0, 0, None, 0, None, None, None, None, None, None, 0, d_weight, cz.BF16,
                                             264, accumulate, None, 0, st)
            assert (d_weight[:, :256] == (77.0 if accumulate else 0.0)).all() and (d_weight[:, 256:] == 77.0).all()
        status = lambda: cz.load_library().cfgzip_poll_status(ctx.h, None, None, None, None)
        status()
        first = run(ctx, case, packed, tokens)
        run_gradient(ctx, case, packed, tokens, first[2], first[1], d, d, d_hidden, None)
        kept = d_hidden.clone()
        assert status() == cz.OK
        cz.cfgzip_set_tuning(ctx.h, "test_expire_waits", 1)  # (waits that are over are reported as run out: nothing hangs)
        run(ctx, case, packed, tokens)
        assert status() == cz.E_CUDA
        run_gradient(ctx, case, packed, tokens, first[2], first[1], d, d, d_hidden, None)
        assert status() == cz.E_CUDA
        cz.cfgzip_set_tuning(ctx.h, "test_expire_waits", 0)
        again = run(ctx, case, packed, tokens)
        run_gradient(ctx, case, packed, tokens, first[2], first[1], d, d, d_hidden, None)
        assert status() == cz.OK and all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(kept, d_hidden)
