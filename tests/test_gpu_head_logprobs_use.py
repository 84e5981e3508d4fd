"""Gradients of log probabilities from hidden states as programs call them: results in the place of inputs, tokens that come again and again."""
import pytest
import torch

from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from test_gpu_head import close, loss_inputs, run_loss
from test_gpu_head_logprobs import gradient, run, run_gradient

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,H,N", [(300, 64, 9), (5003, 256, 300), (2000, 1032, 1000)])
def test_gradient_in_the_place_of_the_hidden_states(V, H, N):
    case, mask, packed, tokens = loss_inputs(V, H, N, 0.5, 8, seed=21)
    d_logp, d_entropy = (torch.randn(N, generator=case.gen, device="cuda") for _ in range(2))
    with Ctx([]) as ctx:
        _, entropy, lse = run(ctx, case, packed, tokens)
        want = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, H), device="cuda")
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, *want)
        hidden = case.hidden.clone()
        for with_weight in (True, False):
            for again in range(3):
                case.hidden.copy_(hidden)
                d_weight = torch.zeros((V, H), device="cuda") if with_weight else None
                run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, case.hidden, d_weight)
                assert torch.equal(case.hidden, want[0])
                assert d_weight is None or torch.equal(d_weight, want[1])
        # some rows further on in the same buffer
        buffer = torch.zeros((N + 3, H), dtype=torch.bfloat16, device="cuda")
        case.hidden = buffer[:N]
        case.hidden.copy_(hidden)
        d_weight = torch.zeros((V, H), device="cuda")
        run_gradient(ctx, case, packed, tokens, lse, entropy, d_logp, d_entropy, buffer[3:], d_weight)
        assert torch.equal(buffer[3:], want[0]) and torch.equal(d_weight, want[1])


@pytest.mark.parametrize("V,H,N,counts", [(300, 64, 60, (2, 15, 16, 17, 1)), (5003, 520, 1300, (1, 18, 1000)), (200, 1032, 2500, (1100, 1025, 33)),
                                          (2000, 264, 5000, (5000,)), (40, 64, 1000, (3,) * 300), (9001, 512, 4100, (16, 17, 2049, 1024))])
def test_tokens_that_come_again_and_again(V, H, N, counts):
    """Chains of rows with one target, of every kind of length, mixed up: what each row's g loses in bf16 comes back in 32 bits."""
    case, mask, packed, tokens = loss_inputs(V, H, N, None, 0, seed=12)
    many = torch.cat([torch.full((n,), (17 * k + 5) % V, dtype=torch.int32, device="cuda") for k, n in enumerate(counts)])[:N]
    order = torch.randperm(N, generator=case.gen, device="cuda")
    tokens[order[:len(many)]] = many
    d_logp = torch.rand(N, generator=case.gen, device="cuda") + 0.5
    rows, t = torch.arange(N, device="cuda"), tokens.long().clamp(0, V - 1)
    has = (tokens >= 0) & (tokens < V)
    at = rows[has], t[has]
    with Ctx([]) as ctx:
        _, _, lse = run(ctx, case, packed, tokens)
        g, g_tol = gradient(case, mask, tokens, d_logp, None)
        g_tol[at] -= g[at].abs() * (2.0 ** -8 - 2.0 ** -23)  # (without its rounding to bf16: twice a rounding in 32 bits)
        for dtype, accumulate in ((torch.float32, 0), (torch.bfloat16, 1)):
            d_weight = torch.randn((V, H), generator=case.gen, device="cuda").to(dtype)
            before = d_weight.clone() if accumulate else None
            d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
            run_gradient(ctx, case, packed, tokens, lse, None, d_logp, None, d_hidden, d_weight, accumulate)
            assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N, before)
            assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
            again = before.clone() if accumulate else torch.zeros_like(d_weight)
            run_gradient(ctx, case, packed, tokens, lse, None, d_logp, None, d_hidden, again, accumulate)
            assert torch.equal(again, d_weight)


def test_tokens_that_come_again_take_no_other_time():
    """A text of one token: no load that waits for the one before for each of its rows (7 ms were beside a tenth of one)."""
    V, H, N = 2000, 4096, 4000
    case, mask, packed, tokens = loss_inputs(V, H, N, None, 0, seed=13)
    d = torch.rand(N, generator=case.gen, device="cuda")
    d_weight = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    with Ctx([]) as ctx:
        _, _, lse = run(ctx, case, packed, tokens)
        ws = case.workspace(cz.HEAD_LOGPROBS_BACKWARD)

        def least(tokens):
            times = []
            for _ in range(6):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                for _ in range(3):
                    run_gradient(ctx, case, packed, tokens, lse, None, d, None, None, d_weight, workspace=ws)
                b.record()
                b.synchronize()
                times.append(a.elapsed_time(b))
            return min(times)

        assert least(torch.full_like(tokens, 7)) <= 4 * least(tokens)


def scored(ctx, weight, hidden, tokens):
    V, H, N = weight.shape[0], weight.shape[1], hidden.shape[0]
    head = cz.cfgzip_head(weight, cz.BF16, V, H)
    ws = torch.empty(cz.cfgzip_head_workspace(head, cz.HEAD_LOGPROBS, N), dtype=torch.uint8, device="cuda")
    logp, entropy, lse = (torch.full((N,), 99.0, device="cuda") for _ in range(3))
    cz.cfgzip_head_logprobs(ctx.h, head, hidden, H, N, None, 0, tokens, logp, entropy, lse, ws, ws.numel(), torch.cuda.current_stream())
    return logp, entropy, lse


@pytest.mark.parametrize("size", [1e35, 3e36, 2e37, 1.5e38])
def test_scores_as_large_as_a_float_holds(size):
    """One token's score, and whole tiles of tokens at 0 or at as much below it."""
    V, H, N = 3000, 64, 300
    weight = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    weight[2500, 0], weight[600:900, 0] = 1.0, -1.0
    hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
    hidden[:, 0] = size
    hidden[1::2, 0] = -size
    tokens = torch.full((N,), 2500, dtype=torch.int32, device="cuda")
    tokens[1::2] = 700
    with Ctx([]) as ctx:
        logp, entropy, lse = scored(ctx, weight, hidden, tokens)
    of = hidden[:, 0].float().abs()
    assert (lse == of).all()
    log_n = torch.log(torch.tensor(300.0, dtype=torch.float64)).item()
    assert (logp[::2] == 0).all() and (entropy[::2] == 0).all()
    # three hundred equal scores, in exact arithmetic: the roundings of a logarithm
    assert ((logp[1::2] + log_n).abs() <= 2.0 ** -20).all() and ((entropy[1::2] - log_n).abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("V,N", [(2000, 3), (50000, 3), (9000, 300)])
def test_a_nearly_certain_token_keeps_what_the_others_have_together(V, N):
    """Scores of small whole numbers, exact in 32 bits: what is left of the log probability is good to the bits of the others' sum, not of
    the 1 beside it; the same of the entropy."""
    H = 64
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    weight = torch.zeros((V, H), device="cuda")
    weight[:, :8] = torch.randint(-4, 5, (V, 8), generator=g, device="cuda") / 4
    weight[5, :] = 0.0
    weight[5, 8] = 1.0
    hidden = torch.zeros((N, H), device="cuda")
    hidden[:, :8] = torch.randint(-2, 3, (N, 8), generator=g, device="cuda") / 2
    hidden[:, 8] = torch.tensor([20.0, 24.0, 28.0], device="cuda").repeat(N // 3)
    weight, hidden = weight.to(torch.bfloat16), hidden.to(torch.bfloat16)
    tokens = torch.full((N,), 5, dtype=torch.int32, device="cuda")
    with Ctx([]) as ctx:
        logp, entropy, _ = scored(ctx, weight, hidden, tokens)
    z = hidden.double() @ weight.double().T
    x = z - z[:, 5:6]
    x[:, 5] = -float("inf")
    rest = torch.exp(x).sum(dim=1)
    want = -torch.log1p(rest)
    want_entropy = torch.log1p(rest) - (torch.exp(x) * x).nan_to_num(0.0).sum(dim=1) / (1.0 + rest)
    # the others' terms: an argument within 40 powers of two rounded twice (40 * 2^-23 ln 2), an exponential good to a few units, 32 additions
    # in a row, some 30 where chains and tiles meet: below 2^-16 of the sum together; the entropy's terms are as many, with a product each
    assert ((logp - want).abs() <= 2.0 ** -16 * want.abs()).all()
    assert ((entropy - want_entropy).abs() <= 2.0 ** -15 * want_entropy).all()


@pytest.mark.parametrize("V,H,N", [(300, 64, 9), (2000, 1032, 1000)])
def test_gradient_of_the_loss_in_the_place_of_the_hidden_states(V, H, N):
    case, mask, packed, targets = loss_inputs(V, H, N, 0.5, 8, seed=22)
    d_loss = torch.rand(N, generator=case.gen, device="cuda")
    ws = case.workspace(cz.HEAD_LOSS_BACKWARD)
    with Ctx([]) as ctx:
        _, lse = run_loss(ctx, case, packed, targets)

        def backward(d_hidden, d_weight):
            cz.cfgzip_head_loss_backward(ctx.h, case.head, case.hidden, case.hidden.stride(0), N, packed, packed.shape[1], targets, lse, d_loss,
                                         d_hidden, d_hidden.stride(0), d_weight, cz.F32, H, 0, ws, ws.numel(), torch.cuda.current_stream())

        want, got = (torch.zeros((V, H), device="cuda") for _ in range(2))
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        backward(d_hidden, want)
        backward(case.hidden, got)
        assert torch.equal(case.hidden, d_hidden) and torch.equal(got, want)
