"""Gradients of log probabilities from hidden states as programs call them: results in the place of inputs, tokens that come again and again."""
import pytest
import torch

from _gpu_util import Ctx
from test_gpu_head import close, loss_inputs
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
