"""The layer in front of a head and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx, dev
from _head_util import class_masks, padded

pytestmark = pytest.mark.gpu
ACTS = {"none": cz.ACT_NONE, "relu": cz.ACT_RELU, "gelu": cz.ACT_GELU, "gelu_tanh": cz.ACT_GELU_TANH, "silu": cz.ACT_SILU}
HALF = 2.0 ** -8  # half a step of bf16


def activation(act, h):
    if act == "relu":
        return h.clamp(min=0), (h > 0).double()
    if act == "silu":
        q = torch.sigmoid(h)
        return h * q, q + h * q * torch.sigmoid(-h)
    if act == "gelu":
        return h * torch.special.ndtr(h), torch.special.ndtr(h) + h * torch.exp(-h * h / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        q, r = torch.sigmoid(k * (h + 0.044715 * h ** 3)), torch.sigmoid(-k * (h + 0.044715 * h ** 3))
        return h * q, q + h * q * r * k * (1 + 3 * 0.044715 * h * h)
    return h, torch.ones_like(h)


class Layer:
    def __init__(self, rows, in_, out, act, bias, pad=0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + rows + 1000 * in_ + 77 * out)
        self.rows, self.in_, self.out, self.act, self.gen, self.pad = rows, in_, out, act, g, pad
        w = torch.empty((out, in_), device="cuda").normal_(0.0, in_ ** -0.5, generator=g).to(torch.bfloat16)
        self.weight, self.w64 = padded(w, pad), w.double()
        self.bias = None
        if bias != "none":
            self.bias = torch.empty(out, device="cuda").normal_(0.0, 1.0, generator=g)
            self.bias = self.bias.to(torch.bfloat16) if bias == "bf16" else self.bias
        self.layer = cz.cfgzip_layer(self.weight, in_, out, ACTS[act], self.bias, cz.BF16 if bias == "bf16" else cz.F32, self.weight.stride(0))
        self.x = self.rows_of(in_, 1.5)
        self.x64 = self.x.double()

    def rows_of(self, n, deviation=1.0):
        return padded(torch.empty((self.rows, n), device="cuda").normal_(0.0, deviation, generator=self.gen).to(torch.bfloat16), self.pad)

    def workspace(self, op, rows=None):
        n = cz.cfgzip_layer_workspace(self.layer, op, self.rows if rows is None else rows)
        return torch.full((max(n, 1),), 255, dtype=torch.uint8, device="cuda")  # (NaN wherever a number is read that was not written)

    def forward(self, ctx, residual, y, slope, stream=None):
        ws = self.workspace(cz.LAYER_FORWARD)
        cz.cfgzip_layer_forward(ctx.h, self.layer, self.x, self.x.stride(0), self.rows, residual,
                                0 if residual is None else residual.stride(0), y, y.stride(0), slope, 0 if slope is None else slope.stride(0),
                                ws, ws.numel(), stream or torch.cuda.current_stream())

    def check(self, y, slope, residual):
        h = self.x64 @ self.w64.T
        # a sum of products in 32 bits, in any order (what tensor memory cuts off, 2^-29 per element, is less), and the bias
        h_tol = self.in_ * 2.0 ** -24 * (self.x64.abs() @ self.w64.abs().T)
        if self.bias is not None:
            h = h + self.bias.double()
            h_tol = h_tol + h.abs() * 2.0 ** -24
        # slopes are 1.13 at most and change by 0.8 at most for each unit; the functions are good to a few units in the last place, which
        # counts 8 times at most where they are taken of arguments of that size
        of, by = activation(self.act, h)
        want = of if residual is None else of + residual.double()
        tol = 1.13 * h_tol + of.abs() * 2.0 ** -19 + 2.0 ** -24 + want.abs() * HALF * 1.001
        if self.act == "gelu":
            tol = tol + h.abs() * 0.5 * 1.5e-7  # the approximation of erf
        assert ((y.double() - want).abs() <= tol).all()
        if slope is None:
            return
        ok = (slope.double() - by).abs() <= 0.8 * h_tol + 2.0 ** -19 * (1 + h.abs()) + by.abs() * HALF * 1.001
        if self.act == "relu":
            ok |= h.abs() <= h_tol  # (on either side of 0)
        assert ok.all()


SHAPES = [
    # rows, in, out, pad
    (1, 8, 8, 0), (1, 64, 40, 8), (2, 72, 128, 0), (15, 128, 136, 8), (16, 256, 256, 0), (17, 200, 264, 0), (31, 1000, 128, 8),
    (32, 2048, 512, 0), (33, 520, 1032, 0), (64, 4096, 128, 0), (100, 328, 2056, 8), (128, 512, 384, 0), (129, 512, 384, 8),
    (200, 1024, 256, 0), (257, 72, 1000, 0), (1, 4096, 4096, 0), (3, 8192, 200, 0), (500, 1032, 2568, 8), (1500, 264, 520, 0),
    (3000, 1024, 1032, 8), (5000, 512, 768, 0), (9001, 136, 264, 0), (2049, 4104, 520, 0), (20000, 8, 8, 0), (4000, 2056, 2312, 8), (1800, 5000, 1024, 0),
]


@pytest.mark.parametrize("rows,in_,out,pad", SHAPES)
def test_layer(rows, in_, out, pad):
    with Ctx([]) as ctx:
        for i, (act, bias, with_residual, with_slope) in enumerate((("none", "none", False, False), ("silu", "bf16", True, True),
                                                                     ("gelu", "f32", False, True), ("gelu_tanh", "none", True, False),
                                                                     ("relu", "f32", True, True), ("none", "bf16", True, True))):
            l = Layer(rows, in_, out, act, bias, pad, seed=i)
            residual = None
            if with_residual:
                residual = l.x if in_ == out and i % 2 else l.rows_of(out)
            y, slope = (torch.full((rows, out + 8), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            l.forward(ctx, residual, y[:, :out], slope[:, :out] if with_slope else None)
            assert (y[:, out:] == 77.0).all() and (slope[:, out:] == 77.0).all()
            l.check(y[:, :out], slope[:, :out] if with_slope and act != "none" else None, residual)
            if with_residual and residual is not l.x:  # in the residual's place
                l.forward(ctx, residual, residual, None)
                assert torch.equal(residual, y[:, :out])


def test_layer_where_activations_end():
    """Arguments far out: nothing that is not a number, and the functions' ends."""
    rows, n = 300, 64
    with Ctx([]) as ctx:
        for rows in (20, 300, 5000):
            for act in ACTS:
                l = Layer(rows, n, n, act, "none")
                l.weight.copy_(torch.eye(n, device="cuda"))
                l.w64 = l.weight.double()
                l.x[:] = (2.0 ** torch.linspace(-20, 100, n, device="cuda")).to(torch.bfloat16)
                l.x[1::2] *= -1
                l.x64 = l.x.double()
                y, slope = torch.zeros_like(l.x), torch.zeros_like(l.x)
                l.forward(ctx, None, y, slope)
                of, by = activation(act, l.x64)
                by = torch.where(l.x64.abs() > 1e3, (l.x64 > 0).double() if act != "none" else 1.0, by)
                of = torch.where(l.x64.abs() > 1e3, torch.where((l.x64 > 0) | (act == "none"), l.x64, 0.0), of)
                assert y.isfinite().all()
                assert ((y.double() - of).abs() <= of.abs() * HALF * 1.01 + 2.0 ** -19 * l.x64.abs().clamp(max=64)).all()
                if act != "none":
                    assert ((slope.double() - by).abs() <= by.abs() * HALF * 1.01 + 2.0 ** -13).all()


# ---- the gradient -----------------------------------------------------------------------------------------------------------
def close(got, want, size, n, before=None):
    """A sum of n exact products, rounded n times in 32 bits at the most, and once to the result."""
    tol = n * 2.0 ** -24 * size
    if before is not None:
        want = want + before.double()
        tol = tol + 2.0 ** -23 * (want.abs() + before.double().abs())
    tol = tol + want.abs() * (HALF if got.dtype == torch.bfloat16 else 2.0 ** -24) * 1.001 + 1e-38
    return ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows,in_,out,pad", SHAPES)
def test_gradient(rows, in_, out, pad):
    st = torch.cuda.current_stream()
    with Ctx([]) as ctx:
        for i, (act, dtype, accumulate, with_add) in enumerate((("silu", torch.bfloat16, 0, True), ("none", torch.float32, 0, False),
                                                                 ("gelu", torch.float32, 1, False), ("none", torch.bfloat16, 1, True))):
            l = Layer(rows, in_, out, act, "f32", pad, seed=i)
            d_y = l.rows_of(out)
            add = (d_y if in_ == out else l.rows_of(in_)) if with_add else None
            slope = l.rows_of(out) if act != "none" else None
            exact = d_y.double() if slope is None else d_y.double() * slope.double()
            g = (d_y if slope is None else (d_y.float() * slope.float()).to(torch.bfloat16)).double()
            d_x = torch.full((rows, in_ + 8), 77.0, dtype=torch.bfloat16, device="cuda")
            d_weight = torch.full((out, in_ + 8), 77.0, dtype=dtype, device="cuda")
            d_bias = torch.full((out,), 77.0, device="cuda")
            w0 = b0 = None
            if accumulate:
                w0, b0 = torch.randn((out, in_), generator=l.gen, device="cuda").to(dtype), torch.randn(out, generator=l.gen, device="cuda")
                d_weight[:, :in_], d_bias[:] = w0, b0
            ws = l.workspace(cz.LAYER_BACKWARD)

            def run(d_x, d_weight, d_bias, add=add):
                cz.cfgzip_layer_backward(ctx.h, l.layer, l.x, l.x.stride(0), rows, slope, 0 if slope is None else slope.stride(0), d_y,
                                         d_y.stride(0), add, 0 if add is None else add.stride(0), d_x, 0 if d_x is None else d_x.stride(0),
                                         d_weight, cz.BF16 if dtype == torch.bfloat16 else cz.F32,
                                         0 if d_weight is None else d_weight.stride(0), d_bias, accumulate, ws, ws.numel(), st)

            run(d_x[:, :in_], d_weight[:, :in_], d_bias)
            assert (d_x[:, in_:] == 77.0).all() and (d_weight[:, in_:] == 77.0).all()
            assert close(d_x[:, :in_], g @ l.w64, g.abs() @ l.w64.abs(), out, add)
            assert close(d_weight[:, :in_], g.T @ l.x64, g.abs().T @ l.x64.abs(), rows, w0)
            assert close(d_bias, exact.sum(dim=0), exact.abs().sum(dim=0), rows, b0)
            # each alone is the same, and d_x may be where `add` is
            alone = add.clone() if add is not None else torch.zeros_like(d_x[:, :in_])
            run(alone, None, None, add=alone if add is not None else None)
            assert torch.equal(alone, d_x[:, :in_])
            alone = d_bias.clone() if not accumulate else b0.clone()
            run(None, None, alone)
            assert torch.equal(alone, d_bias)
            alone = w0.clone() if accumulate else torch.zeros((out, in_), dtype=dtype, device="cuda")
            run(None, alone, None)
            assert torch.equal(alone, d_weight[:, :in_])


def test_gradient_is_that_of_the_layer():
    """Against differences in 64 bits, by way of the slopes that the forward pass left."""
    rows, n = 40, 96
    with Ctx([]) as ctx:
        for act in ("silu", "gelu", "gelu_tanh"):
            l = Layer(rows, n, n, act, "f32")
            y, slope = torch.zeros_like(l.x), torch.zeros_like(l.x)
            l.forward(ctx, l.x, y, slope)
            d_y = l.rows_of(n)
            d_x, d_weight, d_bias = torch.zeros_like(l.x), torch.zeros((n, n), device="cuda"), torch.zeros(n, device="cuda")
            ws = l.workspace(cz.LAYER_BACKWARD)
            cz.cfgzip_layer_backward(ctx.h, l.layer, l.x, n, rows, slope, n, d_y, n, d_y, n, d_x, n, d_weight, cz.F32, n, d_bias, 0, ws,
                                     ws.numel(), torch.cuda.current_stream())

            def value(x, w, b):
                return (d_y.double() * (x + activation(act, x @ w.T + b)[0])).sum()

            eps, at = 1e-6, (l.x64, l.w64, l.bias.double())
            for k, d in enumerate((d_x, d_weight, d_bias)):
                move = [eps * d.double() if i == k else 0.0 for i in range(3)]
                slope_ = ((value(*[a + m for a, m in zip(at, move)]) - value(*[a - m for a, m in zip(at, move)])) / (2 * eps)).item()
                length = (d.double() ** 2).sum().item()
                # elements are off by 2^-8 (slope) + 2^-8 (g) + 2^-8 (result) of their terms: 2 % of the products at the worst
                assert abs(slope_ - length) <= 0.02 * length


def test_no_rows_and_waits_that_run_out():
    st = torch.cuda.current_stream()
    with Ctx([]) as ctx:
        l = Layer(1, 64, 40, "silu", "f32")
        cz.cfgzip_layer_forward(ctx.h, l.layer, None, 0, 0, None, 0, None, 0, None, 0, None, 0, st)
        d_weight, d_bias = torch.full((40, 72), 77.0, device="cuda"), torch.full((40,), 77.0, device="cuda")
        for accumulate in (1, 0):
            cz.cfgzip_layer_backward(ctx.h, l.layer, None, 0, 0, None, 0, None, 0, None, 0, None, 0, d_weight, cz.F32, 72, d_bias, accumulate,
                                     None, 0, st)
            assert (d_weight[:, :64] == (77.0 if accumulate else 0.0)).all() and (d_weight[:, 64:] == 77.0).all()
            assert (d_bias == (77.0 if accumulate else 0.0)).all()
        status = lambda: cz.load_library().cfgzip_poll_status(ctx.h, None, None, None, None)
        for rows, in_, out in ((20, 2048, 512), (3000, 1024, 1032), (40, 64, 72)):
            l = Layer(rows, in_, out, "silu", "bf16")
            y, again, residual = (l.rows_of(out) for _ in range(3))
            status()
            l.forward(ctx, residual, y, None)
            assert status() == cz.OK
            cz.cfgzip_set_tuning(ctx.h, "test_expire_waits", 1)  # (waits that are over are reported as run out: nothing hangs)
            l.forward(ctx, residual, again, None)
            assert status() == cz.E_CUDA
            cz.cfgzip_set_tuning(ctx.h, "test_expire_waits", 0)
            l.forward(ctx, residual, again, None)
            assert status() == cz.OK and torch.equal(y, again)


def test_drafting_and_training_a_layer_under_a_grammar():
    """As they are used together: the layer drafts hidden states, the head chooses under the grammar, the draft is scored; then the layer
    is trained on log probabilities through the head. Captured, and replayed on new inputs on another stream."""
    V, n, B, K = 3001, 256, 24, 60
    st = torch.cuda.Stream()
    p = synth.zipf_partition(V, K, 1.1, seed=2)
    cm = dev(class_masks(K, B, 0.4, (9, 4)))
    VW = (V + 31) // 32
    with Ctx([p]) as ctx:
        l = Layer(B, n, n, "silu", "bf16")
        w = torch.empty((V, n), device="cuda").normal_(0.0, n ** -0.5, generator=l.gen).to(torch.bfloat16)
        head = cz.cfgzip_head(w, cz.BF16, V, n)
        y, slope = torch.zeros_like(l.x), torch.zeros_like(l.x)
        vm = torch.zeros((B, VW), dtype=torch.int32, device="cuda")
        token = torch.zeros(B, dtype=torch.int32, device="cuda")
        step_logp, logp, entropy, lse = (torch.zeros(B, device="cuda") for _ in range(4))
        ones, more = torch.ones(B, device="cuda"), torch.full((B,), 0.01, device="cuda")
        d_y, d_x = torch.zeros_like(l.x), torch.zeros_like(l.x)
        d_weight, d_bias = torch.zeros((n, n), device="cuda"), torch.zeros(n, device="cuda")
        ws = torch.empty(max([cz.cfgzip_head_workspace(head, op, B) for op in (cz.HEAD_STEP, cz.HEAD_LOGPROBS, cz.HEAD_LOGPROBS_BACKWARD)] +
                             [cz.cfgzip_layer_workspace(l.layer, op, B) for op in (cz.LAYER_FORWARD, cz.LAYER_BACKWARD)]),
                         dtype=torch.uint8, device="cuda")
        size = ws.numel()

        def all_of_it():
            cz.cfgzip_layer_forward(ctx.h, l.layer, l.x, n, B, l.x, n, y, n, slope, n, ws, size, st)
            cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, cm, cm.shape[1], head, y, n, B, vm, VW, None, 0, 0, token, None, step_logp, None, ws,
                                size, st)
            cz.cfgzip_head_logprobs(ctx.h, head, y, n, B, vm, VW, token, logp, entropy, lse, ws, size, st)
            cz.cfgzip_head_logprobs_backward(ctx.h, head, y, n, B, vm, VW, token, lse, entropy, ones, more, d_y, n, None, cz.F32, 0, 0, ws,
                                             size, st)
            cz.cfgzip_layer_backward(ctx.h, l.layer, l.x, n, B, slope, n, d_y, n, d_y, n, d_x, n, d_weight, cz.F32, n, d_bias, 0, ws, size, st)

        torch.cuda.synchronize()
        all_of_it()
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            all_of_it()
        l.x.copy_(torch.empty((B, n), device="cuda").normal_(0.0, 2.0, generator=l.gen))
        l.x64 = l.x.double()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        l.check(y, slope, l.x)
        assert (logp - step_logp).abs().max() <= 2.0 ** -16 * (y.double().abs() @ w.double().abs().T).max()
        z = (y.double() @ w.double().T).masked_fill(((vm.repeat_interleave(32, 1)[:, :V] >> (torch.arange(V, device="cuda") % 32)) & 1) == 0, -math.inf)
        logp64 = torch.log_softmax(z, dim=1)
        assert (logp64.gather(1, token.long().unsqueeze(1)).squeeze(1) - logp).abs().max() <= 1e-4
        g = (d_y.float() * slope.float()).to(torch.bfloat16).double()
        assert close(d_x, g @ l.w64, g.abs() @ l.w64.abs(), n, d_y)
        assert close(d_weight, g.T @ l.x64, g.abs().T @ l.x64.abs(), B)
        assert close(d_bias, (d_y.double() * slope.double()).sum(dim=0), (d_y.double() * slope.double()).abs().sum(dim=0), B)


def test_results_in_the_place_of_what_others_still_read_are_refused():
    with Ctx([]) as ctx:
        l = Layer(5, 64, 64, "silu", "none")
        y, slope, d_x = (torch.zeros_like(l.x) for _ in range(3))
        st, ws = torch.cuda.current_stream(), l.workspace(cz.LAYER_BACKWARD)

        def refused(call, *a):
            with pytest.raises(cz.CfgzipError) as e:
                call(ctx.h, l.layer, *a, ws, ws.numel(), st)
            assert e.value.status == cz.E_ARG

        for y_, slope_ in ((l.x, slope), (l.x, None), (y, l.x), (y, y), (y, d_x)):
            refused(cz.cfgzip_layer_forward, l.x, 64, 5, d_x, 64, y_, 64, slope_, 64)
        for d_x_ in (y, l.x, slope):
            refused(cz.cfgzip_layer_backward, l.x, 64, 5, slope, 64, y, 64, y, 64, d_x_, 64, None, cz.F32, 0, None, 0)
        torch.cuda.synchronize()
        assert not y.any() and not slope.any() and not d_x.any()
