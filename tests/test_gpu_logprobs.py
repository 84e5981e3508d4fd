"""Log probabilities of given tokens, entropies and top alternatives from logits, and their gradient, against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx
from _head_util import pack

pytestmark = pytest.mark.gpu
INF = float("inf")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative (bf16: of results in 16 bits)
CODE = {torch.bfloat16: cz.BF16, torch.float32: cz.F32}


def words(n):
    return (n + 31) // 32


class Rows:
    """Logits [N, V] inside a wider buffer, `shift` elements behind its start, with NaN everywhere else."""

    def __init__(self, N, V, dtype=torch.bfloat16, pad=0, shift=0, seed=0, density=None, t=1.0, deviation=2.0, offset=0.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1000003 * N + V)
        self.N, self.V, self.dtype, self.gen, self.t = N, V, dtype, g, t
        self.stride = V + pad
        self.buffer = torch.full((N * self.stride + shift,), float("nan"), dtype=dtype, device="cuda")
        self.logits = self.buffer[shift:shift + N * self.stride].view(N, self.stride)[:, :V]
        self.logits.copy_(torch.empty((N, V), device="cuda").normal_(offset, deviation, generator=g))
        self.tokens = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        self.allowed, self.mask, self.words = None, None, 0
        if density is not None:
            self.allow(torch.rand((N, V), generator=g, device="cuda") < density)

    def allow(self, allowed):
        self.allowed = allowed
        self.words = words(self.V) + 1
        self.mask = torch.full((self.N, self.words), -1, dtype=torch.int32, device="cuda")
        packed = pack(allowed)
        if self.V % 32:
            packed[:, -1] |= -1 << (self.V % 32)  # bits behind the vocabulary must not matter
        self.mask[:, :-1] = packed

    def scores(self):
        z = self.logits.double() * torch.tensor(1.0 / self.t, dtype=torch.float32).double().item()
        return z if self.allowed is None else torch.where(self.allowed, z, -INF)

    def run(self, ctx, n_top=0, stream=None, out=None):
        N = self.N
        if out is None:
            out = dict(logp=torch.full((N,), 99.0, device="cuda"), entropy=torch.full((N,), 99.0, device="cuda"),
                       lse=torch.full((N,), 99.0, device="cuda"))
            if n_top:
                out["top_tokens"] = torch.full((N, n_top), -7, dtype=torch.int32, device="cuda")
                out["top_logp"] = torch.full((N, n_top), 99.0, device="cuda")
        cz.cfgzip_token_logprobs(ctx.h, self.logits, CODE[self.dtype], self.stride, N, self.V, self.mask, self.words, self.tokens,
                                 1.0 / self.t, n_top, out["logp"], out["entropy"], out["lse"], out.get("top_tokens"), out.get("top_logp"),
                                 stream or torch.cuda.current_stream())
        return out

    def tolerances(self, z):
        """A sum of exponentials: at most V / 512 additions in a row for a thread and some 40 where threads, warps and blocks meet, an
        exponential good to a few units and its argument to 2^-23 of itself (whose average is log s - entropy); then the roundings of
        the results. The reference of a sum may be 8 powers of two (6 nats) below its largest value: so much is added and taken away."""
        lse = torch.logsumexp(z, dim=1)
        entropy = torch.special.entr(torch.softmax(z, dim=1)).sum(dim=1)
        log_s = lse - z.amax(dim=1)
        steps = (self.V / 512 + 48) * 2.0 ** -23
        of_sum = steps * (1 + (log_s - entropy).abs())
        lse_tol = (of_sum + lse.abs() * 2.0 ** -22).nan_to_num(0.0, 0.0)  # (rows with nothing allowed: exact)
        return lse, entropy, lse_tol, steps * (8 + log_s + 2 * (log_s - entropy).abs())

    def check(self, out, n_top=0):
        N, V = self.N, self.V
        z = self.scores()
        none = (z == -INF).all(dim=1)
        lse, entropy, lse_tol, entropy_tol = self.tolerances(z)
        assert (out["lse"][none] == -INF).all() and (out["entropy"][none] == 0).all()
        ok = ~none
        assert ((out["lse"] - lse).abs() <= lse_tol)[ok].all()
        assert ((out["entropy"] - entropy).abs() <= entropy_tol)[ok].all()
        rows, t = torch.arange(N, device="cuda"), self.tokens.long()
        of_token = z[rows, t.clamp(0, V - 1)]
        want = torch.where(t < 0, 0.0, torch.where((t < V) & (of_token > -INF), of_token - lse, -INF))
        finite = want > -INF
        assert (out["logp"][~finite] == -INF).all()
        assert ((out["logp"] - want).abs() <= lse_tol + want.abs() * 2.0 ** -22)[finite].all()
        assert (out["logp"][t < 0] == 0).all()
        if not n_top:
            return
        raw = self.logits.double() if self.allowed is None else torch.where(self.allowed, self.logits.double(), -INF)
        values, order = torch.sort(raw, dim=1, descending=True, stable=True)
        n = min(n_top, V)
        want_tokens = torch.full((N, n_top), -1, dtype=torch.int32, device="cuda")
        want_tokens[:, :n] = torch.where(values[:, :n] > -INF, order[:, :n], -1).to(torch.int32)
        assert torch.equal(out["top_tokens"], want_tokens)
        listed = want_tokens >= 0
        assert (out["top_logp"][~listed] == -INF).all()
        want = z.gather(1, want_tokens.long().clamp(min=0)) - lse.unsqueeze(1)
        assert ((out["top_logp"] - want).abs() <= lse_tol.unsqueeze(1) + want.abs() * 2.0 ** -22)[listed].all()


SHAPES = [
    # N, V, pad, shift
    (1, 1, 0, 0), (2, 1, 1, 1), (3, 7, 0, 0), (5, 8, 0, 3), (4, 9, 4, 0), (3, 31, 2, 5), (2, 255, 0, 0), (9, 256, 0, 1), (3, 257, 0, 0),
    (5, 1000, 24, 0), (4, 1003, 0, 2), (70, 4099, 0, 0), (1, 32000, 0, 0), (7, 32003, 5, 4), (33, 50021, 0, 0), (1, 128256, 0, 0),
    (2, 128257, 0, 1), (150, 20011, 0, 0), (300, 9000, 8, 0), (700, 5001, 0, 0), (1, 262144, 0, 0), (1, 1 << 21, 0, 0),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V,pad,shift", SHAPES)
def test_log_probabilities(N, V, pad, shift, dtype):
    with Ctx([]) as ctx:
        for density, t, n_top in ((None, 1.0, 5), (0.3, 0.7, 20), (0.002, 1.0, 32), (None, 0.2, 0), (0.9, 3.0, 1)):
            rows = Rows(N, V, dtype, pad, shift, density=density, t=t)
            if N > 2:
                rows.tokens[1], rows.tokens[2] = -1, V + 5
            if density is not None and N > 3:
                rows.allowed[3] = False
                rows.allow(rows.allowed)
            cz.cfgzip_poll_status(ctx.h)
            out = rows.run(ctx, n_top)
            assert cz.cfgzip_poll_status(ctx.h)[1] == (N > 2)
            rows.check(out, n_top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_is_not_allowed_may_be_anything(dtype):
    N, V = 6, 9001
    with Ctx([]) as ctx:
        rows = Rows(N, V, dtype, density=0.2)
        for value in (float("nan"), INF, -INF, torch.finfo(dtype).min, torch.finfo(dtype).max):
            rows.logits[~rows.allowed] = value
            kept = rows.allowed
            out = rows.run(ctx, 20)
            clean = Rows(N, V, dtype, density=0.2)
            clean.check(out, 20)
            d = backward(ctx, rows, out)
            assert (d[~kept] == 0).all() and d.isfinite().all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_masked_in_place_are_as_good_as_a_mask(dtype):
    N, V = 40, 20003
    with Ctx([]) as ctx:
        rows = Rows(N, V, dtype, density=0.01)
        rows.allowed[7] = False
        rows.allowed[8], rows.allowed[8, 19] = False, True  # a single token: it is certain
        rows.tokens[8] = 19
        rows.allow(rows.allowed)
        a = rows.run(ctx, 32)
        rows.check(a, 32)
        assert a["logp"][8] == 0 and a["entropy"][8] == 0 and a["top_tokens"][8].tolist() == [19] + [-1] * 31
        rows.logits.masked_fill_(~rows.allowed, -INF)
        rows.mask = None
        b = rows.run(ctx, 32)
        rows.check(b, 32)
        assert torch.equal(a["top_tokens"], b["top_tokens"]) and torch.equal(a["logp"], b["logp"])


@pytest.mark.parametrize("values", [1, 2, 5, 40])
@pytest.mark.parametrize("N,V", [(3, 500), (3, 70000), (200, 30011)])
def test_equal_logits_go_by_the_lowest_token(N, V, values):
    with Ctx([]) as ctx:
        for dtype in (torch.bfloat16, torch.float32):
            for density in (None, 0.5, 0.01):
                rows = Rows(N, V, dtype, density=density)
                rows.logits.copy_(torch.randint(0, values, (N, V), generator=rows.gen, device="cuda") - values // 2)
                rows.logits[0, ::3] *= -1.0  # zeros of either sign
                for n_top in (1, 20, 32):
                    rows.check(rows.run(ctx, n_top), n_top)


@pytest.mark.parametrize("offset", [3e4, -3e4, 1e9, -1e9])
def test_rows_far_from_zero(offset):
    # differences of logits are taken before anything is multiplied: what is left of log p is what the logits themselves hold
    N, V = 5, 8003
    with Ctx([]) as ctx:
        rows = Rows(N, V, torch.float32, offset=offset, deviation=abs(offset) * 2.0 ** -20)
        rows.check(rows.run(ctx, 10), 10)


@pytest.mark.parametrize("t", [1e-6, 1e-3, 1e3, 1e6])
def test_temperatures_far_from_one(t):
    with Ctx([]) as ctx:
        for dtype in (torch.bfloat16, torch.float32):
            for density in (None, 0.3):
                rows = Rows(4, 9001, dtype, density=density, t=t)
                out = rows.run(ctx, 10)
                rows.check(out, 10)
                check_gradient(rows, backward(ctx, rows, out), out["lse"], out["entropy"], *rows.d)


def test_rows_that_rise_and_fall():
    # the reference of a sum has to move, upwards from the start of the row or once at its end
    V = 60000
    with Ctx([]) as ctx:
        rows = Rows(4, V, torch.float32)
        ramp = torch.linspace(-200, 200, V, device="cuda")
        rows.logits[0], rows.logits[1] = ramp, ramp.flip(0)
        rows.logits[2] = -300.0
        rows.logits[2, V - 1] = 300.0
        rows.logits[3] = -1e28
        rows.logits[3, 77] = 0.0
        rows.check(rows.run(ctx, 32), 32)


def test_only_what_is_asked_for_is_written():
    with Ctx([]) as ctx:
        rows = Rows(3, 5000)
        want = rows.run(ctx, 7)
        st = torch.cuda.current_stream()
        lse = torch.zeros(3, device="cuda")
        top, of_top = torch.zeros((3, 7), dtype=torch.int32, device="cuda"), torch.zeros((3, 7), device="cuda")
        cz.cfgzip_token_logprobs(ctx.h, rows.logits, cz.BF16, 5000, 3, 5000, None, 0, None, 1.0, 0, None, None, lse, None, None, st)
        cz.cfgzip_token_logprobs(ctx.h, rows.logits, cz.BF16, 5000, 3, 5000, None, 0, None, 1.0, 7, None, None, None, top, of_top, st)
        cz.cfgzip_token_logprobs(ctx.h, rows.logits, cz.BF16, 5000, 0, 5000, None, 0, None, 1.0, 7, None, None, None, top, of_top, st)
        assert torch.equal(lse, want["lse"]) and torch.equal(top, want["top_tokens"]) and torch.equal(of_top, want["top_logp"])


def test_offsets_behind_two_billion_elements():
    V, stride = 1000, (1 << 30) + 8
    buffer = torch.empty(2 * stride + 3 * V, dtype=torch.bfloat16, device="cuda")
    rows = Rows(3, V)
    logits = rows.logits
    rows.logits = buffer.as_strided((3, V), (stride, 1))
    rows.logits.copy_(logits)
    rows.stride = stride
    with Ctx([]) as ctx:
        out = rows.run(ctx, 5)
        rows.check(out, 5)
        d = buffer.as_strided((3, V), (stride, 1), 2 * V)
        cz.cfgzip_token_logprobs_backward(ctx.h, rows.logits, cz.BF16, stride, 3, V, None, 0, rows.tokens, 1.0, out["lse"], out["entropy"],
                                          out["lse"], out["lse"], d, stride, torch.cuda.current_stream())
        check_gradient(rows, d, out["lse"], out["entropy"], out["lse"], out["lse"])


# ---- the gradient -----------------------------------------------------------------------------------------------------------
def backward(ctx, rows, out, d_logp=None, d_entropy=None, stream=None, pad=0, shift=0, both=True):
    if both and d_logp is None:
        d_logp = torch.empty(rows.N, device="cuda").normal_(generator=rows.gen)
        d_entropy = torch.empty(rows.N, device="cuda").normal_(generator=rows.gen)
        rows.d = (d_logp, d_entropy)
    stride = rows.V + pad
    buffer = torch.full((rows.N * stride + shift,), 77.0, dtype=rows.dtype, device="cuda")
    d = buffer[shift:].view(rows.N, stride)
    cz.cfgzip_token_logprobs_backward(ctx.h, rows.logits, CODE[rows.dtype], rows.stride, rows.N, rows.V, rows.mask, rows.words, rows.tokens,
                                      1.0 / rows.t, out["lse"], out["entropy"], d_logp, d_entropy, d, stride,
                                      stream or torch.cuda.current_stream())
    assert (d[:, rows.V:] == 77.0).all() and (buffer[:shift] == 77.0).all()
    return d[:, :rows.V]


def check_gradient(rows, got, lse, entropy, d_logp, d_entropy):
    z, it = rows.scores(), torch.tensor(1.0 / rows.t, dtype=torch.float32).double().item()
    some = lse > -INF
    x = z - torch.where(some, lse, 0.0).double().unsqueeze(1)
    p = torch.where(some.unsqueeze(1), torch.exp(x), 0.0)
    t = rows.tokens.long()
    d = torch.zeros_like(z[:, :1]) if d_logp is None else d_logp.double().unsqueeze(1)
    e = torch.zeros_like(z[:, :1]) if d_entropy is None else d_entropy.double().unsqueeze(1)
    H = entropy.double().unsqueeze(1)
    has = (t >= 0) & (t < rows.V) & some
    has &= z.gather(1, t.clamp(0, rows.V - 1).unsqueeze(1)).squeeze(1) > -INF
    d = torch.where(has.unsqueeze(1), d, 0.0)
    at = torch.arange(rows.N, device="cuda")[has]
    rest = -torch.expm1(x[at, t[has]])  # 1 - p of the given tokens
    x = torch.where(p > 0, x, 0.0)
    want = -p * d - e * p * (x + H)
    want[at, t[has]] = d.squeeze(1)[has] * rest - (e * p * (x + H))[at, t[has]]
    # p: its exponent is off by 2^-22 of itself, the exponential by a few units, and below 2^-126 it is 0; the terms are added in 32 bits
    tol = (d.abs() + e.abs() * (x.abs() + H)) * (p * (2.0 ** -20 + x.abs() * 2.0 ** -21) + 2.0 ** -126)
    tol[at, t[has]] += d.squeeze(1)[has].abs() * (rest.abs() + p[at, t[has]] * x[at, t[has]].abs()) * 2.0 ** -21
    tol = tol * it + (want * it).abs() * HALF[rows.dtype] + 1e-36
    assert got.isfinite().all()
    assert ((got.double() - want * it).abs() <= tol).all()
    if rows.allowed is not None:
        assert (got[~rows.allowed] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V,pad,shift", [s for s in SHAPES if s[1] < 1 << 21])
def test_gradient(N, V, pad, shift, dtype):
    with Ctx([]) as ctx:
        for density, t, to_pad, to_shift in ((None, 1.0, pad, shift), (0.3, 0.7, pad, shift), (0.5, 1.0, 3, 1)):
            rows = Rows(N, V, dtype, pad, shift, density=density, t=t)
            if N > 2:
                rows.tokens[1], rows.tokens[2] = -1, V + 5
            if density is not None and N > 3:
                rows.allowed[3] = False
                rows.allow(rows.allowed)
            out = rows.run(ctx)
            got = backward(ctx, rows, out, pad=to_pad, shift=to_shift)
            check_gradient(rows, got, out["lse"], out["entropy"], *rows.d)
            d_logp, d_entropy = rows.d
            got = backward(ctx, rows, out, d_logp=d_logp, pad=to_pad, shift=to_shift)
            check_gradient(rows, got, out["lse"], out["entropy"], d_logp, None)
            got = backward(ctx, rows, out, d_entropy=d_entropy, pad=to_pad, shift=to_shift, both=False)
            check_gradient(rows, got, out["lse"], out["entropy"], None, d_entropy)


def test_gradient_of_tokens_that_have_no_probability():
    # masked in place or not allowed by the mask: no part in the gradient, whichever of a row's blocks looks
    N, V = 6, 60000
    with Ctx([]) as ctx:
        for dtype in (torch.bfloat16, torch.float32):
            rows = Rows(N, V, dtype, density=0.5)
            rows.allowed[torch.arange(N), rows.tokens.long()] = torch.arange(N, device="cuda") % 2 == 0
            rows.allow(rows.allowed)
            out = rows.run(ctx)
            a = backward(ctx, rows, out)
            check_gradient(rows, a, out["lse"], out["entropy"], *rows.d)
            rows.logits.masked_fill_(~rows.allowed, -INF)
            rows.mask = None
            b = backward(ctx, rows, out, *rows.d)
            assert torch.equal(a, b)
            alone = backward(ctx, rows, out, d_logp=rows.d[0])
            assert (alone[1::2] == 0).all() and (alone[::2] != 0).any(dim=1).all()


def test_gradient_of_sure_tokens():
    # 1 - p of 1e-4 to 1e-7: what a difference to 1 in 32 bits would lose
    N, V = 8, 5000
    with Ctx([]) as ctx:
        rows = Rows(N, V, torch.float32)
        rows.logits[torch.arange(N), rows.tokens.long()] = torch.linspace(20, 27, N, device="cuda")
        out = rows.run(ctx)
        d = torch.ones(N, device="cuda")
        got = backward(ctx, rows, out, d_logp=d)
        z = rows.scores()
        rest = -torch.expm1(z.gather(1, rows.tokens.long().unsqueeze(1)).squeeze(1) - torch.logsumexp(z, dim=1))
        of_token = got.gather(1, rows.tokens.long().unsqueeze(1)).squeeze(1).double()
        # lse was rounded to 2^-24 of itself: so much of d is in it
        assert ((of_token - rest).abs() <= out["lse"].double() * 2.0 ** -23 + rest * 1e-4).all()


def test_gradient_is_that_of_the_results():
    # against differences of the call's own results: logits of 32 bits, a small row, a step that 32 bits resolve
    N, V, h = 1, 37, 2.0 ** -7
    with Ctx([]) as ctx:
        rows = Rows(N, V, torch.float32, density=0.7)
        rows.allowed[:, rows.tokens.long()] = True
        rows.allow(rows.allowed)
        out = rows.run(ctx)
        d_logp, d_entropy = torch.tensor([0.8], device="cuda"), torch.tensor([-1.3], device="cuda")
        got = backward(ctx, rows, out, d_logp=d_logp, d_entropy=d_entropy)[0]
        for i in range(V):
            value = []
            for step in (h, -h):
                moved = Rows(N, V, torch.float32, density=0.7)
                moved.allowed[:, rows.tokens.long()] = True
                moved.allow(moved.allowed)
                moved.logits[0, i] += step
                o = moved.run(ctx)
                value.append((0.8 * o["logp"] - 1.3 * o["entropy"]).double().item())
            # a difference: third derivatives times h^2 / 6 (under 2^-14), results rounded by some 2^-21 each, over 2 h
            assert abs((value[0] - value[1]) / (2 * h) - got[i].item()) <= 6 * h * h + 8 * 2.0 ** -21 / (2 * h), i


def test_captured_calls_on_another_stream_and_two_at_once():
    with Ctx([]) as one, Ctx([]) as two:
        a, b = Rows(20, 32003, torch.bfloat16, density=0.3), Rows(600, 5000, torch.float32)
        streams = [torch.cuda.Stream() for _ in range(2)]
        want = []
        for ctx, rows in ((one, a), (two, b)):
            out = rows.run(ctx, 20)
            want.append((out, backward(ctx, rows, out)))
        torch.cuda.synchronize()
        graphs, results = [], []
        for ctx, rows, st, (out, d) in zip((one, two), (a, b), streams, want):
            o = {k: torch.zeros_like(v) for k, v in out.items()}
            to = torch.zeros((rows.N, rows.V), dtype=rows.dtype, device="cuda")
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                rows.run(ctx, 20, stream=st, out=o)
                cz.cfgzip_token_logprobs_backward(ctx.h, rows.logits, CODE[rows.dtype], rows.stride, rows.N, rows.V, rows.mask, rows.words,
                                                  rows.tokens, 1.0, o["lse"], o["entropy"], rows.d[0], rows.d[1], to, rows.V, st)
            graphs.append(g)
            results.append((o, to))
        for _ in range(3):
            for o, to in results:
                to.zero_()
                for v in o.values():
                    v.zero_()
            torch.cuda.synchronize()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            torch.cuda.synchronize()
            for (out, d), (o, to) in zip(want, results):
                assert all(torch.equal(out[k], o[k]) for k in out) and torch.equal(d, to)


@pytest.mark.parametrize("V", [2000, 50000])
def test_a_nearly_certain_token_keeps_what_the_others_have_together(V):
    """The sum is 1 and little: its logarithm is good to the bits of the little, not of the 1, where both are added up by different threads."""
    N, st = 3, torch.cuda.current_stream()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    z = torch.empty((N, V), device="cuda").normal_(generator=g)
    z[:, :8] = -math.inf
    z[:, 5] = torch.tensor([18.0, 21.5, 25.0], device="cuda")
    tokens = torch.full((N,), 5, dtype=torch.int32, device="cuda")
    logp, entropy, lse = (torch.zeros(N, device="cuda") for _ in range(3))
    with Ctx([]) as ctx:
        cz.cfgzip_token_logprobs(ctx.h, z, cz.F32, V, N, V, None, 0, tokens, 1.0, 0, logp, entropy, lse, None, None, st)
        torch.cuda.synchronize()
    want = torch.log_softmax(z.double(), dim=1)
    # the others' terms: 2^t with t of 45 at most, rounded once (2^-19 ln 2), a scale good to 2^-24 (45 times 2^-24 ln 2), an exponential
    # good to 2^-22, and additions of as many: together below 2^-18; of the entropy's terms t counts once more. 196 runs of 256 tokens are
    # dealt to 16 times 8 warps: one thread adds a second eight tokens to its sum of the certain one, half a step of a number up to sqrt(2)
    # (its sum of 2^t t, t up to 1/2, is smaller)
    second = 2.0 ** -24 if V > 2048 else 0.0
    assert ((logp - want[:, 5]).abs() <= 2.0 ** -17 * want[:, 5].abs() + second).all()
    want_entropy = torch.special.entr(want.exp()).sum(dim=1)
    assert ((entropy - want_entropy).abs() <= 2.0 ** -16 * want_entropy + 2 * second).all()
