"""Scoring answers and drafting them: what a program hands the library beside the decode step when it reports log probabilities, trains a
policy on answers that a grammar allows, or drafts tokens with a layer of its own in front of the head, as cases that can be timed.

Kinds of case
  logprobs            cfgzip_token_logprobs: logits to the log probabilities of given tokens, entropy, normaliser, top alternatives
  logprobs_backward   cfgzip_token_logprobs_backward: gradient of log probabilities and entropies with respect to the logits
  policy              cfgzip_head_logprobs and cfgzip_head_logprobs_backward: the same from hidden states, without the logits, and its
                      gradient with respect to the hidden states and the head
  layer               cfgzip_layer_forward: matrix product with bias, activation and residual (the layer in front of a head)
  layer_backward      cfgzip_layer_backward: its gradient with respect to the input, the weights and the bias

With `own` false every kind is computed in elementary torch operations in 32 bits; with `own` true by the library.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one request that asks for its tokens' log probabilities, logits as the decode step left them (masked in place)
        {"name": "logprobs-v32000-b1", "kind": "logprobs", "V": 32000, "N": 1, "dtype": "f32", "mask": "inplace", "top": 5, "t": 1.0},
        # a decode batch, twenty alternatives each
        {"name": "logprobs-v128256-b32-top20", "kind": "logprobs", "V": 128256, "N": 32, "dtype": "bf16", "mask": "inplace", "top": 20,
         "t": 0.7},
        # an answer scored under the grammar's masks; an odd vocabulary, so that rows start anywhere
        {"name": "logprobs-v100003-n1000", "kind": "logprobs", "V": 100003, "N": 1000, "dtype": "bf16", "mask": "bits", "top": 5, "t": 1.0},
        # a policy's update where the program has the logits in 32 bits
        {"name": "logprobs-backward-v50021-n500", "kind": "logprobs_backward", "V": 50021, "N": 500, "dtype": "f32", "mask": "bits",
         "t": 1.0},
        # a training batch of logits
        {"name": "logprobs-backward-v128256-n4096", "kind": "logprobs_backward", "V": 128256, "N": 4096, "dtype": "bf16", "mask": "none",
         "t": 1.0},
        # an update on a short answer of a small model
        {"name": "policy-v32000-h2048-n77", "kind": "policy", "V": 32000, "H": 2048, "N": 77, "masked": True},
        # an update on a training batch
        {"name": "policy-v128256-h4096-n4096", "kind": "policy", "V": 128256, "H": 4096, "N": 4096, "masked": True},
        # drafting a token for one request
        {"name": "layer-2048-b1", "kind": "layer", "rows": 1, "in": 2048, "out": 2048, "act": "silu", "bias": "bf16", "residual": True,
         "slope": False},
        # drafting for a batch
        {"name": "layer-4096-b32", "kind": "layer", "rows": 32, "in": 4096, "out": 4096, "act": "silu", "bias": "bf16", "residual": True,
         "slope": False},
        # training the layer, forward
        {"name": "layer-4096-n8192", "kind": "layer", "rows": 8192, "in": 4096, "out": 4096, "act": "silu", "bias": "f32",
         "residual": True, "slope": True},
        # ... and backward
        {"name": "layer-backward-4096-n8192", "kind": "layer_backward", "rows": 8192, "in": 4096, "out": 4096, "act": "silu",
         "bias": "f32", "residual": True},
        # a layer that widens, few tokens, odd sizes
        {"name": "layer-backward-1032-2568-n500", "kind": "layer_backward", "rows": 500, "in": 1032, "out": 2568, "act": "gelu",
         "bias": "bf16", "residual": False},
    ]


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw_one(rng)
        if _cost(case) <= most:
            return case


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _draw_one(rng):
    kind = rng.choice(("logprobs", "logprobs", "logprobs_backward", "policy", "layer", "layer", "layer_backward"))
    case = {"kind": kind}
    if kind in ("logprobs", "logprobs_backward"):
        case.update(V=_log_uniform(rng, 1000, 260000), N=_log_uniform(rng, 1, 4096), dtype=rng.choice(("bf16", "f32")),
                    mask=rng.choice(("none", "inplace", "bits")), t=rng.choice((1.0, 1.0, 0.7, 0.2)))
        if kind == "logprobs":
            case["top"] = rng.choice((0, 1, 5, 20, 32))
    elif kind == "policy":
        case.update(V=_log_uniform(rng, 8000, 200000), H=_log_uniform(rng, 32, 640) * 8, N=_log_uniform(rng, 1, 8192),
                    masked=rng.random() < 0.6)
    else:
        case.update(rows=_log_uniform(rng, 1, 16384), act=rng.choice(("none", "gelu", "gelu_tanh", "silu")),
                    bias=rng.choice(("none", "bf16", "f32")), residual=rng.random() < 0.5)
        case["in"], case["out"] = _log_uniform(rng, 32, 1024) * 8, _log_uniform(rng, 32, 1024) * 8
        if case["residual"] and (kind == "layer_backward" or rng.random() < 0.5):
            case["out"] = case["in"]  # the layer's own input
        if kind == "layer":
            case["slope"] = case["act"] != "none" and rng.random() < 0.5
    return case


def _words(n):
    return (n + 31) // 32


def work(case):
    """What a pass cannot do without: every input read once, every output written once."""
    kind = case["kind"]
    if kind in ("logprobs", "logprobs_backward"):
        N, V, size = case["N"], case["V"], 2 if case["dtype"] == "bf16" else 4
        mask = 4 * _words(V) * N if case["mask"] == "bits" else 0
        if kind == "logprobs":
            return {"bytes": float(N * V * size + mask + N * (16 + 8 * case["top"])), "flops": 5.0 * N * V}
        return {"bytes": float(2 * N * V * size + mask + 20 * N), "flops": 5.0 * N * V}
    if kind == "policy":
        V, H, N = case["V"], case["H"], case["N"]
        mask = N * 4 * _words(V) if case["masked"] else 0
        return {"bytes": 4.0 * V * H + 4.0 * N * H + mask + 24 * N, "flops": 6.0 * N * V * H}
    rows, K, O = case["rows"], case["in"], case["out"]
    bias = {"none": 0, "bf16": 2, "f32": 4}[case["bias"]] * O
    if kind == "layer":
        per = 2 + 2 * (case["residual"] and K != O) + 2 * case["slope"]
        return {"bytes": 2.0 * K * O + 2.0 * rows * K + per * rows * O + bias, "flops": 2.0 * rows * K * O}
    slope = 2 * (case["act"] != "none")
    return {"bytes": 4.0 * K * O + 4.0 * rows * K + (2.0 + slope) * rows * O + (4 * O if bias else 0), "flops": 4.0 * rows * K * O}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.4e15)


# ---------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------
class State:
    def __init__(self, case):
        self.case = case
        self.ctx = 0

    def __del__(self):
        if self.ctx:
            self.cz.cfgzip_destroy(self.ctx)


def _pack(bits):
    """Truth values [rows, n] as packed 32-bit words, lowest bit first."""
    rows, n = bits.shape
    padded = torch.zeros((rows, _words(n) * 32), dtype=torch.int32, device=bits.device)
    padded[:, :n] = bits
    shifts = torch.arange(32, device=bits.device, dtype=torch.int32)
    return (padded.view(rows, _words(n), 32) << shifts).sum(dim=2, dtype=torch.int32)


def _unpack(words, n):
    shifts = torch.arange(32, device=words.device, dtype=torch.int32)
    return ((words.unsqueeze(2) >> shifts) & 1).view(words.shape[0], -1)[:, :n] != 0


def _states(case, targets, gen):
    """A few grammar states, met again and again along the text; the token that follows is always allowed."""
    V, N = case["V"], len(targets)
    states = torch.rand((16, V), generator=gen, device="cuda") < torch.rand((16, 1), generator=gen, device="cuda")
    mask = _pack(states)[torch.randint(0, 16, (N,), generator=gen, device="cuda")]
    word, bit = (targets >> 5).long().unsqueeze(1), (1 << (targets & 31)).unsqueeze(1).to(torch.int32)
    return mask.scatter_(1, word, mask.gather(1, word) | bit)


def prepare(case, seed):
    s = State(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] in ("logprobs", "logprobs_backward"):
        _prepare_logits(s, case, gen)
    elif case["kind"] == "policy":
        _prepare_policy(s, case, gen)
    else:
        _prepare_layer(s, case, gen)
    if own:
        _prepare_own(s, case)
    return s


def _prepare_logits(s, case, gen):
    V, N = case["V"], case["N"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s.tokens = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    mask = None if case["mask"] == "none" else _states(case, s.tokens, gen)
    s.logits = torch.empty((N, V), dtype=dtype, device="cuda").normal_(0.0, 2.0, generator=gen)
    # about half of the given tokens are ones that the model is fairly sure of
    sure = 14.0 * (torch.rand((N, 1), generator=gen, device="cuda") < 0.5)
    s.logits.scatter_add_(1, s.tokens.long().unsqueeze(1), sure.to(dtype))
    s.vocab_mask = None
    if case["mask"] == "inplace":  # as the decode step leaves them
        for z, m in zip(s.logits.split(256), mask.split(256)):
            z.masked_fill_(~_unpack(m, V), float("-inf"))
    elif case["mask"] == "bits":
        s.vocab_mask = mask
    if case["kind"] == "logprobs":
        top = case["top"]
        s.logp, s.entropy, s.lse = (torch.zeros(N, dtype=torch.float32, device="cuda") for _ in range(3))
        s.top_tokens = torch.zeros((N, top), dtype=torch.int32, device="cuda") if top else None
        s.top_logp = torch.zeros((N, top), dtype=torch.float32, device="cuda") if top else None
        return
    s.tokens[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1  # the prompt and the padding
    s.d_logp = torch.empty(N, dtype=torch.float32, device="cuda").normal_(0.0, 1.0 / N, generator=gen)  # advantages
    s.d_entropy = torch.full((N,), -0.01 / N, dtype=torch.float32, device="cuda")
    s.lse, s.entropy = (torch.empty(N, dtype=torch.float32, device="cuda") for _ in range(2))  # what the forward pass left
    for lo in range(0, N, 256):
        z = _exact_logits(s, lo, lo + 256)
        s.lse[lo:lo + 256] = torch.logsumexp(z, dim=1)
        p = torch.softmax(z, dim=1)
        s.entropy[lo:lo + 256] = -(p * torch.log(p.clamp(min=1e-300))).sum(dim=1)
    s.d_logits = torch.zeros_like(s.logits)


def _prepare_policy(s, case, gen):
    V, H, N = case["V"], case["H"], case["N"]
    s.weight = torch.empty((V, H), dtype=torch.bfloat16, device="cuda").normal_(0.0, H ** -0.5, generator=gen)
    s.tokens = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    s.hidden = torch.empty((N, H), dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=gen)
    sure = 14.0 * (torch.rand((N, 1), generator=gen, device="cuda") < 0.5)
    for x, t, f in zip(s.hidden.split(2048), s.tokens.split(2048), sure.split(2048)):
        x.copy_(x.float() + f * s.weight[t.long()].float())
    s.vocab_mask = _states(case, s.tokens, gen) if case["masked"] else None
    s.tokens[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1
    s.d_logp = torch.empty(N, dtype=torch.float32, device="cuda").normal_(0.0, 1.0 / N, generator=gen)
    s.d_entropy = torch.full((N,), -0.01 / N, dtype=torch.float32, device="cuda")
    s.logp, s.entropy, s.lse = (torch.zeros(N, dtype=torch.float32, device="cuda") for _ in range(3))
    s.d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
    s.d_weight = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")


def _prepare_layer(s, case, gen):
    rows, K, O = case["rows"], case["in"], case["out"]
    s.weight = torch.empty((O, K), dtype=torch.bfloat16, device="cuda").normal_(0.0, K ** -0.5, generator=gen)
    s.x = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
    s.bias = None
    if case["bias"] != "none":
        s.bias = torch.empty(O, device="cuda").normal_(0.0, 0.5, generator=gen)
        s.bias = s.bias.to(torch.bfloat16) if case["bias"] == "bf16" else s.bias
    if case["kind"] == "layer":
        s.residual = None
        if case["residual"]:  # the layer's own input where it has the size, else another branch's output
            s.residual = s.x if K == O else torch.empty((rows, O), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
        s.y = torch.zeros((rows, O), dtype=torch.bfloat16, device="cuda")
        s.slope = torch.zeros_like(s.y) if case["slope"] else None
        return
    s.d_y = torch.empty((rows, O), dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
    s.slope = None
    if case["act"] != "none":  # what the forward pass left
        s.slope = torch.cat([_activation(case["act"], _pre(s, x))[1].to(torch.bfloat16) for x in s.x.split(2048)])
    s.d_x = torch.zeros_like(s.x)
    s.d_weight = torch.zeros_like(s.weight)
    s.d_bias = None if s.bias is None else torch.zeros(O, dtype=torch.float32, device="cuda")


def _prepare_own(s, case):
    """What the program keeps from call to call: a context, descriptions of the head and the layer, workspaces."""
    from paper_2605_29986_b200 import binding as cz
    s.cz = cz
    s.ctx = cz.cfgzip_create(torch.cuda.current_device())
    s.stream = torch.cuda.current_stream().cuda_stream
    kind, size = case["kind"], 0
    if kind == "policy":
        s.head = cz.cfgzip_head(s.weight, cz.BF16, case["V"], case["H"])
        size = max(cz.cfgzip_head_workspace(s.head, op, case["N"]) for op in (cz.HEAD_LOGPROBS, cz.HEAD_LOGPROBS_BACKWARD))
    elif kind in ("layer", "layer_backward"):
        act = {"none": cz.ACT_NONE, "gelu": cz.ACT_GELU, "gelu_tanh": cz.ACT_GELU_TANH, "silu": cz.ACT_SILU}[case["act"]]
        s.layer = cz.cfgzip_layer(s.weight, case["in"], case["out"], activation=act, bias=s.bias,
                                  bias_dtype=cz.BF16 if case["bias"] == "bf16" else cz.F32)
        size = cz.cfgzip_layer_workspace(s.layer, cz.LAYER_FORWARD if kind == "layer" else cz.LAYER_BACKWARD, case["rows"])
    s.workspace = torch.empty(size, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------
def run(s):
    return (_OWN if own else _PLAIN)[s.case["kind"]](s)


def _rows_of(s, lo, hi):
    """Tempered logits of the rows [lo, hi) in 32 bits, -inf where a token is not allowed."""
    z = s.logits[lo:hi].float()
    if s.vocab_mask is not None:
        z = z.masked_fill(~_unpack(s.vocab_mask[lo:hi], s.case["V"]), float("-inf"))
    return z * (1.0 / s.case["t"])


def _statistics(z):
    """Normaliser, entropy and log probabilities of rows of scores."""
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    logp = (z - top) - torch.log(total)
    entropy = -(e / total * logp.clamp(min=-1e30)).sum(dim=1)
    return (top + torch.log(total)).squeeze(1), entropy, logp


def _of_tokens(logp, t):
    return torch.where(t >= 0, logp.gather(1, t.long().clamp(min=0).unsqueeze(1)).squeeze(1), 0.0)


def _ordered(z):
    """Numbers as whole ones in the same order (both zeros alike), the lower index first among equal ones."""
    bits = (z + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return bits * 2 ** 21 - torch.arange(z.shape[1], device=z.device)


def _plain_logprobs(s):
    out = [[] for _ in range(5)]
    n = s.case["top"]
    for lo in range(0, s.case["N"], 256):
        z = _rows_of(s, lo, lo + 256)
        lse, entropy, logp = _statistics(z)
        out[0].append(_of_tokens(logp, s.tokens[lo:lo + 256]))
        out[1].append(entropy)
        out[2].append(lse)
        if n:
            raw = s.logits[lo:lo + 256].float().masked_fill(z == float("-inf"), float("-inf"))
            top = torch.topk(_ordered(raw), n, dim=1)[1]
            of_top = logp.gather(1, top)
            out[3].append(torch.where(of_top > float("-inf"), top, -1).to(torch.int32))
            out[4].append(of_top)
    return [torch.cat(o) if o else None for o in out]


def _logit_gradient(logp, entropy, t, d_logp, d_entropy):
    p = torch.exp(logp)
    d = torch.where(t >= 0, d_logp, 0.0).unsqueeze(1)
    g = -p * (d + d_entropy.unsqueeze(1) * (logp.clamp(min=-1e30) + entropy.unsqueeze(1)))
    return g.scatter_add_(1, t.long().clamp(min=0).unsqueeze(1), d)


def _plain_logprobs_backward(s):
    out = []
    for lo in range(0, s.case["N"], 256):
        hi = lo + 256
        logp = _rows_of(s, lo, hi) - s.lse[lo:hi].unsqueeze(1)
        g = _logit_gradient(logp, s.entropy[lo:hi], s.tokens[lo:hi], s.d_logp[lo:hi], s.d_entropy[lo:hi])
        out.append((g * (1.0 / s.case["t"])).to(s.logits.dtype))
    return torch.cat(out)


def _plain_policy(s):
    V, w = s.case["V"], s.weight.float()
    out, d_weight = [[] for _ in range(4)], torch.zeros_like(w)
    for lo in range(0, s.case["N"], 1024):
        x, t = s.hidden[lo:lo + 1024].float(), s.tokens[lo:lo + 1024]
        z = x @ w.T
        if s.vocab_mask is not None:
            z = z.masked_fill(~_unpack(s.vocab_mask[lo:lo + 1024], V), float("-inf"))
        lse, entropy, logp = _statistics(z)
        g = _logit_gradient(logp, entropy, t, s.d_logp[lo:lo + 1024], s.d_entropy[lo:lo + 1024])
        for o, v in zip(out, (_of_tokens(logp, t), entropy, lse, (g @ w).to(torch.bfloat16))):
            o.append(v)
        d_weight += g.T @ x
    return [torch.cat(o) for o in out] + [d_weight.to(torch.bfloat16)]


def _pre(s, x):
    """What the activation is given."""
    h = x.float() @ s.weight.float().T
    return h if s.bias is None else h + s.bias.float()


def _activation(act, h):
    """The activation and its derivative."""
    if act == "none":
        return h, torch.ones_like(h)
    if act == "silu":
        q = 1.0 / (1.0 + torch.exp(-h))
        return h * q, q * (1.0 + h * (1.0 - q))
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(h * math.sqrt(0.5)))
        return h * phi, phi + h * torch.exp(-0.5 * h * h) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (h + 0.044715 * h * h * h))
    return 0.5 * h * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * h * (1.0 - th * th) * c * (1.0 + 3.0 * 0.044715 * h * h)


def _plain_layer(s):
    ys, slopes = [], []
    for lo in range(0, s.case["rows"], 4096):
        y, slope = _activation(s.case["act"], _pre(s, s.x[lo:lo + 4096]))
        if s.residual is not None:
            y = y + s.residual[lo:lo + 4096].float()
        ys.append(y.to(torch.bfloat16))
        if s.slope is not None:
            slopes.append(slope.to(torch.bfloat16))
    return [torch.cat(ys), torch.cat(slopes) if slopes else None]


def _plain_layer_backward(s):
    d_y = s.d_y.float()
    g = d_y if s.slope is None else d_y * s.slope.float()
    d_x = g @ s.weight.float()
    if s.case["residual"] and s.case["in"] == s.case["out"]:
        d_x = d_x + d_y
    return [d_x.to(torch.bfloat16), (g.T @ s.x.float()).to(torch.bfloat16), None if s.bias is None else g.sum(dim=0)]


def _own_logprobs(s):
    c = s.case
    s.cz.cfgzip_token_logprobs(s.ctx, s.logits, s.cz.BF16 if c["dtype"] == "bf16" else s.cz.F32, c["V"], c["N"], c["V"], s.vocab_mask,
                               _words(c["V"]), s.tokens, 1.0 / c["t"], c["top"], s.logp, s.entropy, s.lse, s.top_tokens, s.top_logp,
                               s.stream)
    return [s.logp, s.entropy, s.lse, s.top_tokens, s.top_logp]


def _own_logprobs_backward(s):
    c = s.case
    s.cz.cfgzip_token_logprobs_backward(s.ctx, s.logits, s.cz.BF16 if c["dtype"] == "bf16" else s.cz.F32, c["V"], c["N"], c["V"],
                                        s.vocab_mask, _words(c["V"]), s.tokens, 1.0 / c["t"], s.lse, s.entropy, s.d_logp, s.d_entropy,
                                        s.d_logits, c["V"], s.stream)
    return s.d_logits


def _own_policy(s):
    c, cz, size = s.case, s.cz, s.workspace.numel()
    cz.cfgzip_head_logprobs(s.ctx, s.head, s.hidden, c["H"], c["N"], s.vocab_mask, _words(c["V"]), s.tokens, s.logp, s.entropy, s.lse,
                            s.workspace, size, s.stream)
    cz.cfgzip_head_logprobs_backward(s.ctx, s.head, s.hidden, c["H"], c["N"], s.vocab_mask, _words(c["V"]), s.tokens, s.lse, s.entropy,
                                     s.d_logp, s.d_entropy, s.d_hidden, c["H"], s.d_weight, cz.BF16, c["H"], 0, s.workspace, size,
                                     s.stream)
    return [s.logp, s.entropy, s.lse, s.d_hidden, s.d_weight]


def _own_layer(s):
    c = s.case
    s.cz.cfgzip_layer_forward(s.ctx, s.layer, s.x, c["in"], c["rows"], s.residual, c["out"], s.y, c["out"], s.slope, c["out"],
                              s.workspace, s.workspace.numel(), s.stream)
    return [s.y, s.slope]


def _own_layer_backward(s):
    c = s.case
    through = s.d_y if c["residual"] and c["in"] == c["out"] else None  # the gradient that went past the layer
    s.cz.cfgzip_layer_backward(s.ctx, s.layer, s.x, c["in"], c["rows"], s.slope, c["out"], s.d_y, c["out"], through, c["in"], s.d_x,
                               c["in"], s.d_weight, s.cz.BF16, c["in"], s.d_bias, 0, s.workspace, s.workspace.numel(), s.stream)
    return [s.d_x, s.d_weight, s.d_bias]


_PLAIN = {"logprobs": _plain_logprobs, "logprobs_backward": _plain_logprobs_backward, "policy": _plain_policy, "layer": _plain_layer,
          "layer_backward": _plain_layer_backward}
_OWN = {"logprobs": _own_logprobs, "logprobs_backward": _own_logprobs_backward, "policy": _own_policy, "layer": _own_layer,
        "layer_backward": _own_layer_backward}


# ---------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "logprobs_backward": _exact_logprobs_backward, "policy": _exact_policy, "layer": _exact_layer,
            "layer_backward": _exact_layer_backward}[case["kind"]](s)


def _exact_allowed(s, lo, hi):
    t = torch.arange(s.case["V"], device="cuda")
    return (s.vocab_mask[lo:hi][:, t // 32] >> (t % 32).int()) & 1 == 1


def _exact_logits(s, lo, hi):
    z = s.logits[lo:hi].double() / s.case["t"]
    return z if s.vocab_mask is None else torch.where(_exact_allowed(s, lo, hi), z, -float("inf"))


def _exact_entropy(z):
    p = torch.softmax(z, dim=1)
    return torch.special.entr(p).sum(dim=1)


def _exact_pick(z, lse, t):
    rows = torch.arange(len(t), device="cuda")
    return torch.where(t < 0, 0.0, z[rows, t.long().clamp(min=0)] - lse)


def _exact_logprobs(s):
    out, n = [[] for _ in range(5)], s.case["top"]
    for lo in range(0, s.case["N"], 128):
        z = _exact_logits(s, lo, lo + 128)
        lse = torch.logsumexp(z, dim=1)
        out[0].append(_exact_pick(z, lse, s.tokens[lo:lo + 128]))
        out[1].append(_exact_entropy(z))
        out[2].append(lse)
        if n:
            values, order = torch.sort(z, dim=1, descending=True, stable=True)
            values, order = values[:, :n], order[:, :n]
            out[3].append(torch.where(values == -float("inf"), -1, order).to(torch.int32))
            out[4].append(values - lse.unsqueeze(1))
    return [torch.cat(o) if o else None for o in out]


def _exact_gradient(z, lse, entropy, t, d_logp, d_entropy):
    p = torch.exp(z - lse.unsqueeze(1))
    d = torch.where(t < 0, 0.0, d_logp.double())
    # d/dz of -sum p log p is -p (log p + entropy)
    g = d_entropy.double().unsqueeze(1) * (torch.special.entr(p) - p * entropy.unsqueeze(1)) - d.unsqueeze(1) * p
    has = (t >= 0).nonzero().squeeze(1)
    g[has, t[has].long()] += d[has]
    return g


def _exact_logprobs_backward(s):
    out = []
    for lo in range(0, s.case["N"], 128):
        hi = lo + 128
        g = _exact_gradient(_exact_logits(s, lo, hi), s.lse[lo:hi].double(), s.entropy[lo:hi].double(), s.tokens[lo:hi], s.d_logp[lo:hi],
                            s.d_entropy[lo:hi])
        out.append((g / s.case["t"]).to(torch.float32))  # (64 bits of all of them would not fit)
    return torch.cat(out)


def _exact_policy(s):
    V, H, N = s.case["V"], s.case["H"], s.case["N"]
    out, d_weight = [[] for _ in range(4)], torch.zeros((V, H), dtype=torch.float64, device="cuda")
    for lo in range(0, N, 512):
        x, t = s.hidden[lo:lo + 512].double(), s.tokens[lo:lo + 512]
        z = torch.cat([x @ s.weight[v:v + 16384].double().T for v in range(0, V, 16384)], dim=1)
        if s.vocab_mask is not None:
            z = torch.where(_exact_allowed(s, lo, lo + 512), z, -float("inf"))
        lse, entropy = torch.logsumexp(z, dim=1), _exact_entropy(z)
        g = _exact_gradient(z, lse, entropy, t, s.d_logp[lo:lo + 512], s.d_entropy[lo:lo + 512])
        d_x = torch.zeros_like(x)
        for v in range(0, V, 16384):
            d_x += g[:, v:v + 16384] @ s.weight[v:v + 16384].double()
            d_weight[v:v + 16384] += g[:, v:v + 16384].T @ x
        for o, value in zip(out, (_exact_pick(z, lse, t), entropy, lse, d_x)):
            o.append(value)
    return [torch.cat(o) for o in out] + [d_weight]


def _exact_layer(s):
    act, ys, slopes = s.case["act"], [], []
    for lo in range(0, s.case["rows"], 2048):
        h = s.x[lo:lo + 2048].double() @ s.weight.double().T + (0.0 if s.bias is None else s.bias.double())
        if act == "silu":
            y, slope = torch.nn.functional.silu(h), torch.sigmoid(h) + h * torch.sigmoid(h) * torch.sigmoid(-h)
        elif act == "gelu":
            y = h * torch.special.ndtr(h)
            slope = torch.special.ndtr(h) + h * torch.exp(-h * h / 2) / (2 * math.pi) ** 0.5
        elif act == "gelu_tanh":
            u = (2 / math.pi) ** 0.5 * (h + 0.044715 * h ** 3)
            y = h * torch.sigmoid(2 * u)  # (1 + tanh u) / 2 is the logistic function of 2 u
            slope = torch.sigmoid(2 * u) + h * torch.sigmoid(2 * u) * torch.sigmoid(-2 * u) * 2 * (2 / math.pi) ** 0.5 * (
                1 + 3 * 0.044715 * h ** 2)
        else:
            y, slope = h, torch.ones_like(h)
        ys.append(y if s.residual is None else y + s.residual[lo:lo + 2048].double())
        slopes.append(slope)
    return [torch.cat(ys), torch.cat(slopes) if s.slope is not None else None]


def _exact_layer_backward(s):
    g = s.d_y.double() * (1.0 if s.slope is None else s.slope.double())
    d_x = g @ s.weight.double()
    if s.case["residual"] and s.case["in"] == s.case["out"]:
        d_x += s.d_y.double()
    return [d_x, g.T @ s.x.double(), None if s.bias is None else g.sum(dim=0)]
