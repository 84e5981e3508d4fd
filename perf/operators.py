"""The head of a language model under a grammar: what a program hands the library when it decodes from hidden states, trains on
answers that a grammar allows, or keeps the head in 4 bits, as cases that can be timed.

Kinds of case
  step      cfgzip_head_step: hidden states to the next token (product with the head, class masks, normaliser, greedy choice,
            representative), with the masked logits where the program samples by itself
  loss      cfgzip_head_loss: cross entropy over the allowed tokens, per token of a text, without the logits
  backward  cfgzip_head_loss_backward: its gradient with respect to the hidden states and the head
  quantize  cfgzip_head_quantize and cfgzip_head_dequantize: the head to microscaled 4 bits, and the values it then stands for

With `own` false every kind is computed in elementary torch operations in 32 bits; with `own` true by the library.
"""
import torch

own = False


# ---------------------------------------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one request, a small model: nothing but latency
        {"name": "step-v32000-h2048-b1", "kind": "step", "V": 32000, "H": 2048, "K": 256, "B": 1, "head": "bf16", "density": 0.3},
        # the batch the decode step is usually quoted on: together the rows allow nearly all of the vocabulary
        {"name": "step-v128256-h4096-b32", "kind": "step", "V": 128256, "H": 4096, "K": 2048, "B": 32, "head": "bf16",
         "density": 0.1},
        # structural characters and keywords only: hardly any row of the head has to be read
        {"name": "step-v128256-h4096-b8-few", "kind": "step", "V": 128256, "H": 4096, "K": 512, "B": 8, "head": "bf16",
         "density": 0.1, "classes": 5},
        # a program with a sampler of its own takes the masked logits; an odd vocabulary, a batch that is no power of two
        {"name": "step-v100003-h2560-b48-logits", "kind": "step", "V": 100003, "H": 2560, "K": 1500, "B": 48, "head": "bf16",
         "density": 0.2, "logits": "f32"},
        # the same head in 4 bits
        {"name": "step-mx-v128256-h4096-b32", "kind": "step", "V": 128256, "H": 4096, "K": 2048, "B": 32, "head": "mxfp4",
         "density": 0.1},
        # one request on a 4-bit head, as on a desk
        {"name": "step-mx-v151936-h2560-b1", "kind": "step", "V": 151936, "H": 2560, "K": 4096, "B": 1, "head": "mxfp4",
         "density": 0.9},
        # the log-probability of a short answer
        {"name": "loss-v32000-h2048-n77", "kind": "loss", "V": 32000, "H": 2048, "N": 77, "masked": True},
        # a training batch: one sequence of 8192, or several packed ones
        {"name": "loss-v128256-h4096-n8192", "kind": "loss", "V": 128256, "H": 4096, "N": 8192, "masked": True},
        # fine-tuning a small model on a short packed batch, odd sizes, no grammar
        {"name": "backward-v50021-h1024-n1000", "kind": "backward", "V": 50021, "H": 1024, "N": 1000, "masked": False},
        # a training batch under a grammar
        {"name": "backward-v128256-h4096-n4096", "kind": "backward", "V": 128256, "H": 4096, "N": 4096, "masked": True},
        # a small head after an update, from its 32-bit master copy
        {"name": "quantize-f32-v32000-h2048", "kind": "quantize", "V": 32000, "H": 2048, "from": "f32"},
        # a large head when it is loaded
        {"name": "quantize-bf16-v128256-h4096", "kind": "quantize", "V": 128256, "H": 4096, "from": "bf16"},
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
    kind = rng.choice(("step", "step", "step", "loss", "backward", "quantize"))
    V = _log_uniform(rng, 8000, 200000)
    H = _log_uniform(rng, 8, 160) * 32  # 256 to 5120, in scale blocks
    case = {"kind": kind, "V": V, "H": H}
    if kind == "step":
        case["B"] = _log_uniform(rng, 1, 256)
        case["K"] = min(_log_uniform(rng, 256, 16384), V // 8)
        case["head"] = rng.choice(("bf16", "mxfp4"))
        case["density"] = rng.choice((0.0, 0.01, 0.1, 0.3, 0.9))
        if rng.random() < 0.25:
            case["classes"] = rng.randint(1, 8)
        if rng.random() < 0.25:
            case["logits"] = rng.choice(("bf16", "f32"))
    elif kind == "quantize":
        case["from"] = rng.choice(("bf16", "f32"))
    else:
        case["N"] = _log_uniform(rng, 1, 8192)
        case["masked"] = rng.random() < 0.6
    return case


def _words(n):
    return (n + 31) // 32


def work(case):
    """What a pass cannot do without: every input read once, every output written once. Rows of the head that no row of the
    batch allows need not be read; the token -> class vector counts as 16 bits per token."""
    V, H, kind = case["V"], case["H"], case["kind"]
    if kind == "quantize":
        return {"bytes": float(V * H) * ((4 if case["from"] == "f32" else 2) + 0.5 + 1 / 32 + 2), "flops": 3.0 * V * H}
    if kind == "step":
        B, K = case["B"], case["K"]
        if "classes" in case:
            row = min(1.0, 0.5 * (1 + case["classes"]) / K)
        else:
            row = case["density"]
        union = 1.0 - (1.0 - row) ** B if row else B / (B + 1.0)  # (densities of their own: uniform on (0, 1))
        per_weight = 2.0 if case["head"] == "bf16" else 0.5 + 1 / 32
        out = B * (4 * _words(V) + 16) + B * V * {"f32": 4, "bf16": 2}.get(case.get("logits"), 0)
        return {"bytes": union * V * H * per_weight + 2.0 * B * H + 2 * V + B * 4 * _words(K) + out,
                "flops": 2.0 * B * H * V * union}
    N = case["N"]
    masks = N * 4 * _words(V) if case["masked"] else 0
    if kind == "loss":
        return {"bytes": 2.0 * V * H + 2.0 * N * H + masks + 12 * N, "flops": 2.0 * N * V * H}
    return {"bytes": 4.0 * V * H + 4.0 * N * H + masks + 12 * N, "flops": 6.0 * N * V * H}


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


def _partition(V, K, gen):
    """Class sizes by Zipf's law, members scattered over the vocabulary, lowest token id as representative."""
    w = torch.arange(1, K + 1, dtype=torch.float64) ** -1.1
    sizes = 1 + torch.floor(w / w.sum() * (V - K)).to(torch.int64)
    sizes[: V - int(sizes.sum())] += 1
    c = torch.empty(V, dtype=torch.int64)
    c[torch.randperm(V, generator=gen)] = torch.repeat_interleave(torch.arange(K), sizes)
    r = torch.full((K,), V, dtype=torch.int64).scatter_reduce(0, c, torch.arange(V), "amin")
    return c.to(torch.int32), r.to(torch.int32)


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


def _class_bits(case, gen):
    B, K = case["B"], case["K"]
    u = torch.rand((B, K), generator=gen, device="cuda")
    if "classes" in case:
        n = torch.randint(1, case["classes"] + 1, (B, 1), generator=gen, device="cuda")
        return u.argsort(dim=1).argsort(dim=1) < n
    bits = u < (case["density"] or torch.rand((B, 1), generator=gen, device="cuda"))
    bits[:, 0] |= ~bits.any(dim=1)  # the engine never leaves a row without a class
    return bits


def _weights(V, H, gen, dtype=torch.bfloat16):
    return torch.empty((V, H), dtype=dtype, device="cuda").normal_(0.0, H ** -0.5, generator=gen)


def _hidden(w, rows, gen):
    """Hidden states of a trained model: noise that gives every token a logit of deviation 2, and a part that points at the
    token to come."""
    x = torch.empty((w.shape[0], w.shape[1]), dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=gen)
    return (x + rows * w).to(torch.bfloat16)


def prepare(case, seed):
    s = State(case)
    V, H = case["V"], case["H"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "quantize":
        s.weight = _weights(V, H, gen, torch.float32 if case["from"] == "f32" else torch.bfloat16)
        s.weight *= torch.rand((V, 1), generator=gen, device="cuda") + 0.5  # rows differ in size
        s.packed = torch.zeros((V, H // 2), dtype=torch.uint8, device="cuda")
        s.scales = torch.zeros((V, (H // 32 + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
        s.values = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    elif case["kind"] == "step":
        _prepare_step(s, case, gen, seed)
    else:
        _prepare_text(s, case, gen)
    if own:
        _prepare_own(s, case)
    return s


def _prepare_step(s, case, gen, seed):
    V, H, B, K = case["V"], case["H"], case["B"], case["K"]
    host = torch.Generator()
    host.manual_seed(seed)
    s.c, s.r = _partition(V, K, host)
    s.c_dev, s.r_dev = s.c.cuda(), s.r.cuda()
    bits = _class_bits(case, gen)
    s.class_mask = _pack(bits)
    s.weight = _weights(V, H, gen)
    if case["head"] == "mxfp4":
        s.packed, s.scales, values = [], [], []
        for part in s.weight.split(16384):
            p, e, v = _quantize(part)
            s.packed.append(p)
            s.scales.append(e)
            values.append(v)
        s.packed, s.weight = torch.cat(s.packed), torch.cat(values)
        s.scales = torch.nn.functional.pad(torch.cat(s.scales), (0, -(H // 32) % 16)).contiguous()
    # the token to come: one the row allows
    allowed = bits[:, s.c_dev.long()]
    first = torch.rand((B, V), generator=gen, device="cuda").masked_fill_(~allowed, -1.0).argmax(dim=1)
    # ... about as likely as all the others together
    sure = torch.log(allowed.sum(dim=1, keepdim=True).float()) + 2.0 + torch.randn((B, 1), generator=gen, device="cuda")
    s.hidden = _hidden(s.weight[first].float(), sure, gen)
    if case["head"] == "mxfp4":
        s.weight = None
    s.vocab_mask = torch.zeros((B, _words(V)), dtype=torch.int32, device="cuda")
    s.token, s.rep = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    s.logp, s.lse = (torch.zeros(B, dtype=torch.float32, device="cuda") for _ in range(2))
    s.logits = None
    if "logits" in case:
        s.logits = torch.zeros((B, V), dtype=torch.float32 if case["logits"] == "f32" else torch.bfloat16, device="cuda")


def _prepare_text(s, case, gen):
    V, H, N = case["V"], case["H"], case["N"]
    s.weight = _weights(V, H, gen)
    s.targets = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    # a model that is being trained is about right about half of the tokens
    sure = 14.0 * (torch.rand((N, 1), generator=gen, device="cuda") < 0.5)
    s.hidden = torch.cat([_hidden(s.weight[t.long()].float(), f, gen) for t, f in zip(s.targets.split(2048), sure.split(2048))])
    s.vocab_mask = None
    if case["masked"]:
        # a few grammar states, met again and again along the text; the token that follows is always allowed
        states = torch.rand((16, V), generator=gen, device="cuda") < torch.rand((16, 1), generator=gen, device="cuda")
        s.vocab_mask = _pack(states)[torch.randint(0, 16, (N,), generator=gen, device="cuda")]
        word, bit = (s.targets >> 5).long().unsqueeze(1), (1 << (s.targets & 31)).unsqueeze(1).to(torch.int32)
        s.vocab_mask.scatter_(1, word, s.vocab_mask.gather(1, word) | bit)
    s.targets[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1  # the prompt and the padding have no loss
    s.loss, s.lse = (torch.zeros(N, dtype=torch.float32, device="cuda") for _ in range(2))
    if case["kind"] == "backward":
        s.d_loss = torch.full((N,), 1.0 / N, dtype=torch.float32, device="cuda")
        s.lse = torch.empty(N, dtype=torch.float32, device="cuda")  # what the forward pass left
        for rows, out, mask in _row_pieces(s, 1024):
            z = _masked(rows.float() @ s.weight.float().T, mask, V)
            out.copy_(torch.logsumexp(z.double(), dim=1))
        s.d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        s.d_weight = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")


def _prepare_own(s, case):
    """What the program keeps from call to call: a context with the partition loaded, the head's description, workspaces."""
    from paper_2605_29986_b200 import binding as cz
    s.cz = cz
    s.ctx = cz.cfgzip_create(torch.cuda.current_device())
    s.stream = torch.cuda.current_stream().cuda_stream
    V, H, kind = case["V"], case["H"], case["kind"]
    if kind == "quantize" or case.get("head") == "mxfp4":
        s.head = cz.cfgzip_head(s.packed, cz.MXFP4, V, H, scales=s.scales, scale_stride=s.scales.shape[1])
    else:
        s.head = cz.cfgzip_head(s.weight, cz.BF16, V, H)
    if kind == "step":
        s.part = cz.cfgzip_load_partition(s.ctx, s.c.numpy(), V, s.r.numpy(), case["K"], s.stream)
        rows, op = case["B"], cz.HEAD_STEP
    elif kind != "quantize":
        rows, op = case["N"], cz.HEAD_LOSS if kind == "loss" else cz.HEAD_LOSS_BACKWARD
    else:
        return
    s.workspace = torch.empty(cz.cfgzip_head_workspace(s.head, op, rows), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------
def run(s):
    return (_OWN if own else _PLAIN)[s.case["kind"]](s)


def _masked(z, mask, V):
    return z if mask is None else z.masked_fill(~_unpack(mask, V), float("-inf"))


def _row_pieces(s, n):
    """Hidden states, the rows' results and their masks, n rows at a time."""
    masks = s.vocab_mask.split(n) if s.vocab_mask is not None else [None] * len(s.hidden.split(n))
    return zip(s.hidden.split(n), s.lse.split(n), masks)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantize(w):
    """Blocks of 32 along the rows: a power of two that brings the largest to the top octave of e2m1, and the nearest of the
    sixteen values (ties to the even code). Packed codes (the lower half of a byte first), exponents + 127, values."""
    V, H = w.shape
    x = w.float().view(V, H // 32, 32)
    e = torch.frexp(x.abs().amax(dim=2))[1] - 3
    e = torch.where(x.abs().amax(dim=2) > 0, e, -127).clamp(min=-127)
    q = torch.ldexp(x, -e.unsqueeze(2))
    a = q.abs()
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    value = torch.tensor(_E2M1, device=w.device)[code.long()] * torch.where(torch.signbit(q), -1.0, 1.0)
    code |= torch.signbit(q).to(torch.uint8) << 3
    code = code.view(V, H)
    values = torch.ldexp(value, e.unsqueeze(2)).view(V, H).to(torch.bfloat16)
    return code[:, ::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8), values


def _dequantized(packed, scales, H):
    code = torch.stack([packed & 15, packed >> 4], dim=2).view(packed.shape[0], H)
    value = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=packed.device)[code.int()]
    scales = scales[:, : H // 32].int() - 127
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales)
    return (value.view(-1, H // 32, 32) * scale.unsqueeze(2)).view(-1, H)


def _plain_step(s):
    V, H = s.case["V"], s.case["H"]
    allowed = _unpack(s.class_mask, s.case["K"])[:, s.c_dev.long()]
    w = s.weight.float() if s.weight is not None else _dequantized(s.packed, s.scales, H)
    z = (s.hidden.float() @ w.T).masked_fill(~allowed, float("-inf"))
    top, token = z.max(dim=1)
    log_sum = torch.log(torch.exp(z - top.unsqueeze(1)).sum(dim=1))
    rep = s.r_dev[s.c_dev[token].long()]
    logits = None if s.logits is None else z.to(s.logits.dtype)
    return [_pack(allowed), logits, token.to(torch.int32), rep, -log_sum, top + log_sum]


def _plain_loss(s):
    V, w = s.case["V"], s.weight.float()
    losses, lses = [], []
    for (x, _, mask), t in zip(_row_pieces(s, 1024), s.targets.split(1024)):
        z = _masked(x.float() @ w.T, mask, V)
        top = z.amax(dim=1)
        log_sum = torch.log(torch.exp(z - top.unsqueeze(1)).sum(dim=1))
        of_target = z.gather(1, t.long().clamp(min=0).unsqueeze(1)).squeeze(1)
        losses.append(torch.where(t >= 0, (top - of_target) + log_sum, 0.0))
        lses.append(top + log_sum)
    return [torch.cat(losses), torch.cat(lses)]


def _plain_backward(s):
    V, w = s.case["V"], s.weight.float()
    d_hidden, d_weight = [], torch.zeros_like(w)
    for (x, lse, mask), t, d in zip(_row_pieces(s, 1024), s.targets.split(1024), s.d_loss.split(1024)):
        g = torch.exp(_masked(x.float() @ w.T, mask, V) - lse.unsqueeze(1))
        g.scatter_add_(1, t.long().clamp(min=0).unsqueeze(1), torch.full_like(lse, -1.0).unsqueeze(1))
        g *= torch.where(t >= 0, d, 0.0).unsqueeze(1)
        d_hidden.append((g @ w).to(torch.bfloat16))
        d_weight += g.T @ x.float()
    return [torch.cat(d_hidden), d_weight.to(torch.bfloat16)]


def _plain_quantize(s):
    parts = [_quantize(w) for w in s.weight.split(16384)]
    return [torch.cat([p[1] for p in parts]), torch.cat([p[2] for p in parts])]


def _own_step(s):
    c = s.case
    dtype = s.cz.F32 if c.get("logits") == "f32" else s.cz.BF16
    s.cz.cfgzip_head_step(s.ctx, s.part, None, s.class_mask, s.class_mask.shape[1], s.head, s.hidden, c["H"], c["B"],
                          s.vocab_mask, s.vocab_mask.shape[1], s.logits, dtype, c["V"], s.token, s.rep, s.logp, s.lse,
                          s.workspace, s.workspace.numel(), s.stream)
    return [s.vocab_mask, s.logits, s.token, s.rep, s.logp, s.lse]


def _own_loss(s):
    s.cz.cfgzip_head_loss(s.ctx, s.head, s.hidden, s.case["H"], s.case["N"], s.vocab_mask, _words(s.case["V"]), s.targets, s.loss,
                          s.lse, s.workspace, s.workspace.numel(), s.stream)
    return [s.loss, s.lse]


def _own_backward(s):
    H = s.case["H"]
    s.cz.cfgzip_head_loss_backward(s.ctx, s.head, s.hidden, H, s.case["N"], s.vocab_mask, _words(s.case["V"]), s.targets, s.lse,
                                   s.d_loss, s.d_hidden, H, s.d_weight, s.cz.BF16, H, 0, s.workspace, s.workspace.numel(),
                                   s.stream)
    return [s.d_hidden, s.d_weight]


def _own_quantize(s):
    H = s.case["H"]
    dtype = s.cz.F32 if s.case["from"] == "f32" else s.cz.BF16
    s.cz.cfgzip_head_quantize(s.ctx, s.weight, dtype, H, s.head, s.stream)
    s.cz.cfgzip_head_dequantize(s.ctx, s.head, s.values, H, s.stream)
    return [s.scales[:, : H // 32], s.values]


_PLAIN = {"step": _plain_step, "loss": _plain_loss, "backward": _plain_backward, "quantize": _plain_quantize}
_OWN = {"step": _own_step, "loss": _own_loss, "backward": _own_backward, "quantize": _own_quantize}


# ---------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"step": _exact_step, "loss": _exact_loss, "backward": _exact_backward, "quantize": _exact_quantize}[case["kind"]](s)


def _exact_weights(s, lo, hi):
    if s.weight is not None:
        return s.weight[lo:hi].double()
    H = s.case["H"]
    steps = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2
    out = torch.empty((len(s.packed[lo:hi]), H), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        code = (s.packed[lo:hi] >> (4 * half)).int() & 15
        out[:, half::2] = steps[code & 7] * (1.0 - 2.0 * (code >> 3))
    e = s.scales[lo:hi, : H // 32].int() - 127
    power = torch.ldexp(torch.ones_like(e, dtype=torch.float64), e)
    return out * power.repeat_interleave(32, dim=1)


def _exact_scores(s, rows, lo, hi, V):
    """Scores of the rows [lo, hi), disallowed ones -inf."""
    z = torch.cat([rows.double() @ _exact_weights(s, t, t + 16384).T for t in range(0, V, 16384)], dim=1)
    if s.vocab_mask is None:
        return z
    t = torch.arange(V, device="cuda")
    return torch.where((s.vocab_mask[lo:hi][:, t // 32] >> (t % 32).int()) & 1 == 1, z, -float("inf"))


def _exact_step(s):
    V, K, B = s.case["V"], s.case["K"], s.case["B"]
    k = torch.arange(K, device="cuda")
    bits = (s.class_mask[:, k // 32] >> (k % 32).int()) & 1 == 1
    token_bits = torch.zeros((B, _words(V) * 32), dtype=torch.int64, device="cuda")
    token_bits[:, :V] = bits[:, s.c_dev.long()]
    words = sum(token_bits[:, i::32] * 2 ** i for i in range(32))
    s.vocab_mask = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
    z = _exact_scores(s, s.hidden, 0, B, V)
    lse = torch.logsumexp(z, dim=1)
    token = z.argmax(dim=1)
    logp = z.gather(1, token.unsqueeze(1)).squeeze(1) - lse
    return [s.vocab_mask, z if s.logits is not None else None, token.to(torch.int32), s.r_dev[s.c_dev[token].long()], logp, lse]


def _exact_loss(s):
    losses, lses = [], []
    for lo in range(0, s.case["N"], 512):
        rows, t = s.hidden[lo:lo + 512], s.targets[lo:lo + 512].long()
        z = _exact_scores(s, rows, lo, lo + 512, s.case["V"])
        lses.append(torch.logsumexp(z, dim=1))
        losses.append(torch.where(t < 0, 0.0, lses[-1] - z[torch.arange(len(t), device="cuda"), t.clamp(min=0)]))
    return [torch.cat(losses), torch.cat(lses)]


def _exact_backward(s):
    V, H = s.case["V"], s.case["H"]
    d_hidden = torch.empty((s.case["N"], H), dtype=torch.float64, device="cuda")
    d_weight = torch.zeros((V, H), dtype=torch.float64, device="cuda")
    for lo in range(0, s.case["N"], 512):
        rows, t = s.hidden[lo:lo + 512], s.targets[lo:lo + 512].long()
        g = torch.exp(_exact_scores(s, rows, lo, lo + 512, V) - s.lse[lo:lo + 512].double().unsqueeze(1))
        has = t >= 0
        g[torch.arange(len(t), device="cuda")[has], t[has]] -= 1.0
        g *= (s.d_loss[lo:lo + 512].double() * has).unsqueeze(1)
        part = torch.zeros((len(t), H), dtype=torch.float64, device="cuda")
        for v in range(0, V, 16384):
            part += g[:, v:v + 16384] @ _exact_weights(s, v, v + 16384)
            d_weight[v:v + 16384] += g[:, v:v + 16384].T @ rows.double()
        d_hidden[lo:lo + 512] = part
    return [d_hidden, d_weight]


def _exact_quantize(s):
    V, H = s.case["V"], s.case["H"]
    grid = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    edges = (grid[1:] + grid[:-1]) / 2
    scales, values = [], []
    for w in s.weight.split(8192):
        blocks = w.double().view(-1, H // 32, 32)
        most = blocks.abs().amax(dim=2)
        e = torch.where(most > 0, torch.floor(torch.log2(most)) - 2.0, -127.0).clamp(min=-127.0)
        power = torch.ldexp(torch.ones_like(e), e.int()).unsqueeze(2)
        a = blocks.abs() / power
        below = torch.searchsorted(edges, a.contiguous(), right=False)   # the number of edges under a
        on_edge = (below < 7) & (edges[below.clamp(max=6)] == a) & (below % 2 == 1)
        scales.append((e + 127.0).to(torch.uint8))
        values.append((torch.copysign(grid[below + on_edge], blocks) * power).view(-1, H))
    return [torch.cat(scales), torch.cat(values)]
