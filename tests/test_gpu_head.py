"""The head calls against the same formulas in 64 bits: decode steps from hidden states, 4-bit heads, the loss and its gradient."""
import numpy as np
import pytest
import torch

import synth
from paper_2605_29986_b200 import binding as cz
from _gpu_util import Ctx, dev
from _head_util import Case, class_masks, mx_values, pack, padded, unpack

pytestmark = pytest.mark.gpu
INF = float("inf")


def words(n):
    return (n + 31) // 32


# ---- the decode step ------------------------------------------------------------------------------------------------------
def run_step(ctx, case, cm, B, row_part=None, part=None, logits=None, vocab_mask=True, workspace=None, stream=None, pad=5):
    V = case.V
    out = dict(vocab_mask=torch.full((B, words(V) + 1), 0x5A5A5A5A, dtype=torch.int32, device="cuda") if vocab_mask else None,
               argmax=torch.full((B,), -7, dtype=torch.int32, device="cuda"), rep=torch.full((B,), -7, dtype=torch.int32, device="cuda"),
               logp=torch.full((B,), 99.0, device="cuda"), lse=torch.full((B,), 99.0, device="cuda"), logits=None)
    if logits is not None:
        out["logits"] = torch.full((B, V + pad), 77.0, dtype=logits, device="cuda")
    cz.cfgzip_head_step(ctx.h, ctx.ids[0] if part is None else part, row_part, cm, cm.shape[1], case.head, case.hidden,
                        case.hidden.stride(0), B, out["vocab_mask"], words(V) + 1, out["logits"],
                        cz.BF16 if logits == torch.bfloat16 else cz.F32, V + pad, out["argmax"], out["rep"], out["logp"], out["lse"],
                        case.workspace(cz.HEAD_STEP, B) if workspace is None else workspace,
                        case.workspace(cz.HEAD_STEP, B).numel() if workspace is None else workspace.numel(),
                        stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    return out


def check_step(case, out, mask, reps, rows=None):
    """mask: [B, V] truth values; reps: [B, V] or [V] representatives; rows: which rows were done at all."""
    B, V = mask.shape
    rows = torch.ones(B, dtype=torch.bool, device="cuda") if rows is None else rows
    z = case.z[:B].masked_fill(~mask, -INF)
    lse = torch.logsumexp(z, dim=1)
    tol = case.lse_tol(mask)[:B]
    reps = reps.expand(B, V) if reps.dim() == 1 else reps
    none = ~mask.any(dim=1)
    for b in range(B):
        am, rep, logp, got = (out[k][b].item() for k in ("argmax", "rep", "logp", "lse"))
        if not rows[b]:
            assert (am, rep, logp, got) == (-7, -7, 99.0, 99.0), b
            continue
        if none[b]:
            assert (am, rep, logp, got) == (-1, -1, -INF, -INF), b
            continue
        assert mask[b, am] and z[b, am] >= z[b].max() - 2 * case.z_tol[b].max(), b
        assert rep == reps[b, am].item(), b
        assert abs(got - lse[b].item()) <= tol[b].item(), b
        assert abs(logp - (z[b, am] - lse[b]).item()) <= tol[b].item() + case.z_tol[b, am].item(), b
    if out["vocab_mask"] is not None:
        assert torch.equal(unpack(out["vocab_mask"][:, :-1], V)[rows], mask[rows])
        tail = unpack(out["vocab_mask"][:, :-1], words(V) * 32)[rows][:, V:]
        assert not tail.any() and (out["vocab_mask"][:, -1] == 0x5A5A5A5A).all()
    if out["logits"] is not None:
        got, want = out["logits"][:, :V], z
        assert (out["logits"][:, V:] == 77.0).all()
        assert (got[~rows] == 77.0).all()
        assert torch.equal(got[rows] == -INF, ~mask[rows])
        half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
        ok = (got.double() - want).abs() <= case.z_tol[:B] * 1.01 + want.abs() * half
        assert (ok | ~mask)[rows].all()


STEPS = [
    # V, H, B, K, density, head, pad
    (100, 8, 1, 3, 0.5, "bf16", 0),
    (127, 64, 2, 5, 0.9, "bf16", 8),
    (128, 72, 3, 9, 0.5, "bf16", 0),
    (129, 128, 16, 40, 0.1, "bf16", 8),
    (1000, 256, 31, 33, 0.3, "bf16", 0),
    (5003, 200, 32, 100, 0.02, "bf16", 8),
    (5003, 1000, 33, 64, 0.9, "bf16", 0),
    (40000, 136, 7, 2048, 0.3, "bf16", 8),
    (40000, 520, 64, 300, 0.01, "bf16", 0),
    (20011, 320, 129, 300, 0.2, "bf16", 8),
    (9001, 64, 300, 130, 0.3, "bf16", 0),
    (14001, 64, 200, 130, 0.3, "bf16", 0),
    (16001, 72, 150, 130, 0.3, "bf16", 8),
    (18901, 64, 256, 130, 0.3, "bf16", 0),
    (1, 16, 5, 1, 0.9, "bf16", 0),
    (100, 32, 1, 3, 0.5, "mxfp4", 0),
    (129, 64, 3, 9, 0.5, "mxfp4", 8),
    (1000, 96, 17, 33, 0.3, "mxfp4", 0),
    (5003, 1024, 32, 100, 0.02, "mxfp4", 8),
    (40000, 160, 1, 2048, 0.9, "mxfp4", 0),
    (40000, 4128, 8, 300, 0.05, "mxfp4", 8),
    (20011, 320, 129, 300, 0.2, "mxfp4", 8),
    (9001, 64, 300, 130, 0.3, "mxfp4", 0),
    # few tokens to a block, or hardly any, of long rows
    (60000, 2048, 3, 300, 0.002, "bf16", 0),
    (60000, 4104, 40, 300, 0.0005, "bf16", 8),
    (60000, 2080, 3, 300, 0.002, "mxfp4", 0),
    (60000, 4096, 40, 300, 0.0005, "mxfp4", 8),
    # more than a block lists at a time
    (400003, 8, 2, 5, 0.9, "bf16", 0),
    (400003, 32, 2, 300, 0.5, "mxfp4", 0),
]


@pytest.mark.parametrize("everything", [False, True])
@pytest.mark.parametrize("V,H,B,K,density,head,pad", STEPS)
def test_step(V, H, B, K, density, head, pad, everything):
    case = Case(V, H, B, head, seed=V + H + B, pad=pad)
    p = synth.zipf_partition(V, K, 1.1, seed=3) if K > 1 else synth.Partition(V=1, K=1, c=np.zeros(1, np.int32), r=np.zeros(1, np.int32),
                                                                            sizes=np.ones(1, np.int64))
    cm = class_masks(K, B, density, (5, V, B))
    if B > 2:
        cm[B // 2] = 0           # nothing allowed
        if everything:
            cm[B - 1] = 0xFFFFFFFF   # and bits of classes that are not there
    with Ctx([p]) as ctx:
        c, trep = torch.from_numpy(p.c).long().cuda(), torch.from_numpy(p.r[p.c]).cuda()
        mask = unpack(dev(cm), K)[:, c]
        for logits in (None, torch.float32, torch.bfloat16):
            cz.cfgzip_poll_status(ctx.h)
            out = run_step(ctx, case, dev(cm), B, logits=logits, vocab_mask=logits is not torch.float32)
            check_step(case, out, mask, trep)
            assert cz.cfgzip_poll_status(ctx.h) == (int((~mask.any(dim=1)).sum()), 0, 0)


@pytest.mark.parametrize("B", [70, 150])  # (one pass over the weights, and a product of two tall matrices where logits are not asked for)
def test_step_on_rows_of_several_partitions_and_rows_of_none(B):
    V, H = 3001, 128
    parts = [synth.zipf_partition(V, K, 1.1, seed=K) for K in (40, 300, 77)]
    for head in ("bf16", "mxfp4"):
        case = Case(V, H, B, head, seed=11)
        with Ctx(parts) as ctx:
            rs = np.random.RandomState(1)
            which = rs.randint(0, 3, B)
            cm = class_masks(300, B, 0.3, (6, 1))
            mask = torch.zeros((B, V), dtype=torch.bool, device="cuda")
            reps = torch.zeros((B, V), dtype=torch.int32, device="cuda")
            for b in range(B):
                p = parts[which[b]]
                mask[b] = unpack(dev(cm[b:b + 1]), 300)[0][torch.from_numpy(p.c).long().cuda()]
                reps[b] = torch.from_numpy(p.r[p.c]).cuda()
            ids = np.array(ctx.ids, dtype=np.int32)[which]
            bad = np.zeros(B, dtype=bool)
            bad[[0, 33, B - 1]] = True
            ids[bad] = [-1, 1000, 3]
            cz.cfgzip_poll_status(ctx.h)
            for logits in (None, torch.float32):
                out = run_step(ctx, case, dev(cm), B, row_part=dev(ids), logits=logits)
                check_step(case, out, mask, reps, rows=torch.from_numpy(~bad).cuda())
                assert cz.cfgzip_poll_status(ctx.h)[2] == 3
            # the same rows, grouped once (a plan skips bad rows like any other call)
            d_ids = dev(np.array(ctx.ids, dtype=np.int32)[which])
            cz.cfgzip_plan_rows(ctx.h, ctx.ids[0], d_ids, B, torch.cuda.current_stream())
            check_step(case, run_step(ctx, case, dev(cm), B, row_part=cz.ROWS_AS_PLANNED), mask, reps)


def test_step_takes_the_lowest_of_equal_scores_and_scores_of_minus_infinity():
    V, H, B, K = 700, 64, 4, 7
    case = Case(V, H, B, seed=2)
    c = (np.arange(V) % K).astype(np.int32)
    p = synth.Partition(V=V, K=K, c=c, r=np.arange(K, dtype=np.int32), sizes=np.bincount(c))
    case.weight[:] = case.weight[5].clone()  # every token scores the same
    cm = np.array([[0x7F], [0x60], [0x04], [0x00]], dtype=np.uint32)
    with Ctx([p]) as ctx:
        out = run_step(ctx, case, dev(cm), B, logits=torch.float32)
        assert out["argmax"].tolist() == [0, 5, 2, -1] and out["rep"].tolist() == [0, 5, 2, -1]
        # scores far below what a sum of floats holds: -inf, the row keeps its lowest allowed token
        case.weight[:] = -3e38
        case.hidden[:] = 3e38
        out = run_step(ctx, case, dev(cm), B)
        assert out["argmax"].tolist() == [0, 5, 2, -1]
        assert (out["lse"] == -INF).all() and (out["logp"] == -INF).all()


def test_step_reads_nothing_of_tokens_that_no_row_allows():
    V, H, B, K = 6000, 128, 9, 50
    for head in ("bf16", "mxfp4"):
        case = Case(V, H, B, head, seed=4)
        p = synth.zipf_partition(V, K, 1.1, seed=8)
        cm = np.zeros((B, words(K)), dtype=np.uint32)
        for b in range(B):
            cm[b, 0] = 1 << (b % 4 + 3)
        mask = unpack(dev(cm), K)[:, torch.from_numpy(p.c).long().cuda()]
        used = mask.any(dim=0)
        if head == "bf16":
            case.weight[~used] = float("nan")
        else:
            case.scales[~used] = 255
        with Ctx([p]) as ctx:
            out = run_step(ctx, case, dev(cm), B, logits=torch.float32)
            check_step(case, out, mask, torch.from_numpy(p.r[p.c]).cuda())


def test_step_refuses_a_head_of_another_vocabulary_and_short_masks():
    V, K = 300, 40
    case, other = Case(V, 64, 2, seed=1), Case(V + 1, 64, 2, seed=1)
    with Ctx([synth.zipf_partition(V, K, 1.1, seed=1)]) as ctx:
        cm = dev(class_masks(K, 2, 0.5, (1, 1)))
        am = torch.full((2,), -7, dtype=torch.int32, device="cuda")
        ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")

        def status(case, part=None, stride=2):
            with pytest.raises(cz.CfgzipError) as e:
                cz.cfgzip_head_step(ctx.h, ctx.ids[0] if part is None else part, None, cm, stride, case.head, case.hidden, 64, 2, None, 0,
                                    None, 0, 0, am, None, None, None, ws, ws.numel())
            return e.value.status

        assert status(other) == cz.E_RANGE and status(case, part=5) == cz.E_RANGE and status(case, stride=1) == cz.E_ARG
        torch.cuda.synchronize()
        assert am.tolist() == [-7, -7]


def test_two_steps_at_once_with_a_workspace_each():
    V, H, B, K = 30000, 512, 20, 300
    p = synth.zipf_partition(V, K, 1.1, seed=3)
    c, trep = torch.from_numpy(p.c).long().cuda(), torch.from_numpy(p.r[p.c]).cuda()
    cases = [Case(V, H, B, head, seed=k) for k, head in enumerate(("bf16", "mxfp4"))]
    streams = [torch.cuda.Stream() for _ in cases]
    masks = [dev(class_masks(K, B, d, (2, 1))) for d in (0.05, 0.6)]
    ctxs = [Ctx([p]) for _ in cases]  # (a context is one stream's)
    try:
        torch.cuda.synchronize()
        outs = []
        for case, ctx, st, cm in zip(cases, ctxs, streams, masks):
            out = dict(vocab_mask=None, logits=None, argmax=torch.zeros(B, dtype=torch.int32, device="cuda"),
                       rep=torch.zeros(B, dtype=torch.int32, device="cuda"), logp=torch.zeros(B, device="cuda"), lse=torch.zeros(B, device="cuda"))
            outs.append((out, case.workspace(cz.HEAD_STEP)))
        torch.cuda.synchronize()
        for _ in range(10):
            for (out, ws), case, ctx, st, cm in zip(outs, cases, ctxs, streams, masks):
                cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, cm, cm.shape[1], case.head, case.hidden, H, B, None, 0, None, 0, 0, out["argmax"],
                                    out["rep"], out["logp"], out["lse"], ws, ws.numel(), st)
        torch.cuda.synchronize()
        for (out, _), case, cm in zip(outs, cases, masks):
            check_step(case, out, unpack(cm, K)[:, c], trep)
    finally:
        for ctx in ctxs:
            ctx.close()


def test_four_bit_rows_whose_scales_are_far_apart():
    """Blocks up to 2^23 below the largest scale of their row count in full, and far ones do not spoil the near ones."""
    V, H, B, K = 400, 256, 5, 9
    case = Case(V, H, B, "mxfp4", seed=7)
    case.scales[:] = torch.randint(100, 123, (V, H // 32), generator=case.gen, device="cuda").to(torch.uint8)
    case.scales[5], case.scales[6, 1:], case.scales[7] = 0, 0, 200   # hardly anything, one block alone, large weights
    case.hidden[:, 32:] *= 0.25
    case.x64, case.w64 = case.hidden.double(), mx_values(case.packed, case.scales, H).cuda()
    case.refresh()
    # a 4-bit head's weights may be off by 2^-25 of the largest scale of their row
    top = torch.ldexp(torch.ones(V, dtype=torch.float64, device="cuda"), case.scales.int().amax(dim=1) - 127)
    case.z_tol = case.z_tol + case.x64.abs().sum(dim=1, keepdim=True) * top * 2.0 ** -25
    p = synth.zipf_partition(V, K, 1.1, seed=8)
    with Ctx([p]) as ctx:
        cm = class_masks(K, B, 0.6, (3, 1))
        out = run_step(ctx, case, dev(cm), B, logits=torch.float32)
        mask = unpack(dev(cm), K)[:, torch.from_numpy(p.c).long().cuda()]
        check_step(case, out, mask, torch.from_numpy(p.r[p.c]).cuda())


def test_step_replayed_from_a_graph_on_another_stream():
    V, H, B, K = 9001, 256, 24, 120
    p = synth.zipf_partition(V, K, 1.1, seed=9)
    c, trep = torch.from_numpy(p.c).long().cuda(), torch.from_numpy(p.r[p.c]).cuda()
    for head in ("bf16", "mxfp4"):
        case = Case(V, H, B, head, seed=6)
        with Ctx([p]) as ctx:
            cm = dev(class_masks(K, B, 0.4, (7, 1)))
            ws = case.workspace(cz.HEAD_STEP)
            vm = torch.zeros((B, words(V)), dtype=torch.int32, device="cuda")
            am, rep = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
            logp, lse = (torch.zeros(B, device="cuda") for _ in range(2))
            args = (ctx.h, ctx.ids[0], None, cm, cm.shape[1], case.head, case.hidden, H, B, vm, words(V), None, cz.F32, V, am, rep,
                    logp, lse, ws, ws.numel())
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                cz.cfgzip_head_step(*args, side)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                cz.cfgzip_head_step(*args, side)
            for k in range(3):  # other masks, other hidden states, the same memory
                cm.copy_(dev(class_masks(K, B, (0.02, 0.9, 0.3)[k], (7, 2 + k))))
                x = torch.empty((B, H), device="cuda").normal_(0.0, 2.0, generator=case.gen).to(torch.bfloat16)
                case.hidden.copy_(x)
                case.x64 = x.double()
                case.refresh()
                graph.replay()
                torch.cuda.synchronize()
                mask = unpack(cm, K)[:, c]
                check_step(case, dict(vocab_mask=None, logits=None, argmax=am, rep=rep, logp=logp, lse=lse), mask, trep)


def test_masked_scores_go_on_into_the_sampling_calls():
    V, H, B, K = 20000, 128, 12, 200
    case = Case(V, H, B, seed=12)
    p = synth.zipf_partition(V, K, 1.1, seed=13)
    with Ctx([p]) as ctx:
        cm = dev(class_masks(K, B, 0.2, (8, 1)))
        step = run_step(ctx, case, cm, B, logits=torch.float32, pad=0)
        u = torch.rand(B, generator=case.gen, device="cuda")
        token, rep = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
        lse = torch.zeros(B, device="cuda")
        cz.cfgzip_masked_sample(ctx.h, ctx.ids[0], None, cm, cm.shape[1], step["logits"], cz.F32, V, B, None, 0, u, 1.0, token, rep,
                                None, lse, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        mask = unpack(cm, K)[:, torch.from_numpy(p.c).long().cuda()]
        assert mask[torch.arange(B), token.long()].all()
        assert (lse - step["lse"]).abs().max() <= 1e-4
        assert torch.equal(rep, torch.from_numpy(p.r[p.c]).cuda()[token.long()])


# ---- 4-bit heads ----------------------------------------------------------------------------------------------------------
def quantized(w):
    """e2m1 codes and scale bytes by the definition, block by block, in 64 bits."""
    V, H = w.shape
    x = w.double().cpu().reshape(V, H // 32, 32)
    most = x.abs().amax(dim=2)
    bad = ~torch.isfinite(most)
    e = torch.where(bad | (most == 0), torch.ones_like(most), most)
    e = torch.where(most == 0, -127.0, torch.floor(torch.log2(e)) - 2).clamp(min=-127)
    a = x.abs() / torch.ldexp(torch.ones_like(e), e.int()).unsqueeze(2)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    distance = (a.unsqueeze(3) - grid).abs()
    best = distance.amin(dim=3, keepdim=True)
    near = distance == best
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(dim=3), even.int().argmax(dim=3), near.int().argmax(dim=3))
    code += 8 * torch.signbit(x)
    code[bad] = 0
    scale = torch.where(bad, 255.0, e + 127)
    return code.reshape(V, H), scale.to(torch.uint8)


@pytest.mark.parametrize("V,H,dtype,pad", [(1, 32, torch.float32, 0), (3, 64, torch.bfloat16, 8), (1000, 96, torch.float32, 4),
                                           (257, 1024, torch.bfloat16, 0), (77, 4128, torch.float32, 8)])
def test_quantize(V, H, dtype, pad):
    g = torch.Generator(device="cuda")
    g.manual_seed(V + H)
    w = torch.empty((V, H), device="cuda").normal_(0.0, 1.0, generator=g)
    w *= torch.exp2(torch.randint(-20, 20, (V, 1), generator=g, device="cuda").float())
    flat = w.reshape(-1)
    flat[:32] = 0.0
    if V > 2:
        on_grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda")
        w[1, :32] = torch.cat([on_grid, -on_grid, on_grid * 0.999, on_grid * 1.001]) * 0.125     # ties and their neighbours
        w[2, :32] = 3e38                                                                         # the top of the range
        w[2, 32:64] = 1e-44                                                                      # below the normal numbers
    if V > 20:
        w[10, 5], w[11, 40], w[12, :32] = INF, float("nan"), -0.0
        w[13, :32] = 2.0 ** -126
        w[14, :32] = 7.9 * 2.0 ** -126
    w = padded(w.to(dtype), pad)
    packed = torch.full((V, (H // 2 + 15) // 16 * 16 + 16), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((V, (H // 32 + 15) // 16 * 16 + 16), 0xA5, dtype=torch.uint8, device="cuda")
    head = cz.cfgzip_head(packed, cz.MXFP4, V, H, packed.shape[1], scales, scales.shape[1])
    values = torch.full((V, H + 8), 77.0, dtype=torch.bfloat16, device="cuda")
    with Ctx([]) as ctx:
        st = torch.cuda.current_stream()
        cz.cfgzip_head_quantize(ctx.h, w, cz.F32 if dtype == torch.float32 else cz.BF16, w.stride(0), head, st)
        cz.cfgzip_head_dequantize(ctx.h, head, values, H + 8, st)
        torch.cuda.synchronize()
    code, scale = quantized(w)
    got = torch.stack([packed.cpu() & 15, packed.cpu() >> 4], dim=2).reshape(V, -1)
    assert (got[:, H:] == torch.tensor([5, 10] * ((got.shape[1] - H) // 2))).all() and (scales.cpu()[:, H // 32:] == 0xA5).all()
    assert torch.equal(scales.cpu()[:, :H // 32], scale)
    assert torch.equal(got[:, :H].long(), code)
    want = mx_values(packed, scales, H)
    want[scale.repeat_interleave(32, dim=1) == 255] = float("nan")
    assert (values[:, H:] == 77.0).all()
    assert torch.equal(values[:, :H].cpu().double().nan_to_num(nan=123.0), want.nan_to_num(nan=123.0))


# ---- the loss and its gradient --------------------------------------------------------------------------------------------
LOSSES = [
    # V, H, N, density (None: no masks), pad
    (1, 8, 1, None, 0),
    (100, 8, 1, 0.5, 8),
    (127, 64, 5, None, 0),
    (128, 72, 31, 0.3, 8),
    (257, 128, 128, None, 8),
    (1000, 256, 129, 0.1, 0),
    (5003, 200, 77, 0.9, 8),
    (12000, 320, 300, None, 0),
    (33001, 64, 513, 0.5, 0),
    (700, 1032, 260, 0.02, 8),
    # vocabularies that take tiles of 192, 224 and 256 columns (the others: 160)
    (14001, 64, 130, 0.3, 0),
    (16001, 64, 256, None, 8),
    (18901, 136, 40, 0.5, 8),
]


def loss_inputs(V, H, N, density, pad, seed=0):
    case = Case(V, H, N, seed=V + N + seed, pad=pad)
    g = case.gen
    targets = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.ones((N, V), dtype=torch.bool, device="cuda")
    if density is not None:
        mask = torch.rand((N, V), generator=g, device="cuda") < density
        mask[torch.arange(N), targets.long()] = True
        if N > 4:
            mask[1] = False                                    # nothing allowed
            mask[2, targets[2].long()] = False                 # all but the target
            if V > 1:
                mask[2, (targets[2].long() + 1) % V] = True
            mask[3] = False
            mask[3, targets[3].long()] = True                  # the target alone: no loss at all
    if N > 8:
        targets[4], targets[5], targets[6], targets[7] = -1, V, -2 ** 31, 2 ** 31 - 1
    packed = None
    if density is not None:
        packed = torch.full((N, words(V) + 2), -1, dtype=torch.int32, device="cuda")
        packed[:, :words(V)] = pack(mask)
        if V % 32:
            packed[:, words(V) - 1] |= -1 << (V % 32)          # bits behind the vocabulary do not matter
    return case, mask, packed, targets


def run_loss(ctx, case, packed, targets):
    N = case.rows
    loss, lse = torch.full((N,), 99.0, device="cuda"), torch.full((N,), 99.0, device="cuda")
    ws = case.workspace(cz.HEAD_LOSS)
    cz.cfgzip_head_loss(ctx.h, case.head, case.hidden, case.hidden.stride(0), N, packed, packed.shape[1] if packed is not None else 0,
                        targets, loss, lse, ws, ws.numel(), torch.cuda.current_stream())
    torch.cuda.synchronize()
    return loss, lse


@pytest.mark.parametrize("V,H,N,density,pad", LOSSES)
def test_loss(V, H, N, density, pad):
    case, mask, packed, targets = loss_inputs(V, H, N, density, pad)
    with Ctx([]) as ctx:
        cz.cfgzip_poll_status(ctx.h)
        loss, lse = run_loss(ctx, case, packed, targets)
        assert cz.cfgzip_poll_status(ctx.h) == (0, int((targets >= V).sum()), 0)
    z = case.z.masked_fill(~mask, -INF)
    want = torch.logsumexp(z, dim=1)
    tol = case.lse_tol(mask)
    none = ~mask.any(dim=1)
    assert (lse[none] == -INF).all()
    assert ((lse.double() - want).abs() <= tol)[~none].all()
    t = targets.long().clamp(0, V - 1)
    rows = torch.arange(N, device="cuda")
    ignored, lost = targets < 0, (targets >= V) | ~mask[rows, t]
    assert (loss[ignored] == 0).all() and (loss[lost & ~ignored] == INF).all()
    rest = ~ignored & ~lost
    of_target = z[rows, t]
    # (the difference is rounded as well: of the size of the scores and the normaliser)
    tol = tol + case.z_tol[rows, t] + (want.abs() + of_target.abs()) * 2.0 ** -23
    assert ((loss.double() - (want - of_target)).abs() <= tol)[rest].all()


def gradient(case, mask, targets, d_loss):
    """g in 64 bits, and how far the bf16 one may be off: half a step of bf16, and what a score's error moves it by."""
    V, N = case.V, case.rows
    rows, t = torch.arange(N, device="cuda"), targets.long().clamp(0, V - 1)
    has = (targets >= 0) & (targets < V) & mask[rows, t]
    z = case.z.masked_fill(~mask, -INF)
    p = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True)).nan_to_num(nan=0.0)
    one = torch.zeros_like(p)
    one[rows, t] = 1.0
    g = torch.where(has.unsqueeze(1) & mask, d_loss.double().unsqueeze(1) * (p - one), 0.0)
    off = case.z_tol + case.lse_tol(mask).unsqueeze(1) + 2.0 ** -20
    g_tol = g.abs() * 2.0 ** -8 + d_loss.double().abs().unsqueeze(1) * (p * off * 1.1 + one * 2.0 ** -23)
    return g, torch.where(has.unsqueeze(1) & mask, g_tol, 0.0)


def run_backward(ctx, case, packed, targets, lse, d_loss, d_hidden, d_weight, accumulate=0, workspace=None):
    ws = case.workspace(cz.HEAD_LOSS_BACKWARD) if workspace is None else workspace
    cz.cfgzip_head_loss_backward(ctx.h, case.head, case.hidden, case.hidden.stride(0), case.rows, packed,
                                 packed.shape[1] if packed is not None else 0, targets, lse, d_loss, d_hidden,
                                 d_hidden.stride(0) if d_hidden is not None else 0, d_weight,
                                 cz.F32 if d_weight is not None and d_weight.dtype == torch.float32 else cz.BF16,
                                 d_weight.stride(0) if d_weight is not None else 0, accumulate, ws, ws.numel(),
                                 torch.cuda.current_stream())
    torch.cuda.synchronize()


def close(got, want, g, g_tol, other, n, before=None):
    """A sum of n products of g with `other`: off by g's own errors, n roundings in 32 bits, and half a step of the result."""
    size = g.abs() @ other.abs()
    tol = g_tol @ other.abs() * 1.01 + n * 2.0 ** -24 * size
    if before is not None:
        want = want + before.double()
        tol = tol + 2.0 ** -24 * (want.abs() + before.double().abs())
    tol = tol + want.abs() * (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24) + 1e-38
    return ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("V,H,N,density,pad", LOSSES)
def test_gradient(V, H, N, density, pad):
    case, mask, packed, targets = loss_inputs(V, H, N, density, pad, seed=1)
    d_loss = torch.rand(N, generator=case.gen, device="cuda") - 0.3
    d_loss[0] = 0.0 if N > 1 else 1.0
    g, g_tol = gradient(case, mask, targets, d_loss)
    with Ctx([]) as ctx:
        _, lse = run_loss(ctx, case, packed, targets)
        for dtype, accumulate in ((torch.bfloat16, 0), (torch.float32, 0), (torch.bfloat16, 1), (torch.float32, 1)):
            d_hidden = torch.full((N, H + 8), 77.0, dtype=torch.bfloat16, device="cuda")
            d_weight = torch.full((V, H + 8), 77.0, dtype=dtype, device="cuda")
            before = None
            if accumulate:
                before = torch.randn((V, H), generator=case.gen, device="cuda").to(dtype)
                d_weight[:, :H] = before
            run_backward(ctx, case, packed, targets, lse, d_loss, d_hidden[:, :H], d_weight[:, :H], accumulate)
            assert (d_hidden[:, H:] == 77.0).all() and (d_weight[:, H:] == 77.0).all()
            assert close(d_hidden[:, :H], g @ case.w64, g, g_tol, case.w64, V)
            assert close(d_weight[:, :H], g.T @ case.x64, g.T, g_tol.T, case.x64, N, before)
        # either one alone is the same
        alone = torch.full((N, H), 77.0, dtype=torch.bfloat16, device="cuda")
        run_backward(ctx, case, packed, targets, lse, d_loss, alone, None)
        assert torch.equal(alone, d_hidden[:, :H])
        alone = torch.full((V, H), 77.0, dtype=torch.float32, device="cuda")
        run_backward(ctx, case, packed, targets, lse, d_loss, None, alone)
        assert close(alone, g.T @ case.x64, g.T, g_tol.T, case.x64, N)


def test_gradient_in_several_pieces_of_the_vocabulary():
    V, H, N = 27001, 64, 5003  # scores of two pieces, the second one short; more cuts of the sum than it has stages are not made
    case, mask, packed, targets = loss_inputs(V, H, N, 0.5, 0, seed=3)
    assert 2 * N * V > 256 << 20
    d_loss = torch.rand(N, generator=case.gen, device="cuda") / N
    g, g_tol = gradient(case, mask, targets, d_loss)
    with Ctx([]) as ctx:
        _, lse = run_loss(ctx, case, packed, targets)
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        d_weight = torch.zeros((V, H), dtype=torch.float32, device="cuda")
        run_backward(ctx, case, packed, targets, lse, d_loss, d_hidden, d_weight)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
        assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N)
        again = torch.zeros_like(d_weight), torch.zeros_like(d_hidden)
        run_backward(ctx, case, packed, targets, lse, d_loss, again[1], again[0])
        assert torch.equal(again[0], d_weight) and torch.equal(again[1], d_hidden)


def test_gradient_replayed_from_a_graph():
    V, H, N = 5003, 128, 300
    case, mask, packed, targets = loss_inputs(V, H, N, 0.3, 0, seed=4)
    with Ctx([]) as ctx:
        ws = case.workspace(cz.HEAD_LOSS_BACKWARD), case.workspace(cz.HEAD_LOSS)
        loss, lse, d_loss = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda"), torch.full((N,), 1.0 / N, device="cuda")
        d_hidden, d_weight = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda"), torch.zeros((V, H), device="cuda")

        def both(st):
            cz.cfgzip_head_loss(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], targets, loss, lse, ws[1], ws[1].numel(), st)
            cz.cfgzip_head_loss_backward(ctx.h, case.head, case.hidden, H, N, packed, packed.shape[1], targets, lse, d_loss, d_hidden, H,
                                         d_weight, cz.F32, H, 1, ws[0], ws[0].numel(), st)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        both(side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both(side)
        d_weight.zero_()
        x = torch.empty((N, H), device="cuda").normal_(0.0, 2.0, generator=case.gen).to(torch.bfloat16)
        case.hidden.copy_(x)
        case.x64 = x.double()
        case.refresh()
        graph.replay()
        graph.replay()  # (adds up)
        torch.cuda.synchronize()
        g, g_tol = gradient(case, mask, targets, d_loss)
        assert close(d_hidden, g @ case.w64, g, g_tol, case.w64, V)
        assert close(d_weight, 2 * (g.T @ case.x64), 2 * g.T, 2 * g_tol.T, case.x64, N)


def test_gradient_is_that_of_the_loss():
    """Against differences of the loss: a step along the gradient changes the loss by its squared length, to first order."""
    V, H, N = 600, 64, 40
    case, mask, packed, targets = loss_inputs(V, H, N, 0.5, 0, seed=5)
    targets[targets >= V] = -1
    mask[torch.arange(N), targets.long().clamp(min=0)] = True
    mask[1, targets[1].long()] = True
    packed = pack(mask)
    ones = torch.ones(N, device="cuda")
    with Ctx([]) as ctx:
        _, lse = run_loss(ctx, case, packed, targets)
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        d_weight = torch.zeros((V, H), dtype=torch.float32, device="cuda")
        run_backward(ctx, case, packed, targets, lse, ones, d_hidden, d_weight)

        def loss64(x, w):
            z = (x @ w.T).masked_fill(~mask, -INF)
            t = targets.long()
            of = z[torch.arange(N), t.clamp(min=0)]
            return torch.where(t >= 0, torch.logsumexp(z, dim=1) - of, 0.0).sum()

        eps = 1e-5  # (64-bit losses: 1e-13 of noise; second order: eps times the curvature, below 1e-3 of the slope)
        for x, w, d in ((d_hidden.double(), None, d_hidden.double()), (None, d_weight.double(), d_weight.double())):
            up = loss64(case.x64 + eps * x if x is not None else case.x64, case.w64 + eps * w if w is not None else case.w64)
            down = loss64(case.x64 - eps * x if x is not None else case.x64, case.w64 - eps * w if w is not None else case.w64)
            slope, length = ((up - down) / (2 * eps)).item(), (d ** 2).sum().item()
            # every element of the gradient is within 2^-8 (g) + 2^-8 (result) of its size: the products agree to 2 % at the worst
            assert abs(slope - length) <= 0.02 * length


def test_no_rows():
    case = Case(100, 64, 1, seed=1)
    d_weight = torch.full((100, 72), 77.0, dtype=torch.bfloat16, device="cuda")
    with Ctx([synth.zipf_partition(100, 5, 1.1, seed=1)]) as ctx:
        st = torch.cuda.current_stream()
        cz.cfgzip_head_loss(ctx.h, case.head, None, 0, 0, None, 0, None, None, None, None, 0, st)
        cz.cfgzip_head_loss_backward(ctx.h, case.head, None, 0, 0, None, 0, None, None, None, None, 0, d_weight, cz.BF16, 72, 1, None, 0,
                                     st)
        assert (d_weight == 77.0).all()
        cz.cfgzip_head_loss_backward(ctx.h, case.head, None, 0, 0, None, 0, None, None, None, None, 0, d_weight, cz.BF16, 72, 0, None, 0,
                                     st)
        torch.cuda.synchronize()
        assert (d_weight[:, :64] == 0.0).all() and (d_weight[:, 64:] == 77.0).all()
        cz.cfgzip_head_step(ctx.h, ctx.ids[0], None, None, 0, case.head, None, 0, 0, None, 0, None, 0, 0, None, None, None, None, None, 0, st)


def test_training_under_a_grammar_and_decoding_with_the_head_in_4_bits():
    """As they are used together: masks of the grammar, loss, gradient, an update, the head to 4 bits, decode steps from it."""
    V, H, N, K = 2000, 128, 64, 60
    case = Case(V, H, N, seed=21)
    p = synth.zipf_partition(V, K, 1.1, seed=22)
    cm = dev(class_masks(K, N, 0.5, (9, 1)))
    with Ctx([p]) as ctx:
        st = torch.cuda.current_stream()
        vm = torch.zeros((N, words(V)), dtype=torch.int32, device="cuda")
        cz.cfgzip_expand_mask(ctx.h, ctx.ids[0], None, cm, cm.shape[1], vm, words(V), N, cz.AUTO, st)
        mask = unpack(vm, V)
        targets = torch.rand((N, V), generator=case.gen, device="cuda").masked_fill(~mask, -1.0).argmax(dim=1).to(torch.int32)
        loss, lse = run_loss(ctx, case, vm, targets)
        d_weight = torch.zeros((V, H), dtype=torch.float32, device="cuda")
        d_hidden = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
        run_backward(ctx, case, vm, targets, lse, torch.ones(N, device="cuda"), d_hidden, d_weight)
        g, g_tol = gradient(case, mask, targets, torch.ones(N, device="cuda"))
        assert close(d_weight, g.T @ case.x64, g.T, g_tol.T, case.x64, N)
        case.weight.copy_((case.weight.float() - 0.1 * d_weight).to(torch.bfloat16))
        packed = torch.zeros((V, H // 2), dtype=torch.uint8, device="cuda")
        scales = torch.zeros((V, 16), dtype=torch.uint8, device="cuda")
        case.head = cz.cfgzip_head(packed, cz.MXFP4, V, H, scales=scales, scale_stride=16)
        cz.cfgzip_head_quantize(ctx.h, case.weight, cz.BF16, H, case.head, st)
        torch.cuda.synchronize()
        case.w64 = mx_values(packed, scales, H).cuda()
        case.refresh()
        out = run_step(ctx, case, cm, N)
        check_step(case, out, mask, torch.from_numpy(p.r[p.c]).cuda())
