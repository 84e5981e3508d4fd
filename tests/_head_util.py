"""Inputs for the head calls, the same results in 64 bits, and how far 32-bit sums of them may be off."""
from __future__ import annotations

import torch

import synth
from synth import rng
from paper_2605_29986_b200 import binding as cz

E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def padded(t: torch.Tensor, pad: int, fill: float = float("nan")) -> torch.Tensor:
    """The same rows in a wider buffer, whose other elements must not matter: NaN, or bytes of ones."""
    if not pad:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + pad), 255 if t.dtype == torch.uint8 else fill, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def unpack(words: torch.Tensor, n: int) -> torch.Tensor:
    shifts = torch.arange(32, dtype=torch.int32, device=words.device)
    return ((words.unsqueeze(2) >> shifts) & 1).reshape(words.shape[0], -1)[:, :n] != 0


def pack(bits: torch.Tensor) -> torch.Tensor:
    rows, n = bits.shape
    wide = torch.zeros((rows, (n + 31) // 32 * 32), dtype=torch.int64, device=bits.device)
    wide[:, :n] = bits
    words = sum(wide[:, i::32] << i for i in range(32))
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def mx_values(packed: torch.Tensor, scales: torch.Tensor, H: int) -> torch.Tensor:
    packed, scales = packed.cpu(), scales.cpu()
    codes = torch.stack([packed & 15, packed >> 4], dim=2).reshape(packed.shape[0], -1)[:, :H]
    e = scales[:, : H // 32].int() - 127
    return E2M1[codes.long()] * torch.ldexp(torch.ones_like(e, dtype=torch.float64), e).repeat_interleave(32, dim=1)


class Case:
    """Weights, hidden states and (64-bit) scores of a small head on the GPU."""

    def __init__(self, V, H, rows, head="bf16", seed=0, pad=0, deviation=2.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.V, self.H, self.rows, self.gen = V, H, rows, g
        if head == "bf16":
            w = torch.empty((V, H), device="cuda").normal_(0.0, H ** -0.5, generator=g).to(torch.bfloat16)
            self.weight = padded(w, pad)
            self.head = cz.cfgzip_head(self.weight, cz.BF16, V, H, row_stride=self.weight.stride(0))
            self.w64 = w.double()
        else:
            self.packed = padded(torch.randint(0, 256, (V, H // 2), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8),
                                 (-(H // 2)) % 16 + 2 * pad)
            # (e2m1 codes drawn evenly have deviation 3: scales around 2^-5 for rows of a few hundred)
            s = torch.randint(119, 125, (V, H // 32), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
            self.scales = padded(s, (-(H // 32)) % 16 + 16 * (pad > 0))
            self.head = cz.cfgzip_head(self.packed, cz.MXFP4, V, H, self.packed.stride(0), self.scales, self.scales.stride(0))
            self.w64 = mx_values(self.packed, self.scales, H).cuda()
        x = torch.empty((rows, H), device="cuda").normal_(0.0, deviation, generator=g).to(torch.bfloat16)
        self.hidden = padded(x, pad)
        self.x64 = x.double()
        self.refresh()

    def refresh(self):
        self.z = self.x64 @ self.w64.T
        # a sum of H products in 32 bits, in any order: off by at most H roundings of the sum of magnitudes
        self.z_tol = self.H * 2.0 ** -24 * (self.x64.abs() @ self.w64.abs().T)

    def workspace(self, op, rows=None):
        n = cz.cfgzip_head_workspace(self.head, op, self.rows if rows is None else rows)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # (NaN wherever a number is read that was not written)

    def lse_tol(self, mask):
        """Off by at most the largest error of a score, the roundings of the sum of exponentials (n terms, a few units in the last
        place each) and of the result."""
        n = mask.sum(dim=1).clamp(min=1)
        z_tol = torch.where(mask, self.z_tol, 0.0).amax(dim=1)
        lse = torch.logsumexp(self.z.masked_fill(~mask, -float("inf")), dim=1)
        return z_tol + (n + 8) * 2.0 ** -23 + lse.abs().nan_to_num(posinf=0.0) * 2.0 ** -22


def class_masks(K, rows, density, key):
    return synth.class_mask_bernoulli(K, rows, density, rng.stream_key(*key))
