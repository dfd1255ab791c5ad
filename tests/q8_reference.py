"""Plain 64-bit statement of the dense cache in 8 bits (include/fa.h, fa_q8_*) for the tests: rounding of blocks, the
tokens that a row holds, attention with the size of its rounding errors.  Shares nothing with the CUDA code."""
from __future__ import annotations

import math

import torch

TOP = {"int8": 127.0, "e4m3": 448.0}


def codes(x: torch.Tensor, fmt: str) -> torch.Tensor:
    """x * top / amax of one block, rounded half to even to the format's numbers.  x: float64 on the CPU, finite.
    The quotient's ties are found in whole numbers: 2 top x against (z_i + z_(i+1)) amax, both exact for 8- and 24-bit x."""
    top = TOP[fmt]
    amax = x.abs().max()
    if amax == 0:
        return torch.zeros_like(x)
    if fmt == "int8":
        z = torch.arange(-127, 128, dtype=torch.float64)
    else:
        pos = torch.tensor([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119], dtype=torch.float64)
        z = torch.cat((-pos.flip(0), pos[1:]))
    twice = (x * (2 * top)).reshape(-1)
    border = (z[1:] + z[:-1]) * amax
    lo, hi = torch.searchsorted(border, twice), torch.searchsorted(border, twice, right=True)
    mid = z.numel() // 2
    pick = torch.where((lo != hi) & ((lo - mid) % 2 != 0), hi, lo)
    return z[pick].reshape(x.shape)


def scale32(x: torch.Tensor, fmt: str) -> float:
    """The stored scale: amax / top rounded to 32 bits, down where top * scale would overflow (nan if a value is not finite)."""
    if not torch.isfinite(x).all():
        return math.nan
    top = torch.tensor(TOP[fmt], dtype=torch.float32)
    s = x.abs().max().to(torch.float32) / top
    return float(torch.nextafter(s, s * 0) if torch.isinf(s * top) else s)


class Rows:
    """The tokens of every row (tensors [n][H][d] of the storage dtype, on the CPU)."""

    def __init__(self, B, H, d, block, fmt, dtype):
        self.H, self.d, self.block, self.fmt, self.dtype = H, d, block, fmt, dtype
        self.k = [torch.zeros((0, H, d), dtype=dtype) for _ in range(B)]
        self.v = [torch.zeros((0, H, d), dtype=dtype) for _ in range(B)]

    def push(self, b, k, v):
        self.k[b], self.v[b] = torch.cat((self.k[b], k.cpu())), torch.cat((self.v[b], v.cpu()))

    def block_of(self, side, b, h, i):
        x = (self.k if side == "k" else self.v)[b][i * self.block:(i + 1) * self.block, h].double()
        return x

    def held(self, side, b, h):
        """What the cache stands for: [n][d] in 64 bits."""
        x = (self.k if side == "k" else self.v)[b][:, h].double().clone()
        for t in range(0, x.shape[0] // self.block * self.block, self.block):
            blk = x[t:t + self.block]
            s = scale32(blk, self.fmt)
            x[t:t + self.block] = math.nan if math.isnan(s) else codes(blk, self.fmt) * s
        return x


def attention(k, v, q, n_q, scale, dtype):
    """k, v [n][d], q [n_q][G][d] (64 bits): outputs of the last n_q tokens' queries and how far a result may be off.

    A result in `dtype` is off by half a step of it, and by these relative to sum p |v| / sum p:
      * the weights' rounding to halves, 2^-11 (fp32: to two halves, 2^-22), and a largest weight's 2^-24 for what is below the halves' range;
      * a logit's error delta, for p and for the sum of p: sums of d products, each step off by 2^-23 of the sum of magnitudes A (tensor
        cores may cut instead of round), the scales' products, q (and the tail's values) in two halves for fp32: (d + 16) 2^-23 A;
      * ex2.approx and the sums over n tokens in steps of 16, over warps and parts: (n / 16 + 64) 2^-23 + 2^-21."""
    n, d = k.shape
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    half_step = torch.finfo(dtype).eps / 2
    w16 = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    for i in range(n_q):
        seen = n - n_q + i + 1
        if seen <= 0:
            continue
        s = q[i] @ k[:seen].T * scale
        A = (q[i].abs() @ k[:seen].abs().T * scale).amax(-1, keepdim=True)
        p = torch.softmax(s, -1)
        out[i] = p @ v[:seen]
        mass = p @ v[:seen].abs()
        delta = (d + 16) * 2.0 ** -23 * A
        top = (p @ torch.ones_like(v[:seen])) * (p[..., None] * v[:seen].abs()).amax((1, 2))[:, None]
        tol[i] = half_step * out[i].abs() + mass * (w16 + 2 * torch.expm1(delta) + (seen / 16 + 64) * 2.0 ** -23 + 2.0 ** -21) + seen * 2.0 ** -38 * top
    return out, tol + 1e-30
