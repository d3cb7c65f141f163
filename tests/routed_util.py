"""Definitions of the routed operators in 64 bits, with bounds on what 32-bit sums may be off.

Bounds (derived, not fitted).  A sum of K products by the matrix instructions is made of at most K / 4 + 64
additions one after the other (four products at a time at the least, then the waves' sums and the groups'),
each off by at most 2^-23 of the sum of magnitudes that has gone into it: |error| <= (K / 4 + 64) 2^-23 S, S the sum of
the products' magnitudes.  A result rounded to a type is off by its unit roundoff u (2^-8 bf16, 2^-11 fp16,
2^-24 fp32) times its size, and by half the spacing of the smallest fp16 numbers.
Activations are smooth: their derivative is below 1.13, the functions themselves are good to 8 units of 2^-24 and
the multiplications around them to two more.  Hidden rows are held in two parts: 2^-16 of their size in bf16; 2^-21 of
it and 2^-24 in fp16.
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
E2M1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def sum_bound(K, S):
    return (K / 4 + 64) * 2.0 ** -23 * S


def round_bound(y, dtype):
    return UNIT[dtype] * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)


def values(codes, scales, kind, group):
    """codes int8 (.., n, k), scales bf16 (.., n, groups): the weights in 64 bits."""
    w = codes.double() if kind == 0 else E2M1.to(codes.device)[codes.long()]
    return w * scales.double().repeat_interleave(group, dim=-1)[..., :codes.shape[-1]]


def product(x, w, dx=None):
    """x (m, k) times w (n, k) transposed, and the bound on the error (dx: on that of x)."""
    y, S = x @ w.t(), x.abs() @ w.abs().t()
    b = sum_bound(w.shape[1], S)
    if dx is not None:
        b = b + dx @ w.abs().t()
    return y, b


def act(name, x):
    if name == "relu":
        return torch.clamp_min(x, 0)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))
    return x


def layer(x, rowptr, colidx, vals, w1, w2, activation, gated, dtype):
    """x in 64 bits; w1(e), w2(e): weights of an expert in 64 bits.  D and the bound on the error of the kernels' D."""
    T = x.shape[0]
    D = B = None
    for t in range(T):
        for q in range(rowptr[t], rowptr[t + 1]):
            e = colidx[q]
            y = w1(e)
            if y is None:
                continue
            p, dp = product(x[t:t + 1], y)
            if gated:
                i = p.shape[1] // 2
                g, u, dg, du = p[:, :i], p[:, i:], dp[:, :i], dp[:, i:]
            else:
                g, u, dg, du = p, torch.ones_like(p), dp, torch.zeros_like(p)
            a = act(activation, g)
            da = 1.13 * dg + 8 * 2.0 ** -24 * (a.abs() + 1e-30)
            h = a * u
            dh = da * u.abs() + (a.abs() + da) * du + 2 * 2.0 ** -24 * h.abs()
            part = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21, torch.float32: 0.0}[dtype]
            dh = dh + part * h.abs() + (2.0 ** -24 if dtype == torch.float16 else 0.0)
            z, dz = product(h, w2(e), dh)
            if D is None:
                D = torch.zeros(T, z.shape[1], dtype=torch.float64, device=x.device)
                B = torch.zeros_like(D)
            c = vals[q]
            D[t] += c * z[0]
            B[t] += abs(c) * (dz[0] + 2.0 ** -23 * (rowptr[t + 1] - rowptr[t]) * z[0].abs())
    return D, B


def check(got, ref, bound, dtype, what=""):
    bound = bound * (1 + UNIT[dtype]) + round_bound(ref, dtype)
    err = (got.double() - ref).abs()
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: error is {worst:.3f} of the bound"
