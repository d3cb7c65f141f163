"""Definitions of the losses and their gradients in 64 bits, with bounds on what the kernels' results may be off.

Bounds (derived, not fitted; u is the unit roundoff of a type, 2^-8 bf16, 2^-11 fp16, 2^-24 fp32).
  Router.  A share is an exponential (or a sigmoid) over a sum of at most 1024 of them: the difference under the exponential is off by 2^-24 of
  its size, functions, quotient and the reciprocal by 2^-22 each, a sum over lanes by (16 + 6) 2^-24.  With room for the sums' own
  terms: |dp| <= (40 + |l - top|) 2^-23 p.  A mean over n rows is a sum of at most n / 16 terms in a lane, 6 between lanes, 16 between
  waves and 256 between workgroups.  Gradients are shares times differences of gradients: three factors of that kind.
  Cross entropy.  Logits: a sum of K products by the matrix instructions, at least four at a time, |dl| <= (P K / 4 + 64) 2^-23 S
  with S the sum of their magnitudes, P = 1, or 6 where fp32 numbers are multiplied as three parts, whose products that are left out lie
  below 2^-24 S.  log-sum-exp: the largest |dl|, and the sum's own (V / 512 + 80) 2^-23 (32 terms in a lane, 2 between lanes,
  every sixteenth block of 64 classes in a wave), and one rounding.  A gradient of a logit: exp(l - lse) is off by its argument, and is rounded to
  16 bits: u of it (fp32: 2^-24), fp16 also by 2^-25 2^-15 of the largest |dloss|.  dX, dW: that times the other operand, a sum of V (or
  rows) products like the logits', and one rounding to the type.
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SOFTMAX, SOFTMAX_TOP, SIGMOID, SIGMOID_TOP = 0, 1, 2, 3


def rounded(bound, ref, dtype):
    least = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133
    return bound * (1 + UNIT[dtype]) + UNIT[dtype] * ref.abs() + least


def check(got, ref, bound, dtype=torch.float32, what=""):
    bound = rounded(bound, ref, dtype)
    err = (got.double().to(ref.device) - ref).abs()
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: error is {worst:.3f} of the bound"


# ------------------------------------------------------------------------------------------ router

def entries(colidx, T, E, k):
    """How often each row names each expert."""
    m = torch.zeros(T, E, dtype=torch.float64, device=colidx.device)
    c = colidx.long().reshape(T, k)
    for i in range(k):
        ok = (c[:, i] >= 0) & (c[:, i] < E)
        m[torch.arange(T, device=m.device)[ok], c[ok, i]] += 1
    return m


def shares(l, sigmoids, m=None):
    """Shares of the scores over all experts, or of the named ones as often as they are named; 1 - sigma (or 1); and the bound's factor."""
    l = torch.where(torch.isnan(l), -math.inf, l)
    z = torch.nn.functional.logsigmoid(l) if sigmoids else l
    over = z if m is None else z + torch.log(m)
    p = torch.softmax(over, 1) if l.shape[0] else l
    p = torch.where((over > -math.inf).any(1, keepdim=True), p, 0.0)
    each = p if m is None else torch.where(m > 0, p / m, 0.0)
    top = over.amax(1, keepdim=True) if l.shape[0] else l
    factor = torch.where(z > -math.inf, 40 + (z - torch.where(top > -math.inf, top, 0.0)).abs(), 0.0) * 2.0 ** -23
    return each, torch.sigmoid(-l) if sigmoids else torch.ones_like(l), factor


def balance(scores, colidx, k, scoring):
    l = scores.double()
    T, E = l.shape
    m = entries(colidx, T, E, k)
    named = (m.sum(1) > 0)[:, None]
    p, _, factor = shares(l, scoring >= SIGMOID)
    p = torch.where(named, p, 0.0)
    counts, n = m.sum(0), named.sum().item()
    mass = p.sum(0) / max(n, 1)
    bound = (p * factor).sum(0) / max(n, 1) + (n / 16 + 400) * 2.0 ** -24 * mass
    f = counts / max(counts.sum().item(), 1.0)
    loss, loss_bound = E * (f * mass).sum(), E * (f * bound).sum() + 64 * 2.0 ** -24 * E * (f * mass).sum()
    return torch.cat([counts, torch.tensor([n], device=l.device, dtype=torch.float64)]), mass, bound, loss, loss_bound


def route_grad(scores, colidx, k, scoring, scale, dvals, counts, dloss):
    l = scores.double()
    T, E = l.shape
    m = entries(colidx, T, E, k)
    named = (m.sum(1) > 0)[:, None]
    d, b = torch.zeros_like(l), torch.zeros_like(l)
    if dvals is not None:
        c, g = colidx.long().reshape(T, k), torch.zeros_like(l)
        ga = torch.zeros_like(l)
        for i in range(k):
            ok = (c[:, i] >= 0) & (c[:, i] < E)
            r = torch.arange(T, device=l.device)[ok]
            x = scale * dvals.double().reshape(T, k)[ok, i]
            g[r, c[ok, i]] += x
            ga[r, c[ok, i]] += x.abs()
        sig = scoring >= SIGMOID
        if scoring == SIGMOID:
            clean = torch.where(torch.isnan(l), -math.inf, l)
            s, rest = torch.sigmoid(clean), torch.sigmoid(-clean)
            d, b = d + s * rest * g, b + 60 * 2.0 ** -23 * s * rest * ga
        else:
            q, rest, factor = shares(l, sig, None if scoring == SOFTMAX else m)
            inner = (q * g).sum(1, keepdim=True)
            inner_a = (q * ga).sum(1, keepdim=True)
            inner_b = (q * ga * factor).sum(1, keepdim=True) + 40 * 2.0 ** -23 * inner_a
            mm = torch.ones_like(m) if scoring == SOFTMAX else m
            sel = named.double()
            d = d + sel * q * rest * (g - mm * inner)
            b = b + sel * q * rest * (3 * (factor + 60 * 2.0 ** -23) * (ga + mm * inner_a) + mm * inner_b)
    if dloss is not None:
        q, rest, factor = shares(l, scoring >= SIGMOID)
        f = counts[:E].double() / max(counts[:E].double().sum().item(), 1.0)
        c = dloss.double().item() * E / max(counts[E].item(), 1)
        inner = (q * f).sum(1, keepdim=True)
        inner_b = (q * f * factor).sum(1, keepdim=True) + 40 * 2.0 ** -23 * inner
        q = torch.where(named, q, 0.0)
        d = d + c * q * rest * (f - inner)
        b = b + abs(c) * q * rest * (3 * (factor + 60 * 2.0 ** -23) * (f + inner) + inner_b)
    return d, b


# ----------------------------------------------------------------------------------- cross entropy

def sum_bound(K, S, parts):
    return (parts * K / 4 + 64) * 2.0 ** -23 * S + (2.0 ** -24 * S if parts > 1 else 0.0)


def xent(X, W, labels, dloss=None):
    """loss, lse, dX, dW of the formulas in 64 bits, each with the bound on the kernels' (dX, dW: where dloss is given)."""
    dtype, V = X.dtype, W.shape[0]
    parts = 6 if dtype == torch.float32 else 1
    kept = torch.nonzero((labels >= 0) & (labels < V)).squeeze(1)
    x, w, y = X[kept].double(), W.double(), labels[kept].long()
    wt = w.t().contiguous()
    l, dl = x @ wt, sum_bound(X.shape[1], x.abs() @ wt.abs(), parts)
    lse = torch.logsumexp(l, 1)
    at = torch.arange(kept.numel(), device=X.device)
    p = torch.exp(l - lse[:, None])
    dlse = dl.amax(1) + (V / 512 + 80) * 2.0 ** -23 + 2.0 ** -23 * lse.abs() if kept.numel() else lse
    others = p.clone()
    others[at, y] = 0.0
    # (lse - l_y would cancel: 2^-53 of a logit of 50 is a hundredth of a loss of 1e-12)
    from_y = torch.exp(l - l[at, y][:, None])
    from_y[at, y] = 0.0
    loss = torch.where(lse - l[at, y] < 30, torch.log1p(from_y.sum(1)), lse - l[at, y])
    # log(1 + sum of exp(l_v - l_y)): the sum is off by its arguments, the logarithm by that over 1 + the sum
    dloss_b = (others * (dl + dl[at, y][:, None])).sum(1) + (V / 512 + 80) * 2.0 ** -23 * others.sum(1) + 2.0 ** -22 * loss
    dloss_b = torch.where(loss > 30, dlse + dl[at, y] + 2.0 ** -22 * lse.abs(), dloss_b)
    full = lambda v: torch.zeros(X.shape[0], dtype=torch.float64, device=X.device).index_copy_(0, kept, v)  # noqa: E731
    out = {"loss": (full(loss), full(dloss_b)), "lse": (full(lse), full(dlse))}
    if dloss is None:
        return out
    c = dloss[kept].double()
    g = p.clone()
    g[at, y] -= 1.0
    g *= c[:, None]
    dg = c.abs()[:, None] * p * (dl + dlse[:, None] + 2.0 ** -20) + (UNIT[dtype] + 2.0 ** -22) * g.abs() + c.abs()[:, None] * 2.0 ** -23 * (p + 1e-9)
    top = c.abs().max().item() if kept.numel() else 0.0
    dg = dg + (2.0 ** -40 if dtype == torch.float16 else 2.0 ** -126) * top
    ga = g.abs() + dg
    dX = torch.zeros(X.shape, dtype=torch.float64, device=X.device).index_copy_(0, kept, g @ w)
    bX = torch.zeros_like(dX).index_copy_(0, kept, dg @ w.abs() + sum_bound(V, ga @ w.abs(), parts))
    gt = g.t().contiguous()
    out["dX"] = (dX, bX)
    out["dW"] = (gt @ x, dg.t().contiguous() @ x.abs() + sum_bound(kept.numel(), ga.t().contiguous() @ x.abs(), parts))
    return out
