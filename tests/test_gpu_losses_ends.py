"""The losses and their gradients where their numbers end: infinities, sums that cancel, ranges that a type or a row leaves."""
import math

import pytest
import torch

import loss_util as lu
import paper_2407_00243_amd as tf

pytestmark = pytest.mark.gpu

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def matrix(T, E, k, c):
    return tf.DeviceCsr(T, E, torch.zeros(T + 1, dtype=torch.int32, device="cuda"), c, torch.zeros(T * k, device="cuda"))


# ------------------------------------------------------------------------------------------ router

@pytest.mark.parametrize("scoring", range(4))
@pytest.mark.parametrize("E,dtype", [(3, F), (8, HF), (24, BF), (60, F), (130, BF), (256, HF), (500, F), (1024, BF)])
def test_rows_without_an_entry_get_zeros_whatever_they_hold(E, dtype, scoring):
    """Scores of +inf, NaN and the largest number in rows without an entry; and a gradient of the balance that is not finite."""
    T, k = 150, 2
    scores = (2 * torch.randn(T, E, device="cuda", generator=gen(E + scoring))).to(dtype)
    c = scores.float().topk(k, 1).indices.to(torch.int32)
    closed = torch.arange(T, device="cuda") % 3 == 1
    c[closed] = torch.tensor([-1, E], device="cuda", dtype=torch.int32)
    fill = torch.tensor([math.inf, math.nan, torch.finfo(dtype).max, -math.inf, 1.0], device="cuda").to(dtype)
    rows = torch.nonzero(closed).squeeze(1)
    clean = scores.clone()
    scores[rows, torch.arange(rows.numel(), device="cuda") % E] = fill[torch.arange(rows.numel(), device="cuda") % 5]
    scores[rows[::7]] = math.inf
    c = c.reshape(-1).contiguous()
    dvals = torch.randn(T * k, device="cuda", generator=gen(1))
    counts = torch.ones(E + 1, device="cuda", dtype=torch.int32)
    counts[:E] += (torch.arange(E, device="cuda") % 5).int()
    counts[E] = T
    for v, n, d in ((dvals, counts, 0.7), (dvals, None, None), (None, counts, 0.7), (dvals, counts, math.inf), (None, counts, math.nan)):
        dloss = None if d is None else torch.full((1,), d, device="cuda")
        out = torch.full((T, E), math.nan, device="cuda", dtype=dtype)
        tf.tf_moe_route_grad(scores, matrix(T, E, k, c), out, scoring, 1.5, v, n, dloss, stream())
        assert not out[closed].any(), f"E{E} {dtype} scoring {scoring} dloss {d}"
        if d is None or math.isfinite(d):
            ref, bound = lu.route_grad(clean, c, k, scoring, 1.5, v, n, dloss)
            lu.check(out, ref, bound, dtype, f"E{E} {dtype} scoring {scoring}")
