"""Routed operators where their calls end: experts named again and again, the ends of the numbers' range, long launches."""
import itertools
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2407_00243_amd as tf  # noqa: E402
import routed_util as ru  # noqa: E402
from test_gpu_routed import ACT, DT, csr, empty_q4, gen, randn, random_q4, run_layer, run_route, stream  # noqa: E402


# ------------------------------------------------------------------- rows that name an expert more than once

@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("quant", [None, (tf.TF_Q4_INT, 64), (tf.TF_Q4_E2M1, 128)])
@pytest.mark.parametrize("H,I,gated", [(4100, 330, True), (4100, 330, False), (260, 4100, True)])
@pytest.mark.parametrize("rows,E", [
    ([[0, 0]] * 4, 3),                       # 8 entries of an expert from 4 tokens
    ([[7, 7]] * 4, 40),                      # the same where workgroups go by entries
    ([[1] * 20], 3),                         # 20 and 70 from one
    ([[1] * 70], 2),
    ([[0] * 9 + [1]] * 4, 2),                # 36 from 4
    ([[2, 2]] * 12, 3),                      # 24, 72 from 12
    ([[2] * 6] * 12, 3),
    ([[1, 1, 1]] * 20, 2),                   # 60 from 20
    ([[0, 1, 0, 0]] * 33, 2),                # 99 from 33
])
def test_layer_with_experts_named_again(dtype, quant, H, I, gated, rows, E):
    D, ref, b = run_layer(rows, E, H, I, 72, dtype, "silu" if gated else "relu", gated, quant)
    ru.check(D, ref, b, DT[dtype])


# ------------------------------------------------- more rows than the threads of one launch (2^32) have room for

def test_route_of_more_tokens_than_a_launch_takes():
    T = (1 << 26) + 9                   # one wave a token
    scores = torch.zeros(T, 1, dtype=torch.bfloat16, device="cuda")
    scores[T - 1], scores[1 << 26], scores[(1 << 26) - 5] = 3.0, 2.0, -1.0
    A = tf.DeviceCsr(T, 1, torch.full((T + 1,), -9, dtype=torch.int32, device="cuda"),
                     torch.full((T,), -9, dtype=torch.int32, device="cuda"), torch.full((T,), -9.0, device="cuda"))
    tf.tf_moe_route(scores, A, tf.TF_ROUTE_SIGMOID, scale=2.0, stream=stream())
    assert torch.equal(A.rowptr, torch.arange(T + 1, dtype=torch.int32, device="cuda")) and not A.colidx.any()
    ref = 2 * torch.sigmoid(scores[:, 0].float())
    assert ((A.vals - ref).abs() <= 2.0 ** -20).all() and A.vals[T - 1] > 1.9


def test_layer_of_more_rows_than_a_launch_takes():
    T, E, H, I, O = (1 << 24) + 70, 3, 8, 16, 8          # 256 threads a row of D
    at = [0, 5, (1 << 24) - 1, 1 << 24, T - 1]
    g = gen(41)
    W1, W2 = randn(g, E, 2 * I, H).bfloat16(), randn(g, E, O, I).bfloat16()
    X = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    X[at] = randn(g, len(at), H, dtype=torch.bfloat16)
    cols = [0, 2, 1, 1, 0]
    A, _, _ = csr([[e] for e in cols], E)
    rowptr = torch.zeros(T + 1, dtype=torch.int32, device="cuda")
    rowptr[torch.tensor(at, device="cuda") + 1] = 1
    A = tf.DeviceCsr(T, E, torch.cumsum(rowptr, 0).int(), A.colidx, A.vals)
    D = torch.full((T, O), math.nan, dtype=torch.bfloat16, device="cuda")
    with tf.MoePlan(E, H, I, torch.bfloat16, T, len(at), n_out=O) as plan:
        plan.run(A, X, W1, W2, D, stream())
        torch.cuda.synchronize()
    ref, b = ru.layer(X[at].double(), list(range(len(at) + 1)), cols, A.vals.tolist(), lambda e: W1[e].double(),
                      lambda e: W2[e].double(), "silu", True, torch.bfloat16)
    ru.check(D[at], ref, b, torch.bfloat16)
    D[at] = 0
    assert (D == 0).all()


# --------------------------------------------------------------------- the smallest and the largest numbers

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,scale", [(tf.TF_Q4_INT, 1.0), (tf.TF_Q4_E2M1, 64.0)])
@pytest.mark.parametrize("v", [1.3 * 2.0 ** -105, 1.1 * 2.0 ** -113, 1.7 * 2.0 ** -119])
def test_group_sums_of_small_numbers(dtype, kind, scale, v):
    n, k = 16, 256
    codes = torch.ones(1, n, k, dtype=torch.int8, device="cuda")
    scales = torch.full((1, n, 2), scale, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, k, kind, 128)
    tf.tf_q4_pack(q, codes, scales, stream())
    w = ru.values(codes, scales, kind, 128)[0]
    x = torch.full((2, k), v, device="cuda").to(DT[dtype])
    x[1, ::2] *= -0.25
    y = torch.empty(2, n, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    ref, b = ru.product(x.double(), w)
    # additions of subnormal numbers are off by half of 2^-149 each, 2^-10 of what is summed
    ru.check(y, ref, b + scale * 3 * k * 2.0 ** -140, DT[dtype])


def top_q4(n, k, kind, group, scale, mats=1):
    """The largest codes, every second output's negative, and one scale: weights in 64 bits beside them."""
    codes = torch.full((mats, n, k), 7, dtype=torch.int8, device="cuda")
    codes[:, 1::2] = -7 if kind == tf.TF_Q4_INT else 15
    scales = torch.full((mats, n, -(-k // group)), scale, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, k, kind, group, mats)
    tf.tf_q4_pack(q, codes, scales, stream())
    return q, ru.values(codes, scales, kind, group)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,group", itertools.product([tf.TF_Q4_INT, tf.TF_Q4_E2M1], [32, 64, 128]))
@pytest.mark.parametrize("m", [1, 20, 40])
def test_group_sums_may_pass_the_largest_number(dtype, kind, group, m):
    # 300 times the largest number times 7 (6) is far beyond it; with the scale the sums are not
    n, k = 40, 300
    q, w = top_q4(n, k, kind, group, 2.0 ** -12)
    x = torch.full((m, k), torch.finfo(DT[dtype]).max, dtype=DT[dtype], device="cuda")
    x[m // 2, ::3] *= -0.5
    y = torch.empty(m, n, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    ref, b = ru.product(x.double(), w[0])
    assert ref.abs().max() < torch.finfo(DT[dtype]).max
    ru.check(y, ref, b, DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", [tf.TF_Q4_INT, tf.TF_Q4_E2M1])
def test_one_largest_number_comes_back(dtype, kind):
    # code 2 (value 2, and 1 of E2M1) times a scale that makes 1 of it
    n, k = 16, 128
    codes = torch.full((1, n, k), 2, dtype=torch.int8, device="cuda")
    scales = torch.full((1, n, 1), 0.5 if kind == tf.TF_Q4_INT else 1.0, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, k, kind, 128)
    tf.tf_q4_pack(q, codes, scales, stream())
    x = torch.zeros(1, k, dtype=DT[dtype], device="cuda")
    x[0, 77] = torch.finfo(DT[dtype]).max
    y = torch.empty(1, n, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    assert (y == x[0, 77]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 128])
def test_group_sums_of_hidden_rows_may_pass_the_largest_number(dtype, group):
    T, H, I, O = 3, 96, 200, 40
    W1, v1 = top_q4(I, H, tf.TF_Q4_INT, group, 2.0 ** -10, mats=2)
    W2, v2 = top_q4(O, I, tf.TF_Q4_INT, group, 2.0 ** -12, mats=2)
    X = torch.full((T, H), 0.75 * torch.finfo(DT[dtype]).max, device="cuda").to(DT[dtype])
    A, rowptr, cols = csr([[0], [1, 0], [1]], 2, torch.full((4,), 0.5, device="cuda"))
    D = torch.empty(T, O, dtype=DT[dtype], device="cuda")
    with tf.MoePlan(2, H, I, DT[dtype], T, 4, n_out=O, activation=tf.TF_ACT_RELU, gated=False) as plan:
        plan.run(A, X, W1, W2, D, stream())
        torch.cuda.synchronize()
    ref, b = ru.layer(X.double(), rowptr, cols, A.vals.tolist(), lambda e: v1[e], lambda e: v2[e], "relu", False, DT[dtype])
    assert torch.finfo(DT[dtype]).max / 64 < ref.abs().max() < torch.finfo(DT[dtype]).max
    ru.check(D, ref, b, DT[dtype])


# ---------------------------------------------------------------------------------------- router

@pytest.mark.parametrize("scoring", [tf.TF_ROUTE_SIGMOID, tf.TF_ROUTE_SIGMOID_TOP])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sigmoid_weights_of_small_scores(scoring, dtype):
    E, k = 70, 4
    rows = [[-90.0, -91.0], [-87.0, -87.5, -88.0], [-100.0] * 4, [-1000.0, -1001.0, -1003.0, -1000.0], [3.0, -90.0, -95.0],
            [-88.5, -88.75, -89.0, -103.0], [60.0, 50.0, -1.0]]
    scores = torch.full((len(rows), E), -math.inf, device="cuda")
    for t, r in enumerate(rows):
        scores[t, 3:3 + 7 * len(r):7] = torch.tensor(r, device="cuda")
    scores = scores.to(DT[dtype])
    cols, vals = run_route(scores, None, k, scoring, 1.0)
    for t, r in enumerate(rows):
        c = [e for e in cols[t].tolist() if e >= 0]
        assert len(c) == len(r) and (vals[t, len(r):] == 0).all()
        l = scores[t, c].double().cpu()
        log = -torch.nn.functional.softplus(-l, threshold=800.0)        # of the sigmoid
        w = torch.exp(log - log.max()) / torch.exp(log - log.max()).sum() if scoring == tf.TF_ROUTE_SIGMOID_TOP else torch.exp(log)
        # functions good to a few units, arguments rounded once: 2^-24 of their size; below the normal numbers half a spacing and
        # the few units again
        bound = 2.0 ** -24 * (40 + 2 * l.abs().max().item()) * w + 2.0 ** -147
        assert ((vals[t, :len(r)].double() - w).abs() <= bound).all(), (t, vals[t], w)


# ------------------------------------------------------------------------------------- hidden rows

@pytest.mark.parametrize("quant", [False, True])
def test_hidden_rows_of_bf16_reach_the_largest_number_of_fp32(quant):
    # between the largest bf16 number and the largest fp32 number, where rounding to bf16 would make an infinity
    big = torch.finfo(torch.bfloat16).max
    X = torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda")
    X[0, :2] = torch.tensor([big, 1.5 * 2.0 ** 119], device="cuda")
    X[1, :2] = -X[0, :2]
    w1, w2 = torch.ones(1, 8, 8, device="cuda"), torch.full((1, 8, 8), 2.0 ** -10, device="cuda")
    W1, W2 = w1.bfloat16(), w2.bfloat16()
    if quant:
        (W1, w1), (W2, w2) = one_q4(8, 1.0), one_q4(8, 2.0 ** -10)
    A, rowptr, cols = csr([[0], [0]], 1, torch.ones(2, device="cuda"))
    D = torch.empty(2, 8, dtype=torch.bfloat16, device="cuda")
    with tf.MoePlan(1, 8, 8, torch.bfloat16, 2, 2, activation=tf.TF_ACT_IDENTITY, gated=False) as plan:
        plan.run(A, X, W1, W2, D, stream())
        torch.cuda.synchronize()
    h = X.double() @ w1[0].double().t()
    assert (big < h.abs()).all() and (h.abs() < torch.finfo(torch.float32).max).all()
    ref, b = ru.layer(X.double(), rowptr, cols, [1.0, 1.0], lambda e: w1[e].double(), lambda e: w2[e].double(), "identity", False,
                      torch.bfloat16)
    ru.check(D, ref, b, torch.bfloat16)


def one_q4(n, scale):
    codes = torch.ones(1, n, n, dtype=torch.int8, device="cuda")
    scales = torch.full((1, n, 1), scale, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, n, tf.TF_Q4_INT, 128)
    tf.tf_q4_pack(q, codes, scales, stream())
    return q, ru.values(codes, scales, tf.TF_Q4_INT, 128)


# ------------------------------------------------------------------------------------- activations

@pytest.mark.parametrize("activation,lowest", [("gelu", -12.9), ("silu", -91.0)])
def test_activations_keep_their_tails(activation, lowest):
    # both products are with the identity matrix, and exact: D is the activation of X
    n = 64
    X = torch.linspace(lowest, 6.0, 4 * n, device="cuda").view(4, n)
    one = torch.eye(n, device="cuda")[None].contiguous()
    A, _, _ = csr([[0]] * 4, 1, torch.ones(4, device="cuda"))
    D = torch.empty(4, n, device="cuda")
    with tf.MoePlan(1, n, n, torch.float32, 4, 4, activation=ACT[activation], gated=False) as plan:
        plan.run(A, X, one, one, D, stream())
        torch.cuda.synchronize()
    x = X.double()
    if activation == "gelu":
        ref = 0.5 * x * torch.special.erfc(-x * math.sqrt(0.5))
        # the argument of erfc is rounded twice, which moves its logarithm by x^2 times that
        rel = 16 + 2 * x * x
    else:
        ref = x * torch.exp(x.clamp(max=0)) / (1 + torch.exp(-x.abs()))
        rel = 16 + 2 * x.abs()
    assert ((D.double() - ref).abs() <= 2.0 ** -24 * rel * ref.abs() + 2.0 ** -126).all()


def test_hidden_rows_of_fp16_are_off_by_what_the_call_says():
    # the first product is with the identity matrix, the second with 1024 times it: D is 1024 times what is held of X
    n = 64
    X = torch.linspace(1, 2, n, device="cuda") * torch.tensor([[2.0 ** -11], [-2.0 ** -6], [2.0 ** -2], [4.0]], device="cuda")
    X = X.half()
    one = torch.eye(n, dtype=torch.float16, device="cuda")[None]
    A, _, _ = csr([[0]] * 4, 1, torch.ones(4, device="cuda"))
    D = torch.empty(4, n, dtype=torch.float16, device="cuda")
    # h = x^2 / 2 (identity gate times a half of x), which has up to 22 bits and sizes from 2^-23 to 2^5
    W1 = torch.cat([one, one * 0.5], 1).contiguous()
    with tf.MoePlan(1, n, n, torch.float16, 4, 4, activation=tf.TF_ACT_IDENTITY) as plan:
        plan.run(A, X, W1, (one * 1024).contiguous(), D, stream())
        torch.cuda.synchronize()
    h = X.double() ** 2 / 2
    bound = 1024 * torch.maximum(2.0 ** -22 * h, torch.full_like(h, 2.0 ** -25))
    ru.check(D, 1024 * h, bound, torch.float16)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("quant,I", [(None, 71), ((tf.TF_Q4_INT, 32), 3), ((tf.TF_Q4_E2M1, 64), 133)])
def test_what_lies_between_hidden_rows_is_not_read(dtype, quant, I):
    # a workspace in memory that held NaN before, as far as the allocator gives it out again
    torch.cuda.empty_cache()
    junk = torch.full((1 << 26,), math.nan, device="cuda")
    torch.cuda.synchronize()
    del junk
    torch.cuda.empty_cache()
    D, ref, b = run_layer([[0, 2], [1], [2, 0, 1]] * 7, 3, 130, I, 50, dtype, quant=quant)
    ru.check(D, ref, b, DT[dtype])


# ---------------------------------------------------------------- launches that other tests' sizes do not lead to

@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind,group", [(tf.TF_Q4_INT, 64), (tf.TF_Q4_E2M1, 32)])
@pytest.mark.parametrize("m,n,k", [(1, 33000, 200), (7, 40000, 300), (20, 40000, 200), (90, 60000, 200)])
def test_matvec_with_many_outputs(dtype, kind, group, m, n, k):
    # two blocks of rows a wave without a gate
    check_matvec(dtype, kind, group, m, n, k)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind,group", [(tf.TF_Q4_INT, 128), (tf.TF_Q4_E2M1, 32)])
@pytest.mark.parametrize("m,n,k", [(1, 1024, 8192), (20, 1024, 8192), (33, 1040, 8200), (64, 1000, 6001), (90, 520, 4100)])
def test_matvec_with_few_outputs_and_many_inputs(dtype, kind, group, m, n, k):
    check_matvec(dtype, kind, group, m, n, k)


def check_matvec(dtype, kind, group, m, n, k):
    g = gen(m + n + k)
    q, w = random_q4(g, n, k, kind, group)
    x = randn(g, m, k, dtype=DT[dtype])
    y = torch.full((m, n), math.nan, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    ref, b = ru.product(x.double(), w[0])
    ru.check(y, ref, b, DT[dtype])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("H,I,O", [(200, 33000, 64), (64, 200, 33000)])
def test_layer_with_many_outputs_and_no_gate(dtype, H, I, O):
    D, ref, b = run_layer([[0], [1], [0, 1]], 2, H, I, O, dtype, "relu", False)
    ru.check(D, ref, b, DT[dtype])
