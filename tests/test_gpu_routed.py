"""Router, mixture-of-experts layer and 4-bit products against their definitions in 64 bits."""
import itertools
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2407_00243_amd as tf  # noqa: E402
import routed_util as ru  # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACT = {"identity": tf.TF_ACT_IDENTITY, "relu": tf.TF_ACT_RELU, "silu": tf.TF_ACT_SILU, "gelu": tf.TF_ACT_GELU}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def stream():
    return torch.cuda.current_stream().cuda_stream


def empty_q4(n, k, kind, group, mats=1):
    cb, sb = tf.tf_q4_sizes(n, k, kind, group, mats)
    fill = lambda b: torch.full((b,), 0x5a, dtype=torch.uint8, device="cuda")       # noqa: E731
    return tf.Q4Matrix(n, k, kind, group, fill(cb), fill(sb), n_mats=mats)


def random_q4(g, n, k, kind, group, mats=1):
    lo, hi = (-7, 8) if kind == tf.TF_Q4_INT else (0, 16)
    codes = torch.randint(lo, hi, (mats, n, k), device="cuda", dtype=torch.int8, generator=g)
    scales = ((0.5 + torch.rand(mats, n, -(-k // group), device="cuda", generator=g)) / (4 * math.sqrt(k))).to(torch.bfloat16)
    q = empty_q4(n, k, kind, group, mats)
    tf.tf_q4_pack(q, codes, scales, stream())
    return q, ru.values(codes, scales, kind, group)


# ------------------------------------------------------------------------------------ 4-bit weights

@pytest.mark.parametrize("kind,group", itertools.product([tf.TF_Q4_INT, tf.TF_Q4_E2M1], [32, 64, 128]))
@pytest.mark.parametrize("mats,n,k", [(1, 1, 1), (3, 17, 129), (2, 40, 300), (1, 16, 128)])
def test_pack_and_unpack_are_exact(kind, group, mats, n, k):
    q, w = random_q4(gen(n + k), n, k, kind, group, mats)
    for dt in DT.values():
        out = torch.empty(mats, n, k, dtype=dt, device="cuda")
        tf.tf_q4_unpack(q, out, stream())
        # values have at most 4 + 8 significant bits: rounded once
        assert torch.equal(out, w.float().to(dt))


@pytest.mark.parametrize("kind,code", [(tf.TF_Q4_INT, -8), (tf.TF_Q4_INT, 8), (tf.TF_Q4_E2M1, -1), (tf.TF_Q4_E2M1, 16)])
def test_pack_refuses_codes_out_of_range(kind, code):
    q = empty_q4(20, 40, kind, 32)
    codes = torch.ones(1, 20, 40, dtype=torch.int8, device="cuda")
    scales = torch.ones(1, 20, 2, dtype=torch.bfloat16, device="cuda")
    tf.tf_q4_pack(q, codes, scales, stream())
    codes[0, 19, 39] = code
    with pytest.raises(tf.TfError) as e:
        tf.tf_q4_pack(q, codes, scales, stream())
    assert e.value.status_name == "TF_EINVAL"


@pytest.mark.parametrize("kind", [tf.TF_Q4_INT, tf.TF_Q4_E2M1])
@pytest.mark.parametrize("dtype", DT)
def test_quantize_takes_the_nearest_code(kind, dtype):
    dt, group, n, k = DT[dtype], 64, 33, 200
    w = randn(gen(7), 2, n, k, dtype=dt)
    w[0, 3] = 0
    w[1, 5, 64:128] = 0.0
    w[1, 6, 0] = 300.0
    q = empty_q4(n, k, kind, group, 2)
    tf.tf_q4_quantize(q, w, stream())
    out = torch.empty(2, n, k, device="cuda")
    tf.tf_q4_unpack(q, out, stream())
    top = 7.0 if kind == tf.TF_Q4_INT else 6.0
    pad = torch.zeros(2, n, 256, device="cuda")
    pad[..., :k] = w.float()
    s = (pad.view(2, n, 4, group).abs().amax(-1) / top).to(torch.bfloat16).float()
    ratio = (pad.view(2, n, 4, group) / s[..., None]).nan_to_num(0.0)
    if kind == tf.TF_Q4_INT:
        code = torch.round(ratio).clamp(-7, 7)
    else:
        # nearest of the eight, halfway cases to the even code
        table = ru.E2M1[:8].float().cuda()
        dist = (ratio.abs()[..., None] - table).abs()
        dist[..., 1::2] += 1e-12
        even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device="cuda")
        code = table[even_first[(dist[..., even_first]).argmin(-1)]] * torch.sign(ratio)
    ref = (code * s[..., None]).reshape(2, n, 256)[..., :k]
    assert torch.equal(out, ref)


def test_quantize_marks_groups_that_are_not_finite():
    w = torch.ones(1, 4, 96, device="cuda")
    w[0, 1, 40] = math.inf
    w[0, 2, 3] = math.nan
    q = empty_q4(4, 96, tf.TF_Q4_INT, 32)
    tf.tf_q4_quantize(q, w, stream())
    out = torch.empty_like(w)
    tf.tf_q4_unpack(q, out, stream())
    bad = torch.zeros_like(w, dtype=torch.bool)
    bad[0, 1, 32:64] = True
    bad[0, 2, :32] = True
    assert torch.equal(torch.isnan(out), bad)


# --------------------------------------------------------------------------------------- product

@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind,group", itertools.product([tf.TF_Q4_INT, tf.TF_Q4_E2M1], [32, 64, 128]))
@pytest.mark.parametrize("m,n,k", [(1, 16, 128), (1, 1, 1), (2, 33, 127), (5, 70, 515), (17, 48, 1100), (70, 37, 260)])
def test_matvec(dtype, kind, group, m, n, k):
    g = gen(m * 1000 + n)
    q, w = random_q4(g, n, k, kind, group)
    x = randn(g, m, k, dtype=DT[dtype])
    y = torch.full((m, n), math.nan, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    ref, b = ru.product(x.double(), w[0])
    ru.check(y, ref, b, DT[dtype])


@pytest.mark.parametrize("dtype", DT)
def test_matvec_with_rows_apart(dtype):
    g = gen(3)
    q, w = random_q4(g, 50, 200, tf.TF_Q4_INT, 64)
    x = randn(g, 9, 421, dtype=DT[dtype])[:, 7:207]
    y = torch.full((9, 91), -3.0, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y[:, 11:61], stream())
    ref, b = ru.product(x.double(), w[0])
    ru.check(y[:, 11:61], ref, b, DT[dtype])
    assert (y[:, :11] == -3).all() and (y[:, 61:] == -3).all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind", [tf.TF_Q4_INT, tf.TF_Q4_E2M1])
def test_matvec_keeps_infinities_in_their_rows(dtype, kind):
    g = gen(4)
    n, k = 40, 300
    codes = torch.full((1, n, k), 3, dtype=torch.int8, device="cuda")
    codes[0, ::2] = -3 if kind == tf.TF_Q4_INT else 11
    scales = torch.full((1, n, -(-k // 32)), 0.25, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, k, kind, 32)
    tf.tf_q4_pack(q, codes, scales, stream())
    w = ru.values(codes, scales, kind, 32)[0]
    x = randn(g, 4, k, dtype=DT[dtype])
    x[1, 299], x[2, 5] = math.inf, math.nan
    # beyond the row: what lies behind X must not be read into it
    wide = torch.full((4, 512), math.nan, dtype=DT[dtype], device="cuda")
    wide[:, :k] = x
    y = torch.empty(4, n, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, wide[:, :k], y, stream())
    ref, b = ru.product(x.double(), w)
    ru.check(y[[0, 3]], ref[[0, 3]], b[[0, 3]], DT[dtype])
    assert torch.equal(y[1].double(), ref[1]) and torch.isinf(ref[1]).all()
    assert torch.isnan(y[2]).all()


def test_matvec_keeps_the_smallest_and_the_largest_numbers():
    # fp16 below its normal range, bf16 and fp32 near the ends of theirs
    n, k = 16, 128
    codes = torch.ones(1, n, k, dtype=torch.int8, device="cuda")
    scales = torch.ones(1, n, 1, dtype=torch.bfloat16, device="cuda")
    q = empty_q4(n, k, tf.TF_Q4_INT, 128)
    tf.tf_q4_pack(q, codes, scales, stream())
    for dt, v in ((torch.float16, 2.0 ** -24), (torch.float16, 500.0), (torch.bfloat16, 2.0 ** -100),
                  (torch.bfloat16, 2.0 ** 120), (torch.float32, 1.1 * 2.0 ** -100), (torch.float32, 1.3 * 2.0 ** 120)):
        x = torch.full((1, k), v, dtype=dt, device="cuda")
        y = torch.empty(1, n, dtype=dt, device="cuda")
        tf.tf_q4_matvec(q, x, y, stream())
        ref, b = ru.product(x.double(), ru.values(codes, scales, 0, 128)[0])
        ru.check(y, ref, b, dt, f"{dt} {v}")
    x = torch.zeros(1, k, device="cuda")
    x[0, 5] = torch.finfo(torch.float32).max
    y = torch.empty(1, n, device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    assert (y == x[0, 5]).all()


# ---------------------------------------------------------------------------------------- router

def route_ref(scores, bias, k, scoring, scale):
    T, E = scores.shape
    l = torch.where(torch.isnan(scores.double()), -math.inf, scores.double())
    key = l if bias is None else (l.float() + bias).double()
    key = torch.where(torch.isnan(key), -math.inf, key)
    cols, vals = torch.full((T, k), -1), torch.zeros(T, k, dtype=torch.float64)
    key, l = key.cpu(), l.cpu()
    for t in range(T):
        order = [e for e in sorted(range(E), key=lambda e: (-key[t, e].item(), e)) if key[t, e] > -math.inf][:k]
        if not order:
            continue
        s = l[t, order]
        if scoring in (tf.TF_ROUTE_SOFTMAX, tf.TF_ROUTE_SOFTMAX_TOP):
            over = l[t] if scoring == tf.TF_ROUTE_SOFTMAX else s
            w = torch.exp(s - over.max()) / torch.exp(over - over.max()).sum()
        else:
            w = torch.sigmoid(s)
            if scoring == tf.TF_ROUTE_SIGMOID_TOP:
                w = w / w.sum()
        cols[t, :len(order)] = torch.tensor(order)
        vals[t, :len(order)] = w * scale
    return cols, vals


def run_route(scores, bias, k, scoring, scale):
    T, E = scores.shape
    A = tf.DeviceCsr(T, E, torch.full((T + 1,), -9, dtype=torch.int32, device="cuda"),
                     torch.full((T * k,), -9, dtype=torch.int32, device="cuda"),
                     torch.full((T * k,), math.nan, device="cuda"))
    tf.tf_moe_route(scores, A, scoring, bias=bias, scale=scale, stream=stream())
    assert A.rowptr.tolist() == list(range(0, T * k + 1, k))
    return A.colidx.view(T, k).cpu().long(), A.vals.view(T, k).cpu()


@pytest.mark.parametrize("scoring", range(4))
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T,E,k,bias", [(1, 1, 1, False), (1, 64, 6, False), (5, 65, 8, True), (3, 8, 8, False),
                                        (130, 128, 2, True), (7, 256, 8, False), (2, 1000, 64, True)])
def test_route(scoring, dtype, T, E, k, bias):
    g = gen(T + E)
    scores = randn(g, T, E + 3, dtype=DT[dtype])[:, :E]
    # ties: a few values, many times
    if T > 1:
        scores[1] = torch.randint(-2, 3, (E,), device="cuda", generator=g).to(DT[dtype])
        scores[0, ::3] = -math.inf
        scores[T - 1, E // 2:] = math.nan
    b = randn(g, E) if bias else None
    cols, vals = run_route(scores, b, k, scoring, 2.5)
    rcols, rvals = route_ref(scores, b, k, scoring, 2.5)
    assert torch.equal(cols, rcols)
    # sums of up to 1024 numbers of one sign, functions good to a few units, a division
    assert ((vals.double() - rvals).abs() <= 2.0 ** -24 * (40 + 8 * scores[torch.isfinite(scores)].abs().max().item()) * rvals).all()


def test_route_with_closed_experts():
    scores = torch.full((4, 70), -math.inf, device="cuda")
    scores[1, 69] = 0.0
    scores[2, [0, 64]] = torch.tensor([-0.0, 0.0], device="cuda")        # equal: the lower one first
    scores[3] = math.nan
    for scoring in range(4):
        cols, vals = run_route(scores, None, 3, scoring, 1.0)
        assert cols.tolist() == [[-1, -1, -1], [69, -1, -1], [0, 64, -1], [-1, -1, -1]]
        share = {2: (0.5, 0.5)}.get(scoring, (1.0, 0.5))
        assert vals.tolist() == [[0, 0, 0], [share[0], 0, 0], [share[1], share[1], 0], [0, 0, 0]]


# ----------------------------------------------------------------------------------------- layer

def csr(rows, n_experts, values=None, seed=5):
    """rows: for each token its experts."""
    rowptr = [0]
    for r in rows:
        rowptr.append(rowptr[-1] + len(r))
    cols = [e for r in rows for e in r]
    g = gen(seed)
    vals = torch.rand(max(1, len(cols)), device="cuda", generator=g)[:len(cols)] if values is None else values
    A = tf.DeviceCsr(len(rows), n_experts, torch.tensor(rowptr, dtype=torch.int32, device="cuda"),
                     torch.tensor(cols, dtype=torch.int32, device="cuda"), vals)
    return A, rowptr, cols


def run_layer(rows, E, H, I, O, dtype, activation="silu", gated=True, quant=None, X=None, seed=1, values=None):
    dt, g, T = DT[dtype], gen(seed), len(rows)
    A, rowptr, cols = csr(rows, E, values)
    X = randn(g, T, H, dtype=dt) if X is None else X
    first = I * (2 if gated else 1)
    if quant:
        W1, v1 = random_q4(g, first, H, *quant, mats=E)
        W2, v2 = random_q4(g, O, I, *quant, mats=E)
    else:
        W1 = (randn(g, E, first, H) / math.sqrt(H)).to(dt)
        W2 = (randn(g, E, O, I) / math.sqrt(I)).to(dt)
        v1, v2 = W1.double(), W2.double()
    inside = lambda e: 0 <= e < E                                     # noqa: E731
    with tf.MoePlan(E, H, I, dt, max_tokens=T + 1, max_entries=len(cols) + 1, n_out=O, activation=ACT[activation],
                    gated=gated) as plan:
        D = torch.full((T, O), math.nan, dtype=dt, device="cuda")
        plan.run(A, X, W1, W2, D, stream())
        again = torch.full((T, O), math.nan, dtype=dt, device="cuda")
        plan.run(A, X, W1, W2, again, stream())
        torch.cuda.synchronize()
    assert torch.equal(D, again) or not torch.isfinite(D).all()
    ref, b = ru.layer(X.double(), rowptr, cols, A.vals.tolist(), lambda e: v1[e] if inside(e) else None,
                      lambda e: v2[e], activation, gated, dt)
    if ref is None:
        ref = torch.zeros(T, O, dtype=torch.float64, device="cuda")
        b = torch.zeros_like(ref)
    return D, ref, b


def some_rows(T, E, k, seed=11):
    g = torch.Generator().manual_seed(seed)
    return [torch.randperm(E, generator=g)[:k].tolist() for _ in range(T)]


QUANT = [None] + list(itertools.product([tf.TF_Q4_INT, tf.TF_Q4_E2M1], [32, 64, 128]))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("quant", QUANT)
@pytest.mark.parametrize("T,E,k,H,I,O", [(1, 4, 2, 256, 128, 256), (9, 5, 3, 133, 71, 90), (40, 3, 2, 64, 40, 48)])
def test_layer(dtype, quant, T, E, k, H, I, O):
    for gated, activation in ((True, "silu"), (False, "gelu")):
        D, ref, b = run_layer(some_rows(T, E, k), E, H, I, O, dtype, activation, gated, quant)
        ru.check(D, ref, b, DT[dtype], f"gated {gated}")


@pytest.mark.parametrize("activation", ACT)
@pytest.mark.parametrize("gated", [True, False])
def test_layer_activations(activation, gated):
    D, ref, b = run_layer(some_rows(6, 4, 2), 4, 96, 64, 80, "f32", activation, gated)
    ru.check(D, ref, b, torch.float32)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("quant", [None, (tf.TF_Q4_INT, 64)])
@pytest.mark.parametrize("rows,E", [
    ([[]], 3),                                            # nothing at all
    ([[], [], []], 2),
    ([[2], [], [0, 1, 2], [], []], 3),                    # rows of different lengths, the last ones empty
    ([[1, 1, 0], [1]], 4),                                # an expert twice in a row
    ([[-1, 0], [5, -7], [4, 3], [-1, -1]], 5),            # columns that are no experts
    ([[0]] * 90, 1),                                      # one expert, more entries than are multiplied at a time
    ([[0, 1]] * 17 + [[1]] * 40 + [[]] + [[0]] * 9, 2),
    ([[i % 200] for i in range(150)], 200),               # many experts, one entry each
])
def test_layer_routing(dtype, quant, rows, E):
    D, ref, b = run_layer(rows, E, 72, 48, 56, dtype, quant=quant)
    ru.check(D, ref, b, DT[dtype])
    for t, r in enumerate(rows):
        if not any(0 <= e < E for e in r):
            assert (D[t] == 0).all()


@pytest.mark.parametrize("dtype", DT)
def test_layer_keeps_infinities_in_their_rows(dtype):
    X = randn(gen(2), 5, 100, dtype=DT[dtype])
    X[1, 99], X[3, 0] = math.nan, math.inf
    D, ref, b = run_layer([[0, 1]] * 5, 3, 100, 64, 40, dtype, X=X)
    ok = [0, 2, 4]
    ru.check(D[ok], ref[ok], b[ok], DT[dtype])
    assert not torch.isfinite(D[[1, 3]]).any()


@pytest.mark.parametrize("quant", [None, (tf.TF_Q4_E2M1, 32)])
def test_layer_holds_hidden_numbers_beyond_fp16(quant):
    # a gate and what it multiplies of some thousands each: their product passes 65504
    X = 2000.0 * randn(gen(2), 3, 64, dtype=torch.float16)
    values = torch.full((6,), 2.0 ** -12, device="cuda")
    D, ref, b = run_layer([[0, 1]] * 3, 2, 64, 96, 40, "f16", quant=quant, X=X, values=values)
    assert torch.isfinite(D).all()
    ru.check(D, ref, b, torch.float16)


def test_layer_with_rows_apart_on_another_stream():
    E, H, I, T = 4, 70, 50, 6
    g = gen(9)
    W1, W2 = (randn(g, E, 2 * I, H) / 8).bfloat16(), (randn(g, E, H, I) / 7).bfloat16()
    X, D = randn(g, T, 200, dtype=torch.bfloat16), torch.full((T, 150), 7.0, dtype=torch.bfloat16, device="cuda")
    A, rowptr, cols = csr(some_rows(T, E, 2), E)
    other = torch.cuda.Stream()
    with tf.MoePlan(E, H, I, "torch.bfloat16", T, 2 * T) as plan:
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            plan.run(A, X[:, 5:75], W1, W2, D[:, 3:73], stream())
        other.synchronize()
    ref, b = ru.layer(X[:, 5:75].double(), rowptr, cols, A.vals.tolist(), lambda e: W1[e].double(),
                      lambda e: W2[e].double(), "silu", True, torch.bfloat16)
    ru.check(D[:, 3:73], ref, b, torch.bfloat16)
    assert (D[:, :3] == 7).all() and (D[:, 73:] == 7).all()


def test_layer_with_weights_beyond_32_bit_offsets():
    # two experts of 2.1 GiB in the first product; the last rows of the last expert
    E, H, I = 2, 8192, 140000
    W1 = torch.empty(E, I, H, dtype=torch.bfloat16, device="cuda").normal_(0, 0.01, generator=gen(1))
    W2 = torch.empty(E, 8, I, dtype=torch.bfloat16, device="cuda").normal_(0, 0.01, generator=gen(2))
    X = randn(gen(3), 1, H, dtype=torch.bfloat16)
    A, _, _ = csr([[1]], E, torch.ones(1, device="cuda"))
    with tf.MoePlan(E, H, I, "torch.bfloat16", 1, 1, n_out=8, activation=tf.TF_ACT_RELU, gated=False) as plan:
        D = torch.empty(1, 8, dtype=torch.bfloat16, device="cuda")
        plan.run(A, X, W1, W2, D, stream())
        torch.cuda.synchronize()
    ref, b = ru.layer(X.double(), [0, 1], [1], [1.0], lambda e: W1[e].double(), lambda e: W2[e].double(), "relu", False,
                      torch.bfloat16)
    ru.check(D, ref, b, torch.bfloat16)


def test_route_and_layer_in_a_graph():
    """The router and the layer captured once, replayed over changing inputs with eager work in between."""
    E, k, H, I, T = 16, 4, 128, 96, 5
    g = gen(21)
    W1, W2 = (randn(g, E, 2 * I, H) / 11).bfloat16(), (randn(g, E, H, I) / 10).bfloat16()
    scores, X = randn(g, T, E), randn(g, T, H, dtype=torch.bfloat16)
    A = tf.DeviceCsr(T, E, torch.empty(T + 1, dtype=torch.int32, device="cuda"),
                     torch.empty(T * k, dtype=torch.int32, device="cuda"), torch.empty(T * k, device="cuda"))
    D = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    with tf.MoePlan(E, H, I, "torch.bfloat16", T, T * k) as plan:
        def once():
            tf.tf_moe_route(scores, A, tf.TF_ROUTE_SOFTMAX_TOP, stream=stream())
            plan.run(A, X, W1, W2, D, stream())
        once()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            once()
        for i in range(4):
            scores.copy_(randn(g, T, E))
            X.copy_(randn(g, T, H, dtype=torch.bfloat16))
            torch.cuda.synchronize()
            once()
            torch.cuda.synchronize()
            eager = D.clone()
            D.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(D, eager) and eager.abs().sum() > 0


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind,group", [(tf.TF_Q4_INT, 128), (tf.TF_Q4_E2M1, 32)])
@pytest.mark.parametrize("m,n,k", [(3, 50, 9001), (12, 40, 5000), (30, 33, 4111), (64, 530, 2500), (100, 20, 3000), (1, 4097, 640)])
def test_matvec_over_many_chunks(dtype, kind, group, m, n, k):
    g = gen(m + n)
    q, w = random_q4(g, n, k, kind, group)
    x = randn(g, m, k, dtype=DT[dtype])
    y = torch.full((m, n), math.nan, dtype=DT[dtype], device="cuda")
    tf.tf_q4_matvec(q, x, y, stream())
    ref, b = ru.product(x.double(), w[0])
    ru.check(y, ref, b, DT[dtype])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("quant", [None, (tf.TF_Q4_E2M1, 32), (tf.TF_Q4_INT, 128)])
@pytest.mark.parametrize("T,E,k,H,I", [
    (8, 100, 8, 1500, 530),        # 64 entries: the most that every wave looks for by itself
    (13, 90, 5, 2100, 300),        # 65
    (16, 30, 20, 520, 1100),       # more entries than the sum over them finds in LDS
    (17, 12, 3, 900, 260),         # more tokens than the last workgroups add up
    (300, 6, 2, 200, 136),         # more row pointers than fit LDS, more entries than are multiplied at a time
])
def test_layer_at_the_borders_of_its_cases(dtype, quant, T, E, k, H, I):
    rows = some_rows(T, E, k)
    rows[T // 2] = rows[T // 2][:1]                # (rows of different lengths)
    D, ref, b = run_layer(rows, E, H, I, H, dtype, quant=quant)
    ru.check(D, ref, b, DT[dtype])


def test_layer_with_unaligned_rows():
    g = gen(31)
    E, H, I, T = 3, 77, 41, 5
    for dt in DT.values():
        W1, W2 = (randn(g, E, 2 * I, H) / 9).to(dt), (randn(g, E, H, I) / 6).to(dt)
        X = randn(g, T * 79 + 1, dtype=dt)[1:].as_strided((T, H), (79, 1))
        D = torch.zeros(T * 81 + 3, dtype=dt, device="cuda")[3:].as_strided((T, H), (81, 1))
        A, rowptr, cols = csr(some_rows(T, E, 2), E)
        with tf.MoePlan(E, H, I, dt, T, 2 * T) as plan:
            plan.run(A, X, W1, W2, D, stream())
            torch.cuda.synchronize()
        ref, b = ru.layer(X.double(), rowptr, cols, A.vals.tolist(), lambda e: W1[e].double(), lambda e: W2[e].double(),
                          "silu", True, dt)
        ru.check(D, ref, b, dt)
