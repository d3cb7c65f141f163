"""What the Python calls of the routed operators refuse of their operands, before the library sees an address."""
import pytest

import paper_2407_00243_amd as tf

torch = pytest.importorskip("torch")

T, E, K, H, I = 4, 8, 2, 64, 32


def routing(**over):
    f = dict(rowptr=torch.zeros(T + 1, dtype=torch.int32), colidx=torch.zeros(T * K, dtype=torch.int32),
             vals=torch.zeros(T * K))
    f.update(over)
    return tf.DeviceCsr(T, E, f["rowptr"], f["colidx"], f["vals"])


def plan():
    """A plan as far as the checks of its operands go (no device is needed for them)."""
    p = object.__new__(tf.MoePlan)
    p.handle, p.n_experts, p.n_in, p.n_hidden, p.n_out, p.dtype, p.gated = None, E, H, I, H, tf.TF_F32, True
    return p


def q4(n_rows, n_cols, mats=1):
    sizes = tf.tf_q4_sizes(n_rows, n_cols, tf.TF_Q4_INT, 32, mats)
    return tf.Q4Matrix(n_rows, n_cols, tf.TF_Q4_INT, 32, *(torch.zeros(n, dtype=torch.uint8) for n in sizes), n_mats=mats)


def calls(A):
    X, D = torch.zeros(T, H), torch.zeros(T, H)
    W1, W2 = torch.zeros(E, 2 * I, H), torch.zeros(E, H, I)
    Q1, Q2 = q4(2 * I, H, E), q4(H, I, E)
    return [lambda: tf.tf_moe_route(torch.zeros(T, E), A), lambda: plan().run(A, X, W1, W2, D),
            lambda: plan().run(A, X, Q1, Q2, D), lambda: tf.tf_moe_layer(1, A, X, W1, W2, D),
            lambda: tf.tf_moe_layer_q4(1, A, X, Q1, Q2, D)]


@pytest.mark.parametrize("over,error,words", [
    (dict(colidx=torch.zeros(T * K, dtype=torch.int64)), TypeError, "int32"),
    (dict(rowptr=torch.zeros(T + 1, dtype=torch.int64)), TypeError, "int32"),
    (dict(rowptr=torch.zeros(T + 1)), TypeError, "int32"),
    (dict(vals=torch.zeros(T * K, dtype=torch.bfloat16)), TypeError, "fp32"),
    (dict(rowptr=torch.zeros(T, dtype=torch.int32)), ValueError, "hold"),
    (dict(vals=torch.zeros(T * K - 1)), ValueError, "hold"),
    (dict(rowptr=torch.zeros(2 * T + 2, dtype=torch.int32)[::2]), ValueError, "contiguous"),
    (dict(colidx=torch.zeros(2 * T * K, dtype=torch.int32)[::2]), ValueError, "contiguous"),
    (dict(vals=torch.zeros(1).expand(T * K)), ValueError, "contiguous"),
    (dict(), ValueError, "device"),
])
def test_arrays_of_a_routing_matrix(over, error, words):
    for call in calls(routing(**over)):
        with pytest.raises(error, match=words):
            call()


def test_columns_that_shrink_after_the_matrix_was_made():
    A = routing()
    A.colidx = A.colidx[:-1].contiguous()
    for call in calls(A):
        with pytest.raises(ValueError, match="hold"):
            call()


def test_operands_on_the_host():
    W = q4(32, 64)
    for call in (lambda: tf.tf_q4_matvec(W, torch.zeros(2, 64), torch.zeros(2, 32)),
                 lambda: tf.tf_q4_quantize(W, torch.zeros(1, 32, 64)),
                 lambda: tf.tf_q4_unpack(W, torch.zeros(1, 32, 64)),
                 lambda: tf.tf_q4_pack(W, torch.zeros(1, 32, 64, dtype=torch.int8), torch.zeros(1, 32, 2, dtype=torch.bfloat16)),
                 lambda: tf.tf_moe_route(torch.zeros(T, E), routing(), bias=torch.zeros(E))):
        with pytest.raises(ValueError, match="device"):
            call()


def test_arrays_of_a_4_bit_matrix():
    sizes = tf.tf_q4_sizes(32, 64, tf.TF_Q4_INT, 32)
    codes, scales = (torch.zeros(n, dtype=torch.uint8) for n in sizes)
    for bad in ((torch.zeros(1, dtype=torch.uint8).expand(sizes[0]), scales), (codes, torch.zeros(2 * sizes[1], dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            tf.Q4Matrix(32, 64, tf.TF_Q4_INT, 32, *bad)


def test_layer_calls_by_handle_look_at_their_rows():
    A = routing()
    X, W1, W2 = torch.zeros(T, H), torch.zeros(E, 2 * I, H), torch.zeros(E, H, I)
    for X, D, error in ((X[1:], X, ValueError), (X, X[1:], ValueError), (X, X.bfloat16(), TypeError), (X, X.t().contiguous().t(), ValueError)):
        with pytest.raises(error):
            tf.tf_moe_layer(1, A, X, W1, W2, D)


def test_numpy_arrays_are_on_the_host():
    np = pytest.importorskip("numpy")
    address = 4096
    W = tf.Q4Matrix(32, 64, tf.TF_Q4_INT, 32, address, address)          # addresses are the caller's affair
    assert W.device is None
    for codes, scales in ((np.zeros((1, 32, 64), np.int8), address), (address, np.zeros((1, 32, 2), np.uint16))):
        with pytest.raises(ValueError, match="device"):
            tf.tf_q4_pack(W, codes, scales)
    sizes = tf.tf_q4_sizes(32, 64, tf.TF_Q4_INT, 32)
    host = tf.Q4Matrix(32, 64, tf.TF_Q4_INT, 32, *(np.zeros(n, np.uint8) for n in sizes))
    with pytest.raises(ValueError, match="device"):
        tf.tf_q4_pack(host, address, address)
