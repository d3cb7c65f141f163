"""What the routed operators refuse, on the host: nothing here launches a kernel."""
import ctypes

import pytest

import paper_2407_00243_amd as tf
from paper_2407_00243_amd import binding

P = 4096          # an aligned address that nothing reads


def q4(**over):
    f = dict(n_mats=1, n_rows=32, n_cols=64, codes=P, scales=P, kind=0, group=32)
    f.update(over)
    return binding.tf_q4(f["n_mats"], f["n_rows"], f["n_cols"], f["codes"], f["scales"], f["kind"], f["group"])


def csr(**over):
    f = dict(n_rows=4, n_cols=8, nnz=8, rowptr=P, colidx=P, vals=P, dtype=tf.TF_F32, on_device=1)
    f.update(over)
    return binding.tf_csr(f["n_rows"], f["n_cols"], f["nnz"], f["rowptr"], f["colidx"], f["vals"], f["dtype"],
                          f["on_device"])


def status(code):
    return binding._STATUS[code]


def test_struct_layouts():
    assert ctypes.sizeof(binding.tf_q4) == 3 * 8 + 2 * 8 + 2 * 4
    assert ctypes.sizeof(binding.tf_moe_desc) == 6 * 8 + 4 * 4


def test_q4_sizes():
    # blocks of 16 x 128 codes, scales of each group of them
    assert tf.tf_q4_sizes(1, 1, tf.TF_Q4_INT, 128) == (1024, 32)
    assert tf.tf_q4_sizes(17, 129, tf.TF_Q4_E2M1, 32, 3) == (3 * 4 * 1024, 3 * 4 * 16 * 4 * 2)
    for bad in (dict(n_rows=0), dict(n_cols=-1), dict(n_mats=0), dict(group=16), dict(group=0), dict(kind=2)):
        a = dict(n_rows=8, n_cols=8, kind=0, group=32, n_mats=1)
        a.update(bad)
        with pytest.raises(tf.TfError) as e:
            tf.tf_q4_sizes(**a)
        assert e.value.status_name == "TF_EINVAL"
    with pytest.raises(tf.TfError) as e:
        tf.tf_q4_sizes(1 << 28, 1 << 28, 0, 32, 1 << 10)
    assert e.value.status_name == "TF_EUNSUPPORTED"


@pytest.mark.parametrize("over,args,want", [
    (dict(codes=None), {}, "TF_EINVAL"), (dict(scales=P + 2), {}, "TF_EINVAL"), (dict(n_mats=2), {}, "TF_EMISMATCH"),
    (dict(group=48), {}, "TF_EINVAL"), ({}, dict(dtype=tf.TF_F64), "TF_EUNSUPPORTED"), ({}, dict(dtype=9), "TF_EUNSUPPORTED"),
    ({}, dict(X=None), "TF_EINVAL"), ({}, dict(Y=None), "TF_EINVAL"), ({}, dict(ldx=63), "TF_EINVAL"),
    ({}, dict(ldy=31), "TF_EINVAL"), ({}, dict(m=-1), "TF_EINVAL"), ({}, dict(X=P + 1), "TF_EINVAL"),
])
def test_matvec_refuses(over, args, want):
    a = dict(X=P, ldx=64, Y=P, ldy=32, m=2, dtype=tf.TF_BF16)
    a.update(args)
    w = q4(**over)
    st = tf.load_library().tf_q4_matvec(ctypes.byref(w), a["X"], a["ldx"], a["Y"], a["ldy"], a["m"], a["dtype"], None)
    assert status(st) == want and tf.tf_last_error()


def test_nothing_to_do_is_no_error():
    lib = tf.load_library()
    assert lib.tf_q4_matvec(ctypes.byref(q4()), None, 64, None, 32, 0, tf.TF_F32, None) == 0
    assert lib.tf_moe_route(None, 8, tf.TF_F32, None, 0, 1.0, ctypes.byref(csr(n_rows=0, nnz=0)), None) == 0
    assert lib.tf_moe_destroy(None) == 0


@pytest.mark.parametrize("over,args,want", [
    (dict(on_device=0), {}, "TF_EINVAL"), (dict(nnz=7), {}, "TF_EINVAL"), (dict(nnz=0), {}, "TF_EINVAL"),
    (dict(nnz=36), {}, "TF_EINVAL"), (dict(n_cols=2000), dict(ld=2000), "TF_EUNSUPPORTED"),
    (dict(nnz=4 * 65, n_cols=100), dict(ld=100), "TF_EUNSUPPORTED"), (dict(dtype=tf.TF_F64), {}, "TF_EMISMATCH"),
    (dict(rowptr=None), {}, "TF_EINVAL"), ({}, dict(scores=None), "TF_EINVAL"), ({}, dict(ld=7), "TF_EINVAL"),
    ({}, dict(dtype=tf.TF_F64), "TF_EUNSUPPORTED"), ({}, dict(scoring=4), "TF_EINVAL"), ({}, dict(scoring=-1), "TF_EINVAL"),
    ({}, dict(bias=P + 2), "TF_EINVAL"), (dict(n_rows=-1), {}, "TF_EINVAL"),
])
def test_route_refuses(over, args, want):
    a = dict(scores=P, ld=8, dtype=tf.TF_F32, bias=None, scoring=0)
    a.update(args)
    A = csr(**over)
    st = tf.load_library().tf_moe_route(a["scores"], a["ld"], a["dtype"], a["bias"], a["scoring"], 1.0, ctypes.byref(A), None)
    assert status(st) == want and tf.tf_last_error()


@pytest.mark.parametrize("over,want", [
    (dict(n_experts=0), "TF_EINVAL"), (dict(n_in=0), "TF_EINVAL"), (dict(n_hidden=-3), "TF_EINVAL"),
    (dict(n_out=0), "TF_EINVAL"), (dict(max_tokens=0), "TF_EINVAL"), (dict(max_entries=0), "TF_EINVAL"),
    (dict(dtype=tf.TF_F64), "TF_EUNSUPPORTED"), (dict(activation=4), "TF_EINVAL"), (dict(gated=2), "TF_EINVAL"),
    (dict(n_hidden=1 << 40), "TF_EUNSUPPORTED"), (dict(n_hidden=1 << 28, n_experts=1 << 20, max_entries=1 << 20), "TF_EUNSUPPORTED"),
])
def test_create_refuses(over, want):
    f = dict(n_experts=4, n_in=64, n_hidden=32, n_out=64, max_tokens=2, max_entries=4, dtype=tf.TF_BF16, activation=2, gated=1)
    f.update(over)
    d = binding.tf_moe_desc(f["n_experts"], f["n_in"], f["n_hidden"], f["n_out"], f["max_tokens"], f["max_entries"],
                            f["dtype"], f["activation"], f["gated"], 0)
    out = ctypes.c_void_p(1)
    st = tf.load_library().tf_moe_create(ctypes.byref(d), ctypes.byref(out))
    assert status(st) == want and not out.value and tf.tf_last_error()


def test_limits_of_rows_of_weights():
    lib = tf.load_library()
    w = q4(n_cols=(1 << 24) + 1)
    assert status(lib.tf_q4_matvec(ctypes.byref(w), P, 1 << 25, P, 32, 1, tf.TF_BF16, None)) == "TF_EUNSUPPORTED"
    d = binding.tf_moe_desc(4, (1 << 24) + 1, 32, 64, 2, 4, tf.TF_BF16, 2, 1, 0)
    out = ctypes.c_void_p()
    assert status(lib.tf_moe_create(ctypes.byref(d), ctypes.byref(out))) == "TF_EUNSUPPORTED"


def test_binding_checks_its_operands():
    torch = pytest.importorskip("torch")
    W = tf.Q4Matrix(32, 64, tf.TF_Q4_INT, 32, torch.empty(2048, dtype=torch.uint8), torch.empty(256, dtype=torch.uint8))
    with pytest.raises(ValueError):
        tf.Q4Matrix(32, 64, tf.TF_Q4_INT, 32, torch.empty(2047, dtype=torch.uint8), torch.empty(256, dtype=torch.uint8))
    x, y = torch.empty(2, 64), torch.empty(2, 32)
    for bad in ((torch.empty(2, 63), y), (x, torch.empty(3, 32)), (x, y.double()), (x, y.half()), (torch.empty(64, 2).t(), y),
                (torch.empty(64), y)):
        with pytest.raises((ValueError, TypeError)):
            tf.tf_q4_matvec(W, *bad)
    with pytest.raises(ValueError):
        tf.tf_q4_pack(W, torch.empty(1, 32, 63, dtype=torch.int8), torch.empty(1, 32, 2, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        tf.tf_q4_pack(W, torch.empty(1, 32, 64, dtype=torch.int8), torch.empty(1, 32, 2, dtype=torch.float16))
