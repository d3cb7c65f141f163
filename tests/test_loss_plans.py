"""Plans of the cross entropy on the host: what their calls refuse, and what they hold.  Nothing here launches a kernel."""
import ctypes

import pytest
import torch

import paper_2407_00243_amd as tf
from paper_2407_00243_amd import binding

P = 4096          # an aligned address that nothing reads


def status(code):
    return binding._STATUS[code]


def test_gradient_by_loss_refuses():
    lib = tf.load_library()
    assert status(lib.tf_xent_grad_by_loss(None, P, 8, P, 8, P, P, P, P, 4, P, 8, P, 8, None)) == "TF_EINVAL"
    t = 4
    X, W, y = torch.zeros(t, 8), torch.zeros(5, 8), torch.zeros(t, dtype=torch.int32)
    with pytest.raises(ValueError):
        tf.tf_xent_grad_by_loss(1, X, W, y, torch.zeros(t), torch.zeros(t), torch.zeros(t), X, W)


@pytest.mark.parametrize("over,want", [
    (dict(n_classes=0), "TF_EINVAL"), (dict(n_in=(1 << 22) + 1), "TF_EUNSUPPORTED"), (dict(max_rows=-1), "TF_EINVAL"),
    (dict(dtype=tf.TF_F64), "TF_EUNSUPPORTED"), (dict(gradients=2), "TF_EINVAL"),
])
def test_size_refuses_what_create_refuses(over, want):
    f = dict(n_classes=8, n_in=8, max_rows=8, dtype=tf.TF_BF16, gradients=1)
    f.update(over)
    d, out = binding.tf_xent_desc(*f.values()), ctypes.c_int64(-5)
    assert status(tf.load_library().tf_xent_size(ctypes.byref(d), ctypes.byref(out))) == want
    assert out.value == -5 and tf.tf_last_error()
    assert status(tf.load_library().tf_xent_size(None, ctypes.byref(out))) == "TF_EINVAL"
    assert status(tf.load_library().tf_xent_size(ctypes.byref(d), None)) == "TF_EINVAL"


@pytest.mark.parametrize("classes,n_in,dtype,rows,gradients,most", [
    # one row, few rows: no copy of W, no slabs that nothing is cut into
    (65536, 4096, torch.bfloat16, 1, False, 8 << 20), (65536, 4096, torch.bfloat16, 1, True, 128 << 20), (10, 16, torch.float32, 8, True, 1 << 20),
    # a batch that is only scored: X, and a small piece of W for rows that begin anywhere; a fifth of the logits
    (65536, 4096, torch.bfloat16, 4096, False, 65536 * 4096 * 2 // 5),
    # training: 2^29 bytes of g, 2^28 of W (fp32), X, slabs of dX; each less than the logits
    (131072, 4096, torch.bfloat16, 8192, True, 1200 << 20), (131072, 4096, torch.float32, 8192, True, 1600 << 20),
])
def test_workspaces_are_bounded(classes, n_in, dtype, rows, gradients, most):
    size = tf.tf_xent_size(classes, n_in, dtype, rows, gradients)
    assert 0 < size <= most
    assert size <= tf.tf_xent_size(classes, n_in, dtype, 2 * rows, gradients)
    assert tf.tf_xent_size(classes, n_in, dtype, rows, False) <= tf.tf_xent_size(classes, n_in, dtype, rows, True)
