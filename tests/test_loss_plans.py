"""Plans of the cross entropy on the host: what their calls refuse.  Nothing here launches a kernel."""
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
