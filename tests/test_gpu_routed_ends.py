"""Routed operators where their calls end: experts named again and again, the ends of the numbers' range, long launches."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2407_00243_amd as tf  # noqa: E402
import routed_util as ru  # noqa: E402
from test_gpu_routed import DT, run_layer  # noqa: E402


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
