"""Layer operators on the GPU where values, not sizes, are at the edge of what fp32 holds."""
import numpy as np
import pytest

from tests import layers_reference as ref
from tests.test_gpu_layers import TYPES, Rows, close, normal, rows_of, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("width", [1, 3, 64, 129, 321, 1023, 2049, 8193, 16_383, 16_384])
def test_layer_norm_grad_of_large_constant_rows(width, params, act):
    """Rows of 2^100 with a small eps: xh is 0 in every column, though mean * rstd is beyond fp32.  Nothing but the
    columns of the row may count in its means, whatever its width."""
    import torch

    say("large constant rows", width, params, act)
    ptr = np.array([0, 3, 3, 8])
    n, rows, eps = 3, 8, 1e-20
    r = Rows(n, 2 * width, 0, params)
    gain = r.put(1 + 0.1 * normal(1, n, width))
    x, xs, _ = rows_of(torch.full((rows, width), 2.0 ** 100, device="cuda"), act)
    dout, d, _ = rows_of(normal(2, rows, width), act)
    stats = torch.tensor([[2.0 ** 100, eps ** -0.5]] * rows, dtype=torch.float32, device="cuda")
    dx = r.run.layer_norm_grad(0, width, width, x, ptr, stats, dout, r.grads)
    want = ref.layer_norm_grad(xs, stats.double().cpu().numpy(), gain, d, ptr, act)
    torch.cuda.synchronize()
    close(dx.double().cpu().numpy(), want[0], want[1], "dx")
    got = r.gradient()
    assert not got[:, :width].any()
    close(got[:, width:], want[4], want[5], "dbias")
