"""How large products are cut (no GPU): those that the GPU tests mean for tiles of 256 take them."""
import ctypes

import numpy as np
import pytest

from tests.test_gpu_layers_tiles import PRODUCTS
from tests.test_layers_host import BF16, F32, OK, Context, call, calls, shim  # noqa: F401 (shim is a fixture)


def plan_of(shim, kind, ptr, m, k, params, act, begin=0, extra=0):  # noqa: F811
    """What the call is cut into: tile, vec, chunk, then n + 1 starts of tiles."""
    n = len(ptr) - 1
    ptr = np.array(ptr, np.int64)
    ctx = Context(shim, n=n, P=begin + m * k + 8, dtype=params)
    size = ctypes.c_size_t()
    assert shim.gasloc_linear_workspace(ctx.c, m, k, ptr.ctypes.data, act, ctypes.byref(size)) == OK
    lds = dict(x_ld=k + extra, dx_ld=k + extra, out_ld=m + extra, dout_ld=m + extra,
               grad_ld=(begin + m * k + 11) // 4 * 4)
    changes = {key: lds[key] for key in calls(ptr)["gasloc_" + kind] if key in lds}
    assert call(ctx, "gasloc_" + kind, ptr=ptr, act=act, weight=begin, out_features=m, in_features=k,
                workspace_bytes=size.value, **changes) == OK, shim.shim_error()
    plan = np.zeros(3 + 3 * n + 2, np.int64)
    shim.shim_linear_plan(n, plan.ctypes.data_as(ctypes.c_void_p))
    return [int(v) for v in plan]


@pytest.mark.parametrize("params", [F32, BF16])
@pytest.mark.parametrize("begin,extra", [(0, 0), (24, 8), (8, 8)])
@pytest.mark.parametrize("kind,ptr,m,k", PRODUCTS)
def test_these_products_take_tiles_of_256(shim, kind, ptr, m, k, begin, extra, params):  # noqa: F811
    plan = plan_of(shim, kind, ptr, m, k, params, BF16, begin, extra)
    assert plan[0] == 256 and plan[1] == 1 and plan[2] == 0


def test_some_of_them_make_more_than_one_round(shim):  # noqa: F811
    """Two tiles per CU and more, for each pass."""
    for kind in ("linear", "linear_grad_input", "linear_grad_weight"):
        tiles = [plan_of(shim, *p, F32, BF16)[3 + len(p[1]) - 1] for p in PRODUCTS if p[0] == kind]
        assert max(tiles) >= 512 and min(tiles) < 256, (kind, tiles)
