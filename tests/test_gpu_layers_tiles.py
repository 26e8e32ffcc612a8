"""Products large enough for tiles of 256 outputs a side, which do most of a training step: whole numbers, whose sums
are exact, in all three passes; ragged edges in rows and columns, workers without rows, strided rows, weights behind
others, sums that are no whole number of loads, adding to what is there, and rows that are not finite."""
import numpy as np
import pytest

from tests.test_gpu_layers import Rows, integers, out_buffer, rows_of, say

pytestmark = pytest.mark.gpu

# (pass, row_ptr, out_features, in_features): 256 CUs give each of them tiles of 256 (asserted on the CPU)
PRODUCTS = [
    ("linear", [0, 1400, 2100], 4104, 72),
    ("linear", [0, 0, 2500, 2500, 4300], 8200, 200),
    ("linear", [2048 * i for i in range(9)], 1024, 1024),
    ("linear_grad_input", [0, 1400, 2100], 72, 4104),
    ("linear_grad_input", [0, 0, 2500, 2500, 4300], 200, 8200),
    ("linear_grad_input", [2048 * i for i in range(9)], 1024, 1024),
    ("linear_grad_weight", [0, 50, 77], 2056, 2064),
    ("linear_grad_weight", [0, 0, 300, 300, 700, 1111], 3000, 2064),
    ("linear_grad_weight", [0, 1000, 2024, 2025], 2048, 2048),
]
PARAMS = ["f32", "bf16"]


def expect(kind, x, d, w, ptr):
    """The exact results in fp64, on the GPU: rows of all workers, or [n, out, in]."""
    import torch

    out = []
    for i, (a, b) in enumerate(zip(ptr, ptr[1:])):
        if kind == "linear":
            out.append(x[a:b] @ w[i].t().contiguous())
        elif kind == "linear_grad_input":
            out.append(d[a:b] @ w[i])
        else:
            out.append(d[a:b].t().contiguous() @ x[a:b])
    return torch.stack(out) if kind == "linear_grad_weight" else torch.cat(out)


class Product:
    """bf16 rows and weights of whole numbers; worker i's live iterate is y for odd i."""

    def __init__(self, ptr, m, k, params, begin, extra):
        import torch

        n, rows = len(ptr) - 1, ptr[-1]
        self.ptr, self.m, self.k, self.n, self.rows, self.extra = ptr, m, k, n, rows, extra
        self.r = Rows(n, m * k, begin, params, stepped=np.arange(n) % 2)
        self.begin = begin
        w = integers(1, -2, 2, n, m * k)
        self.r.put(w)
        self.w = w.view(n, m, k).double()
        self.xs, self.ds = integers(2, -2, 2, rows, k), integers(3, -2, 2, rows, m)
        torch.cuda.synchronize()

    def run(self, kind, accumulate=False):
        """What the call wrote: rows, or [n, out, in]; nothing else may have changed."""
        import torch

        run, ptr, m, k, rows = self.r.run, self.ptr, self.m, self.k, self.rows
        x, _, _ = rows_of(self.xs, "bf16", self.extra)  # NaN between and behind the rows
        d, _, _ = rows_of(self.ds, "bf16", self.extra)
        if kind == "linear_grad_weight":
            self.r.grads.fill_(7.0)
            run.linear_grad_weight(self.begin, m, k, x, d, ptr, self.r.grads, accumulate=accumulate)
            got = self.r.grads[:, self.begin:self.begin + m * k].double().view(self.n, m, k)
            rest = self.r.grads.clone()
            rest[:, self.begin:self.begin + m * k] = 7.0
            assert bool((rest == 7.0).all()), "columns of other parameters were written"
            return got
        cols = m if kind == "linear" else k
        out, buf = out_buffer(rows, cols, "bf16", self.extra)
        if kind == "linear":
            run.linear(self.begin, m, k, x, ptr, out=out)
        else:
            run.linear_grad_input(self.begin, m, k, d, ptr, dx=out)
        got = out[:rows].double()
        rest = buf.view(rows + 2, cols + self.extra).clone()
        rest[:rows, :cols] = 5.0
        assert bool((rest == 5.0).all()), "something beside the rows was written"
        return got


@pytest.mark.parametrize("begin,extra", [(0, 0), (24, 8)])
@pytest.mark.parametrize("params", PARAMS)
@pytest.mark.parametrize("kind,ptr,m,k", PRODUCTS)
def test_tiles_of_256(kind, ptr, m, k, params, begin, extra):
    import torch

    say("tiles of 256", kind, ptr, m, k, params, begin, extra)
    p = Product(ptr, m, k, params, begin, extra)
    want = expect(kind, p.xs.double(), p.ds.double(), p.w, ptr)
    if kind != "linear_grad_weight":  # sums of at most 4 * 4104: exact in fp32, rounded once to bf16
        assert torch.equal(p.run(kind), want.float().bfloat16().double())
        return
    for accumulate in (False, True):
        assert torch.equal(p.run(kind, accumulate), want + 7.0 * accumulate), accumulate


@pytest.mark.parametrize("params", PARAMS)
@pytest.mark.parametrize("kind,ptr,m,k", [p for p in PRODUCTS if p[1] != [0, 50, 77]])
def test_not_finite_rows_in_tiles_of_256(kind, ptr, m, k, params):
    """NaN and infinities in some rows of one worker stay in the results of these rows (of the worker's weight)."""
    import torch

    say("not finite, tiles of 256", kind, ptr, m, k, params)
    p = Product(ptr, m, k, params, 8, 8)
    clean = expect(kind, p.xs.double(), p.ds.double(), p.w, ptr)
    worker = max(range(p.n), key=lambda i: ptr[i + 1] - ptr[i])
    a = ptr[worker] + 130
    p.xs[a:a + 70:3] = float("nan")
    p.ds[a:a + 70:3] = float("inf")
    got = p.run(kind)
    if kind == "linear_grad_weight":
        assert bool(torch.isnan(got[worker]).all())
        others = [i for i in range(p.n) if i != worker]
        assert torch.equal(got[others], clean[others])
        return
    bad = torch.zeros(p.rows, dtype=torch.bool, device="cuda")
    bad[a:a + 70:3] = True
    assert torch.equal(got[~bad], clean[~bad].float().bfloat16().double())
    assert not bool(torch.isfinite(got[bad]).any())
