"""Every pass of the layer operators on rows that lie behind 2^32 bytes of their activation."""
import numpy as np
import pytest

import paper_2606_11081_amd as g
from tests import layers_reference as ref
from tests.test_gpu_layers import close, say

pytestmark = pytest.mark.gpu

N, ROWS, LD, WIDTH, OUT, LAST = 2, 60_000, 40_000, 64, 96, 59_000
PTR = np.array([0, LAST, ROWS])


def long_rows(cols, seed=None):
    """[ROWS, cols] bf16 rows of LD elements each (4.8 GB), filled with whole numbers if a seed is given."""
    import torch

    t = torch.empty((ROWS, LD), dtype=torch.bfloat16, device="cuda")[:, :cols]
    if seed is not None:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        t.copy_(torch.randint(-3, 4, (ROWS, cols), device="cuda", generator=gen))
    return t


@pytest.fixture(scope="module")
def run():
    import torch

    run = g.GASLoC(N, OUT * WIDTH, outer_momentum=0.0, consensus_momentum=0.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    run.x[:, :OUT * WIDTH] = torch.randint(-3, 4, (N, OUT * WIDTH), device="cuda", generator=gen).float()
    yield run
    run.close()


def weights(run):
    return run.x[:, :OUT * WIDTH].view(N, OUT, WIDTH)


def test_input_gradient(run):
    import torch

    say("long activations: input gradient")
    d, dx = long_rows(OUT, 2), long_rows(WIDTH)
    run.linear_grad_input(0, OUT, WIDTH, d, PTR, dx=dx)
    for i, (a, b) in enumerate(zip(PTR, PTR[1:])):  # whole numbers: exact in fp32, rounded once
        assert torch.equal(dx[a:b], (d[a:b].double().contiguous() @ weights(run)[i].double()).float().bfloat16())


def test_norm_and_its_gradients(run):
    import torch

    say("long activations: norm")
    x, h = long_rows(WIDTH, 3), long_rows(WIDTH)
    gain, bias = (weights(run)[:, k].double().cpu().numpy() for k in (0, 1))
    _, stats = run.layer_norm(0, WIDTH, WIDTH, x, PTR, out=h)
    xs = x.double().cpu().numpy()
    want, bound, want_stats, stats_bound = ref.layer_norm(xs, gain, bias, PTR, np.float64(np.float32(1e-5)), "bf16")
    close(h.double().cpu().numpy(), want, bound, "out")
    close(stats.double().cpu().numpy(), want_stats, stats_bound, "stats")

    dout, dx = long_rows(WIDTH, 4), h
    grads = torch.zeros((N, run.ld), device="cuda")
    run.layer_norm_grad(0, WIDTH, WIDTH, x, PTR, stats, dout, grads, dx=dx)
    want = ref.layer_norm_grad(xs, stats.double().cpu().numpy(), gain, dout.double().cpu().numpy(), PTR, "bf16")
    close(dx.double().cpu().numpy(), want[0], want[1], "dx")
    got = grads[:, :2 * WIDTH].double().cpu().numpy()
    close(got[:, :WIDTH], want[2], want[3], "dgain")
    close(got[:, WIDTH:], want[4], want[5], "dbias")
