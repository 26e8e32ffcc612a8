"""The layer calls by their names of the C ABI: the results of GASLoC's methods, bit for bit."""
import numpy as np
import pytest

import paper_2606_11081_amd as g

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("params,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_functions_are_the_methods(params, act):
    import torch

    print("functions", params, act, flush=True)
    n, vocab, width, out = 3, 50, 24, 40
    ptr = [0, 60, 60, 131]
    rows, dtype = ptr[-1], torch.float32 if act == "f32" else torch.bfloat16
    run = g.GASLoC(n, vocab * width, param_dtype=params, outer_momentum=0.0, consensus_momentum=0.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    normal = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)
    run.x[:, :run.P] = torch.empty((n, run.P), device="cuda").normal_(generator=gen)
    x, d, do = normal(rows, width), normal(rows, width), normal(rows, out)
    tokens = torch.randint(-1, vocab + 1, (rows,), dtype=torch.int32, device="cuda", generator=gen)
    grads, other = (torch.full((n, run.ld), 2.0, device="cuda") for _ in range(2))
    res = lambda cols: torch.empty((rows, cols), dtype=dtype, device="cuda")

    def space(need):
        return torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), need

    def same(a, b):
        torch.cuda.synchronize()
        return torch.equal(a, b) and torch.equal(grads, other)

    ctx, ld = run.ctx, run.ld
    o = res(width)
    g.gasloc_embedding(ctx, 0, vocab, width, 0.5, ptr, tokens, act, o, width)
    assert same(o, run.embedding(0, vocab, width, tokens, ptr, scale=0.5, dtype=act))
    ws = space(g.gasloc_embedding_grad_workspace(ctx, width, ptr))
    g.gasloc_embedding_grad(ctx, 0, vocab, width, 0.5, ptr, tokens, act, d, width, grads, ld, 1, *ws)
    run.embedding_grad(0, vocab, width, tokens, ptr, d, other, scale=0.5, accumulate=True)
    assert same(d, d) and not bool((grads[:, :run.P] == 2.0).all())

    o, stats = res(width), torch.empty((rows, 2), device="cuda")
    g.gasloc_layer_norm(ctx, 0, width, width, 1e-5, ptr, x, width, act, o, width, stats)
    h, kept = run.layer_norm(0, width, width, x, ptr)
    assert same(o, h) and torch.equal(stats, kept)
    ws = space(g.gasloc_layer_norm_grad_workspace(ctx, width, ptr))
    g.gasloc_layer_norm_grad(ctx, 0, width, width, ptr, x, width, stats, d, width, act, o, width, grads, ld, 0, *ws)
    assert same(o, run.layer_norm_grad(0, width, width, x, ptr, stats, d, other))

    ws = space(g.gasloc_linear_workspace(ctx, out, width, ptr, act))
    o = res(out)
    g.gasloc_linear(ctx, 0, out, width, ptr, x, width, act, o, out, *ws)
    assert same(o, run.linear(0, out, width, x, ptr))
    o = res(width)
    g.gasloc_linear_grad_input(ctx, 0, out, width, ptr, do, out, act, o, width, *ws)
    assert same(o, run.linear_grad_input(0, out, width, do, ptr))
    g.gasloc_linear_grad_weight(ctx, 0, out, width, ptr, x, width, do, out, act, grads, ld, 0, *ws)
    run.linear_grad_weight(0, out, width, x, do, ptr, other)
    assert same(d, d)
    assert run.ctx in g.gasloc._workers
    run.close()


def test_gradients_in_columns_of_a_larger_tensor():
    """The layers write them and the local steps read them as if the tensor held nothing else."""
    import torch

    n, width = 3, 16
    cols = width * width
    ptr = [0, 4, 4, 13]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    start = torch.empty(cols, device="cuda").normal_(generator=gen)
    x, d = (torch.empty((13, width), device="cuda").normal_(generator=gen) for _ in range(2))
    states = []
    for view in (False, True):
        run = g.GASLoC(n, cols, topology="ring")
        run.set_params(start)
        grads = torch.full((n, 100 + cols + 60), float("nan"), device="cuda")[:, 100:100 + cols] if view else \
            torch.full((n, cols), float("nan"), device="cuda")
        for t in range(2):
            run.linear_grad_weight(0, width, width, x, d, ptr, grads)
            run.local_step(grads, 1e-2)
            run.linear_grad_weight(0, width, width, d, x, ptr, grads)
            run.local_step_gossip_round(grads, 1e-2, t)
        torch.cuda.synchronize()
        states.append([run.bufs[k][:, :cols].clone() for k in ("x", "m", "v", "u", "zp")])
        run.close()
    for a, b in zip(*states):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
