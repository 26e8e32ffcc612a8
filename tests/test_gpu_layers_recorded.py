"""Recorded layer calls between local steps: which iterate a recording reads."""
import numpy as np
import pytest

import paper_2606_11081_amd as g
from tests.test_gpu_layers_run import P, VOCAB, backward, forward, start_params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("params,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_one_recording_before_and_one_after_the_first_local_step(params, act):
    """A recording keeps the iterates that were live when it was made: x for workers that have not stepped since the
    round, y for the others.  So a program with several local steps per round records its step twice, once for the
    first of a round and once for those after it; replayed in their places both give the eager results."""
    import torch

    print("recorded and live iterates", params, act, flush=True)
    n, steps = 3, 3
    ptr = np.array([0, 33, 50, 117])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        run = g.GASLoC(n, P, topology="ring", param_dtype=params, stream=stream)
        run.set_params(start_params(n, 4).cuda())
        dtype = torch.float32 if act == "f32" else torch.bfloat16
        tokens = torch.zeros(int(ptr[-1]), dtype=torch.int32, device="cuda")
        dlogits = torch.zeros((int(ptr[-1]), VOCAB), dtype=dtype, device="cuda")
        grads = torch.zeros((n, run.ld), device="cuda")
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)

        def inputs():
            tokens.copy_(torch.randint(0, VOCAB, tokens.shape, device="cuda", generator=gen).int())
            dlogits.copy_(torch.empty(dlogits.shape, device="cuda").normal_(0.0, 0.1, generator=gen))

        def step(into):
            kept = forward(run, tokens, ptr, act)
            backward(run, tokens, ptr, kept, dlogits, into)
            return kept

        def record():
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                kept = step(grads)
            return graph, kept

        inputs()
        step(grads)  # warm-up
        graphs = [record()]
        run.local_step(grads, 1e-3)
        graphs.append(record())
        run.gossip_round(0)
        for t in range(1, 4):
            for h in range(steps):
                inputs()
                other = torch.zeros_like(grads)
                eager = step(other)
                graph, kept = graphs[min(h, 1)]
                grads.zero_()
                graph.replay()
                torch.cuda.synchronize()
                for a, b in zip(kept, eager):
                    assert torch.equal(a, b), (t, h)
                assert torch.equal(grads, other), (t, h)
                if h > 0:  # the other recording still reads x, where the round began
                    graphs[0][0].replay()
                    torch.cuda.synchronize()
                    assert not torch.equal(graphs[0][1][0], eager[0]), (t, h)
                    grads.copy_(other)
                run.local_step(grads, 1e-2)
            run.gossip_round(t)
        run.close()
