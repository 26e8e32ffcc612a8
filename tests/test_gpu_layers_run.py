"""The layer operators as a training program uses them: whole steps of a small
tied model for several workers between local steps and rounds, recorded in a
HIP graph, called from another stream than the context's, at columns and rows
whose offsets pass 32 bits, and twice with the same bits."""
import numpy as np
import pytest

import paper_2606_11081_amd as g

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


VOCAB, WIDTH, HIDDEN, EPS = 89, 40, 72, 1e-5
TABLE, GAIN = 0, VOCAB * WIDTH
BIAS = GAIN + WIDTH
UP = BIAS + WIDTH + 8
DOWN = UP + HIDDEN * WIDTH
P = DOWN + WIDTH * HIDDEN + 5
SCALE = 0.75


def forward(run, tokens, ptr, act):
    """Embedding, norm, two linear layers around a square, then logits with the embedding table."""
    import torch

    e = run.embedding(TABLE, VOCAB, WIDTH, tokens, ptr, scale=SCALE, dtype=act)
    h, stats = run.layer_norm(GAIN, BIAS, WIDTH, e, ptr, eps=EPS)
    u = run.linear(UP, HIDDEN, WIDTH, h, ptr)
    s = (u.float() * u.float()).to(u.dtype)
    d = run.linear(DOWN, WIDTH, HIDDEN, s, ptr)
    logits = run.linear(TABLE, VOCAB, WIDTH, d, ptr)
    return e, h, stats, u, s, d, logits


def backward(run, tokens, ptr, kept, dlogits, grads):
    e, h, stats, u, s, d, _ = kept
    run.linear_grad_weight(TABLE, VOCAB, WIDTH, d, dlogits, ptr, grads)
    dd = run.linear_grad_input(TABLE, VOCAB, WIDTH, dlogits, ptr)
    run.linear_grad_weight(DOWN, WIDTH, HIDDEN, s, dd, ptr, grads)
    ds = run.linear_grad_input(DOWN, WIDTH, HIDDEN, dd, ptr)
    du = (2.0 * ds.float() * u.float()).to(u.dtype)
    run.linear_grad_weight(UP, HIDDEN, WIDTH, h, du, ptr, grads)
    dh = run.linear_grad_input(UP, HIDDEN, WIDTH, du, ptr)
    de = run.layer_norm_grad(GAIN, BIAS, WIDTH, e, ptr, stats, dh, grads)
    run.embedding_grad(TABLE, VOCAB, WIDTH, tokens, ptr, de, grads, scale=SCALE, accumulate=True)  # the tied table


def reference(params, tokens, targets):
    """Loss gradient of one worker's row in fp64 by autograd (on the CPU)."""
    import torch

    w = torch.tensor(params, dtype=torch.float64, requires_grad=True)
    table = w[TABLE:GAIN].view(VOCAB, WIDTH)
    e = SCALE * table[torch.as_tensor(tokens, dtype=torch.long)]
    c = e - e.mean(1, keepdim=True)
    h = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * w[GAIN:BIAS] + w[BIAS:BIAS + WIDTH]
    u = h @ w[UP:DOWN].view(HIDDEN, WIDTH).T
    d = (u * u) @ w[DOWN:DOWN + WIDTH * HIDDEN].view(WIDTH, HIDDEN).T
    logits = d @ table.T
    loss = torch.nn.functional.cross_entropy(logits, torch.as_tensor(targets, dtype=torch.long), reduction="sum")
    loss.backward()
    return w.grad.numpy()


def start_params(n, seed):
    import torch

    gen = torch.Generator()
    gen.manual_seed(seed)
    w = torch.empty(P).normal_(0.0, 0.3, generator=gen)
    w[GAIN:BIAS] = 1 + 0.1 * w[GAIN:BIAS]
    return w


def test_training_steps_between_rounds():
    """Gradients of whole steps against fp64 autograd, worker by worker, through local steps and fused rounds with
    other rows for every worker in every step.  fp32: an operator's sums are at most 89 terms long, off by at most
    2 (89 + 4) 2^-24 = 1.1e-5 of the sum of their magnitudes; a gradient passes seven operators, and magnitudes
    add up to at most eight times the largest value here: 6.3e-4 of the largest gradient."""
    import torch

    n = 3
    run = g.GASLoC(n, P, topology="ring", consensus_momentum=0.1)
    run.x.fill_(float("nan"))
    run.y.fill_(float("nan"))
    run.set_params(start_params(n, 1).cuda())
    grads = torch.empty((n, run.ld), device="cuda")
    rng = np.random.default_rng(5)
    step = 0
    for t in range(3):
        for h in range(3):
            rows = rng.integers(1, 40, n)
            if h == 1:
                rows[step % n] = 0
            ptr = np.concatenate([[0], np.cumsum(rows)])
            k = rng.integers(0, VOCAB, ptr[-1]).astype(np.int32)
            target = rng.integers(0, VOCAB, ptr[-1])
            _, stepped, _ = run.counters()
            torch.cuda.synchronize()
            live = np.stack([(run.y if stepped[i] else run.x)[i, :P].double().cpu().numpy() for i in range(n)])
            tokens = torch.as_tensor(k, device="cuda")
            kept = forward(run, tokens, ptr, "f32")
            dlogits = torch.softmax(kept[-1].double(), 1)
            dlogits[torch.arange(len(k), device="cuda"), torch.as_tensor(target, device="cuda")] -= 1
            grads.fill_(0.0)
            backward(run, tokens, ptr, kept, dlogits.float(), grads)
            torch.cuda.synchronize()
            got = grads[:, :P].double().cpu().numpy()
            for i in range(n):
                a, b = ptr[i], ptr[i + 1]
                want = reference(live[i], k[a:b], target[a:b]) if b > a else np.zeros(P)
                worst = np.abs(got[i] - want).max()
                say("round", t, "step", h, "worker", i, "rows", b - a, "worst", worst, "largest", np.abs(want).max())
                assert worst <= 6.3e-4 * np.abs(want).max()
            active = (rows > 0).astype(np.uint8)
            if h < 2:
                run.local_step(grads, 1e-3, active)
            else:
                run.local_step_gossip_round(grads, 1e-3, t, active)
            step += 1
    assert np.isfinite(run.consensus_error())


@pytest.mark.parametrize("params,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_recorded_steps_replay(params, act):
    """Forward and backward recorded once give, on every replay, what eager calls give for the inputs then in place,
    with eager work of the same context between the replays."""
    import torch

    say("graph", params, act)
    n = 4
    ptr = np.array([0, 33, 33, 200, 217])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        run = g.GASLoC(n, P, param_dtype=params, outer_momentum=0.0, consensus_momentum=0.0, stream=stream)
        run.set_params(start_params(n, 2).cuda())
        tokens = torch.zeros(int(ptr[-1]), dtype=torch.int32, device="cuda")
        dlogits = torch.zeros((int(ptr[-1]), VOCAB), dtype=torch.float32 if act == "f32" else torch.bfloat16,
                              device="cuda")
        grads = torch.zeros((n, run.ld), device="cuda")

        def step(into):
            kept = forward(run, tokens, ptr, act)
            backward(run, tokens, ptr, kept, dlogits, into)
            return kept

        step(grads)  # warm-up
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            recorded = step(grads)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(3)
        for replay in range(4):
            tokens.copy_(torch.randint(-1, VOCAB + 1, tokens.shape, device="cuda", generator=gen).int())
            dlogits.copy_(torch.empty(dlogits.shape, device="cuda").normal_(generator=gen))
            other = torch.full_like(grads, 3.0)
            eager = step(other)
            grads.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(recorded, eager):
                assert torch.equal(a.view(torch.int32 if a.dtype == torch.float32 else torch.int16),
                                   b.view(torch.int32 if b.dtype == torch.float32 else torch.int16)), replay
            assert torch.equal(grads, other), replay
        run.close()


def test_graph_recorded_on_another_stream():
    """A context with a stream of its own: calls recorded from another stream replay with the eager results."""
    import torch

    n, rows, width = 3, 300, 64
    ptr = np.array([0, 100, 100, rows])
    run = g.GASLoC(n, width * width, outer_momentum=0.0, consensus_momentum=0.0, stream=torch.cuda.Stream())
    run.set_params(torch.empty(width * width, device="cuda").normal_(0.0, 0.05))
    x = torch.empty((rows, width), device="cuda").normal_()
    grads = torch.zeros((n, run.ld), device="cuda")

    def step(into):
        out = run.linear(0, width, width, x, ptr)
        run.linear_grad_weight(0, width, width, x, out, ptr, into)
        return out

    step(grads)  # warm-up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step(grads)
    for replay in range(4):
        x.normal_()
        other = torch.full_like(grads, 3.0)
        eager = step(other)
        grads.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(recorded, eager) and torch.equal(grads, other), replay
    run.close()


def test_graph_refuses_the_default_stream():
    """A context on the default stream cannot take part in a graph: an error, and both go on."""
    import torch

    width, ptr = 64, np.array([0, 8, 16])
    run = g.GASLoC(2, width * width, outer_momentum=0.0, consensus_momentum=0.0)
    run.set_params(torch.empty(width * width, device="cuda").normal_(0.0, 0.05))
    x = torch.empty((16, width), device="cuda").normal_()
    out = torch.zeros_like(x)
    expect = run.linear(0, width, width, x, ptr)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="default stream"):
            run.linear(0, width, width, x, ptr, out=out)
        out.add_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, torch.ones_like(out))
    assert torch.equal(run.linear(0, width, width, x, ptr), expect)
    run.close()


def test_called_from_another_stream():
    """The context has a stream of its own; the program computes inputs and uses results on the current one, and
    frees them at once.  Nothing waits on the host."""
    import torch

    n, rows, width = 3, 3000, 512
    ptr = np.array([0, 1000, 1000, rows])
    side = torch.cuda.Stream()
    run = g.GASLoC(n, width * width + 2 * width, outer_momentum=0.0, consensus_momentum=0.0, stream=side)
    same = g.GASLoC(n, width * width + 2 * width, outer_momentum=0.0, consensus_momentum=0.0)
    w = torch.empty(width * width + 2 * width, device="cuda").normal_(0.0, 0.05)
    run.set_params(w)
    same.set_params(w)
    torch.cuda.synchronize()
    want, got = [], []
    for out, r in ((want, same), (got, run)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(7)
        for k in range(30):
            x = torch.empty((rows, width), device="cuda").normal_(generator=gen)
            h, stats = r.layer_norm(width * width, width * width + width, width, x, ptr)
            y = r.linear(0, width, width, h, ptr)
            del h
            grads = torch.zeros((n, r.ld), device="cuda")
            d = y * y
            dh = r.linear_grad_input(0, width, width, d, ptr)
            r.linear_grad_weight(0, width, width, x, d, ptr, grads)
            del d
            dx = r.layer_norm_grad(width * width, width * width + width, width, x, ptr, stats, dh, grads)
            del dh, x
            out.append((dx.double().sum() + grads.double().sum()).clone())
            del dx, grads
    torch.cuda.synchronize()
    assert [float(a) for a in want] == [float(a) for a in got]


def test_same_bits_twice():
    import torch

    say("same bits")
    n, rows = 5, 20_011
    ptr = np.array([0, 9000, 9001, 9001, 15_000, rows])
    run = g.GASLoC(n, 600 * 256, outer_momentum=0.0, consensus_momentum=0.0)
    run.set_params(torch.empty(600 * 256, device="cuda").normal_())
    x = torch.empty((rows, 256), device="cuda").normal_()
    d = torch.empty((rows, 600), device="cuda").normal_()
    tokens = (torch.rand(rows, device="cuda") ** 4 * 600).int()
    results = []
    for fill in (1.0, -2.0):
        grads = torch.full((n, run.ld), fill, device="cuda")
        ws = torch.full((1 << 28,), int(fill) % 200, dtype=torch.uint8, device="cuda")
        _, stats = run.layer_norm(0, 256, 256, x, ptr)
        dx = run.layer_norm_grad(0, 256, 256, x, ptr, stats, x, grads, workspace=ws)
        a = grads[:, :512].clone()
        run.embedding_grad(0, 600, 256, tokens, ptr, x, grads, workspace=ws)
        b = grads[:, :600 * 256].clone()
        run.linear_grad_weight(0, 600, 256, x, d, ptr, grads, workspace=ws)
        c = grads[:, :600 * 256].clone()
        out = run.linear(0, 600, 256, x[:300], np.array([0, 100, 100, 200, 300, 300]), workspace=ws)
        results.append((dx, a, b, c, out))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_columns_behind_32_bits():
    """Weights near the end of long rows: offsets of several 2^32 bytes."""
    import torch

    n, p, vocab, width = 3, 800_000_004, 50, 64
    begin = p - vocab * width - 3
    say("long rows, columns from", begin)
    run = g.GASLoC(n, p, outer_momentum=0.0, consensus_momentum=0.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randint(-3, 4, (n, vocab * width), device="cuda", generator=gen).float()
    run.x[:, begin:begin + vocab * width] = w
    grads = torch.full((n, run.ld), 9.0, device="cuda")
    ptr = np.array([0, 30, 60, 100])
    worker = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor([30, 30, 40], device="cuda"))
    tokens = torch.randint(0, vocab, (100,), device="cuda", generator=gen).int()
    x = torch.randint(-3, 4, (100, width), device="cuda", generator=gen).float()
    d = torch.randint(-3, 4, (100, vocab), device="cuda", generator=gen).float()
    table = w.view(n, vocab, width)
    assert torch.equal(run.embedding(begin, vocab, width, tokens, ptr), table[worker, tokens.long()])
    assert torch.equal(run.linear(begin, vocab, width, x, ptr), (table[worker] * x[:, None, :]).sum(2))
    assert torch.equal(run.linear_grad_input(begin, vocab, width, d, ptr), (table[worker] * d[:, :, None]).sum(1))
    run.linear_grad_weight(begin, vocab, width, x, d, ptr, grads)
    want = torch.stack([(d[a:b, :, None] * x[a:b, None, :]).sum(0) for a, b in ((0, 30), (30, 60), (60, 100))])
    assert torch.equal(grads[:, begin:begin + vocab * width].view(n, vocab, width), want)
    run.embedding_grad(begin, vocab, width, tokens, ptr, x, grads)
    want = torch.zeros_like(want)
    want.index_put_((worker, tokens.long()), x, accumulate=True)
    assert torch.equal(grads[:, begin:begin + vocab * width].view(n, vocab, width), want)
    out, stats = run.layer_norm(begin, begin + width, width, x, ptr)
    run.layer_norm_grad(begin, begin + width, width, x, ptr, stats, x, grads)
    assert torch.equal(grads[:, begin + width:begin + 2 * width],
                       torch.stack([x[a:b].sum(0) for a, b in ((0, 30), (30, 60), (60, 100))]))
    assert bool((grads[:, :begin] == 9.0).all()) and bool((grads[:, begin + vocab * width:] == 9.0).all())


def test_rows_behind_32_bits():
    """Activations whose last rows lie behind 2^32 bytes."""
    import torch

    n, rows, ld, width = 2, 60_000, 40_000, 64
    say("long activations", rows, ld)
    run = g.GASLoC(n, 96 * width, outer_momentum=0.0, consensus_momentum=0.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randint(-3, 4, (n, 96 * width), device="cuda", generator=gen).float()
    run.x[:, :96 * width] = w
    x = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")[:, :width]
    x.copy_(torch.randint(-3, 4, (rows, width), device="cuda", generator=gen))
    out = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")[:, :96]
    ptr = np.array([0, 59_000, rows])
    run.linear(0, 96, width, x, ptr, out=out)
    table = w.view(n, 96, width)
    for i, (a, b) in enumerate(((0, 59_000), (59_000, rows))):
        want = (x[a:b].float().contiguous() @ table[i].t().contiguous()).bfloat16()
        assert torch.equal(out[a:b], want)
    grads = torch.empty((n, run.ld), device="cuda")
    run.linear_grad_weight(0, 96, width, x, out, ptr, grads)
    last = out[59_000:].double().t().contiguous() @ x[59_000:].double().contiguous()
    assert torch.equal(grads[1, :96 * width].view(96, width).double(), last)
    tokens = torch.randint(0, 96, (rows,), device="cuda", generator=gen).int()
    e = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")[:, :width]
    run.embedding(0, 96, width, tokens, ptr, out=e)
    assert torch.equal(e[59_000:].float(), table[1][tokens[59_000:].long()])
    run.embedding_grad(0, 96, width, tokens, ptr, x, grads)
    want = torch.zeros((96, width), device="cuda").index_add_(0, tokens[59_000:].long(), x[59_000:].float())
    assert torch.equal(grads[1, :96 * width].view(96, width), want)
    h, stats = run.layer_norm(0, None, width, x, ptr, out=e)
    assert bool((stats[:, 0] - x.float().mean(1)).abs().max() < 1e-5)
