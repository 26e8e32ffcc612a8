"""The binding of the layer calls (no GPU): arguments that must not reach the library."""
import pytest

import paper_2606_11081_amd as g

CTX = 0x1000  # no context: nothing may be called with it


def functions(row_ptr, **changes):
    """The module functions by name, with good arguments for a context of three workers but for the changes."""
    a = dict(vocab=8, width=4, out=4, inp=4)
    a.update(changes)
    v, w, m, k, p = a["vocab"], a["width"], a["out"], a["inp"], 0x30000000
    f = g.gasloc
    return {
        "embedding": lambda: f.gasloc_embedding(CTX, 0, v, w, 1.0, row_ptr, p, "f32", p, 4),
        "embedding_grad": lambda: f.gasloc_embedding_grad(CTX, 0, v, w, 1.0, row_ptr, p, "f32", p, 4, p, 64, 0, p,
                                                          1 << 20),
        "embedding_grad_workspace": lambda: f.gasloc_embedding_grad_workspace(CTX, w, row_ptr),
        "layer_norm": lambda: f.gasloc_layer_norm(CTX, 0, 4, w, 1e-5, row_ptr, p, 4, "f32", p, 4),
        "layer_norm_grad": lambda: f.gasloc_layer_norm_grad(CTX, 0, 4, w, row_ptr, p, 4, p, p, 4, "f32", p, 4, p, 64, 0,
                                                            p, 1 << 20),
        "layer_norm_grad_workspace": lambda: f.gasloc_layer_norm_grad_workspace(CTX, w, row_ptr),
        "linear": lambda: f.gasloc_linear(CTX, 0, m, k, row_ptr, p, 4, "f32", p, 4),
        "linear_grad_input": lambda: f.gasloc_linear_grad_input(CTX, 0, m, k, row_ptr, p, 4, "f32", p, 4),
        "linear_grad_weight": lambda: f.gasloc_linear_grad_weight(CTX, 0, m, k, row_ptr, p, 4, p, 4, "f32", p, 64, 0,
                                                                  None, 0),
        "linear_workspace": lambda: f.gasloc_linear_workspace(CTX, m, k, row_ptr, "f32"),
    }


NAMES = sorted(functions(None))


@pytest.mark.parametrize("row_ptr", [[0, 1, 2], [0, 1, 2, 3, 4], [], [[0, 1, 2, 3]], 0])
@pytest.mark.parametrize("name", NAMES)
def test_row_ptr_of_another_length(monkeypatch, name, row_ptr):
    """The library would read behind the end of a shorter one."""
    monkeypatch.setitem(g.gasloc._workers, CTX, 3)
    with pytest.raises(ValueError, match="row_ptr needs 4 numbers"):
        functions(row_ptr)[name]()


def test_contexts_are_forgotten(monkeypatch):
    class Library:
        gasloc_destroy = staticmethod(lambda ctx: None)

    monkeypatch.setattr(g.gasloc, "library", lambda: Library)
    monkeypatch.setitem(g.gasloc._workers, CTX, 3)
    g.gasloc_destroy(CTX)
    assert CTX not in g.gasloc._workers
    g.gasloc_destroy(CTX)
    g.gasloc_destroy(None)


@pytest.mark.parametrize("value", [(1 << 32) + 4, 1 << 31, -(1 << 31) - 1, -(1 << 32) + 4])
@pytest.mark.parametrize("key", ["vocab", "width", "out", "inp"])
def test_sizes_beyond_32_bits(monkeypatch, key, value):
    """Their low 32 bits may be a size that the library takes."""
    monkeypatch.setitem(g.gasloc._workers, CTX, 3)
    uses = {"vocab": ("embedding", "embedding_grad"), "out": ("linear",), "inp": ("linear",),
            "width": ("embedding", "layer_norm")}[key]
    hit = [n for n in NAMES if n.startswith(uses) and (key != "vocab" or "workspace" not in n)]
    assert hit
    for name in hit:
        with pytest.raises(ValueError, match="does not fit in 32 bits"):
            functions([0, 1, 2, 3], **{key: value})[name]()


@pytest.mark.parametrize("vocab", [(1 << 32) + 8, -(1 << 32) + 8])
def test_methods_with_a_vocabulary_beyond_32_bits(monkeypatch, vocab):
    import torch

    run = g.GASLoC.__new__(g.GASLoC)
    run.n, run.P, run.bufs = 3, 64, dict(x=torch.zeros(3, 64))
    called = []
    monkeypatch.setattr(run, "_run", lambda *a: called.append(a), raising=False)
    monkeypatch.setattr(run, "_workspace", lambda *a: ((), None, 0), raising=False)
    tokens, rows, grads = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 4), torch.zeros(3, 64)
    run.embedding(0, 8, 4, tokens, [0, 1, 2, 3])
    run.embedding_grad(0, 8, 4, tokens, [0, 1, 2, 3], rows, grads)
    assert [a[0] for a in called] == ["gasloc_embedding", "gasloc_embedding_grad"]
    with pytest.raises(ValueError, match="does not fit in 32 bits"):
        run.embedding(0, vocab, 4, tokens, [0, 1, 2, 3])
    with pytest.raises(ValueError, match="does not fit in 32 bits"):
        run.embedding_grad(0, vocab, 4, tokens, [0, 1, 2, 3], rows, grads)
    assert len(called) == 2


def test_local_steps_take_the_rows_of_a_view(monkeypatch):
    """Gradients in some columns of a larger tensor, as the layer calls take them, lie that tensor's rows apart."""
    import torch

    run = g.GASLoC.__new__(g.GASLoC)
    run.ctx, run.n, run.P, run.bufs = None, 3, 8, dict(x=torch.zeros(3, 8))
    got = []
    monkeypatch.setattr(g.gasloc, "gasloc_local_step", lambda ctx, grads, ld, active, lr: got.append(ld))
    monkeypatch.setattr(g.gasloc, "gasloc_local_step_gossip_round",
                        lambda ctx, grads, ld, active, lr, W, t: got.append(ld))
    whole = torch.zeros(3, 20)
    for grads, ld in ((whole, 20), (whole[:, :8], 20), (whole[:, 4:12], 20), (torch.zeros(6, 8)[::2], 16),
                      (torch.zeros(1, 8).expand(3, 8), 0), (torch.zeros(1, 8), 8)):
        run.local_step(grads, 1e-3)
        run.local_step_gossip_round(grads, 1e-3, 0)
        assert got == [ld, ld]  # the library refuses rows of 0
        del got[:]
    with pytest.raises(ValueError, match="contiguous"):
        run.local_step(torch.zeros(8, 3).t(), 1e-3)
    assert not got
