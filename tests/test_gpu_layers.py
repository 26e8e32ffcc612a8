"""The layer operators on the GPU against fp64: sizes and layouts where they
can go wrong (one row, workers without rows, odd and ragged sizes, weights at
odd columns, strided rows, rows and columns that belong to others)."""
import numpy as np
import pytest

import paper_2606_11081_amd as g
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")]  # (parameters, activations)
NAN = float("nan")


def _torch(dtype):
    import torch

    return torch.float32 if dtype == "f32" else torch.bfloat16


def say(*a):
    print(*a, flush=True)


class Rows:
    """A context whose workers' rows hold NaN except the weights put into them; gradients likewise."""

    def __init__(self, n, size, begin, params, tail=3, stepped=None):
        import torch

        self.n, self.begin, self.size = n, begin, size
        self.run = g.GASLoC(n, begin + size + tail, param_dtype=params, outer_momentum=0.0, consensus_momentum=0.0)
        self.run.x.fill_(NAN)
        self.run.y.fill_(NAN)
        self.stepped = np.zeros(n, np.uint8) if stepped is None else np.asarray(stepped, np.uint8)
        self.run.set_counters(self.stepped.astype(np.int64), self.stepped, 0)
        self.grads = torch.full((n, self.run.ld), 7.0, dtype=torch.float32, device="cuda")

    def put(self, values, at=0):
        """values: torch [n, size] into the live iterate of every worker; returns what is stored, as fp64."""
        import torch

        values = values.reshape(self.n, -1).to(_torch(self.run.param_dtype))
        a = self.begin + at
        for i in range(self.n):
            (self.run.y if self.stepped[i] else self.run.x)[i, a:a + values.shape[1]] = values[i]
        torch.cuda.synchronize()
        return values.double().cpu().numpy()

    def gradient(self, size=None, at=0):
        """The gradient's columns as fp64; everything else must have been left alone."""
        import torch

        size = self.size if size is None else size
        torch.cuda.synchronize()
        a = self.begin + at
        got = self.grads[:, a:a + size].double().cpu().numpy()
        rest = self.grads.clone()
        rest[:, a:a + size] = 7.0
        assert bool((rest == 7.0).all()), "columns of other parameters were written"
        return got


def rows_of(values, act, extra=0, behind=2, offset=0):
    """[T, W] values as a strided activation with NaN in `extra` columns, in `behind` rows after the last and
    in `offset` elements before the first: (view, what it holds as fp64, the whole buffer)."""
    import torch

    t, w = values.shape
    buf = torch.full(((t + behind) * (w + extra) + offset,), NAN, dtype=_torch(act), device="cuda")
    view = buf[offset:].view(t + behind, w + extra)[:, :w]
    view[:t] = values.to(_torch(act))
    return view, view[:t].double().cpu().numpy(), buf


def out_buffer(t, w, act, extra=0, behind=2, offset=0):
    import torch

    buf = torch.full(((t + behind) * (w + extra) + offset,), 5.0, dtype=_torch(act), device="cuda")
    return buf[offset:].view(t + behind, w + extra)[:, :w], buf


def read_rows(view, buf, t):
    """The first t rows as fp64; the rest of the buffer must still hold 5."""
    import torch

    torch.cuda.synchronize()
    got = view[:t].double().cpu().numpy()
    left = buf.clone()
    left[buf.numel() - view.shape[0] * view.stride(0):].view(view.shape[0], view.stride(0))[:t, :view.shape[1]] = 5.0
    assert bool((left == 5.0).all()), "something behind the rows was written"
    return got


def close(got, want, bound, what):
    assert np.isfinite(got).all(), "%s: not finite" % what
    over = np.abs(got - want) - bound
    if over.size and over.max() > 0:
        at = np.unravel_index(np.argmax(over), over.shape)
        raise AssertionError("%s: %d of %d outside the bound; at %s %r for %r (bound %.3g)"
                             % (what, int((over > 0).sum()), over.size, at, got[at], want[at], bound[at]))


def normal(seed, *shape):
    import torch

    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(generator=gen)


def integers(seed, low, high, *shape):
    import torch

    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randint(low, high + 1, shape, device="cuda", generator=gen).float()


SPLITS = {
    "one": [0, 1],
    "each1": [0, 1, 2, 3],
    "empty": [0, 0, 5, 5],
    "none": [0, 0, 0],
    "ragged": [0, 130, 131, 131, 400],
    "edges": [0, 64, 128, 256, 512, 513],
}

# --------------------------------------------------------------------------
# embedding
# --------------------------------------------------------------------------

TABLES = [("one", 1, 1, 0, 0, 0), ("each1", 7, 64, 0, 0, 0), ("empty", 300, 8, 8, 0, 0), ("none", 5, 16, 0, 0, 0),
          ("ragged", 1000, 320, 16, 8, 0), ("ragged", 37, 129, 3, 1, 1), ("edges", 65, 1024, 0, 0, 0),
          ("edges", 257, 24, 4, 0, 3), ("ragged", 64, 2056, 0, 0, 0)]


def tokens_for(seed, rows, vocab, skew):
    """int32 tokens, some of them padding on either side of the table; skew: one token makes up half of them."""
    rng = np.random.default_rng(seed)
    k = rng.integers(0, vocab, rows)
    if skew:
        k = np.where(rng.random(rows) < 0.5, vocab // 2, k)
    pad = rng.random(rows)
    k = np.where(pad < 0.05, -1, np.where(pad > 0.95, vocab, k))
    return k.astype(np.int32)


@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("split,vocab,width,begin,extra,offset", TABLES)
def test_embedding(split, vocab, width, begin, extra, offset, params, act):
    import torch

    say("embedding", split, vocab, width, begin, extra, offset, params, act)
    ptr = SPLITS[split]
    n, rows = len(ptr) - 1, ptr[-1]
    r = Rows(n, vocab * width, begin, params, stepped=np.arange(n) % 2)
    table = r.put(normal(1, n, vocab * width)).reshape(n, vocab, width)
    k = tokens_for(2, rows, vocab, False)
    tokens = torch.as_tensor(np.concatenate([k, np.zeros(3, np.int32)]), device="cuda")
    out, buf = out_buffer(rows, width, act, extra, offset=offset)
    got_view = r.run.embedding(begin, vocab, width, tokens, ptr, scale=0.3, out=out)
    assert got_view is out
    want = ref.embedding(table, k, ptr, np.float64(np.float32(0.3)))
    bound = (ref.HALF_STEP[act] + ref.U) * np.abs(want) * 1.01
    close(read_rows(out, buf, rows), want, bound, "embedding")


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("skew", [False, True])
@pytest.mark.parametrize("split,vocab,width,begin,extra,offset", TABLES)
def test_embedding_grad(split, vocab, width, begin, extra, offset, skew, act, accumulate):
    import torch

    say("embedding_grad", split, vocab, width, begin, extra, offset, skew, act, accumulate)
    ptr = SPLITS[split]
    n, rows = len(ptr) - 1, ptr[-1]
    r = Rows(n, vocab * width, begin, "f32")
    k = tokens_for(3, rows, vocab, skew)
    tokens = torch.as_tensor(np.concatenate([k, np.zeros(3, np.int32)]), device="cuda")
    dout, d, _ = rows_of(normal(4, rows, width), act, extra, offset=offset)
    r.run.embedding_grad(begin, vocab, width, tokens, ptr, dout, r.grads, scale=0.3, accumulate=accumulate)
    want, bound = ref.embedding_grad(n, vocab, k, ptr, d, np.float64(np.float32(0.3)))
    want, bound = want.reshape(n, -1), bound.reshape(n, -1)
    if accumulate:
        want = want + 7.0
        bound = bound + ref.U * np.abs(want) * 1.01
    close(r.gradient(), want, bound, "embedding_grad")


@pytest.mark.parametrize("rows", [[31, 32, 33], [1024, 1025, 64], [8191, 8192, 8193], [70_001, 0, 9000],
                                  [3, 530_000, 5]])
@pytest.mark.parametrize("vocab", [1, 3, 255, 256, 70_000])
def test_embedding_grad_sums_every_token_once(rows, vocab):
    """Whole numbers add up exactly in fp32, whatever the lengths the sort has to merge."""
    import torch

    say("embedding_grad rows", rows, "vocab", vocab)
    width = 4
    ptr = np.concatenate([[0], np.cumsum(rows)])
    r = Rows(3, vocab * width, 0, "f32")
    k = tokens_for(5, ptr[-1], vocab, vocab > 3)
    d = integers(6, -3, 3, int(ptr[-1]), width)
    r.run.embedding_grad(0, vocab, width, torch.as_tensor(k, device="cuda"), ptr, d, r.grads)
    want, _ = ref.embedding_grad(3, vocab, k, ptr, d.double().cpu().numpy(), 1.0)
    assert np.array_equal(r.gradient(), want.reshape(3, -1))


# --------------------------------------------------------------------------
# layer norm
# --------------------------------------------------------------------------

NORMS = [("one", 1, 0, 0, 0), ("each1", 64, 0, 0, 0), ("empty", 8, 8, 0, 0), ("none", 16, 0, 0, 0),
         ("ragged", 320, 16, 8, 0), ("ragged", 129, 3, 1, 1), ("edges", 1024, 0, 0, 0), ("ragged", 511, 5, 0, 1),
         ("edges", 2048, 0, 0, 0), ("ragged", 2049, 1, 0, 0), ("ragged", 8192, 0, 0, 0), ("empty", 8200, 0, 8, 0),
         ("empty", 16_384, 0, 0, 0), ("each1", 16_383, 0, 0, 0)]


def norm_inputs(ptr, width, seed):
    """Rows off centre and of different size, one of them constant, one tiny."""
    import torch

    rows = ptr[-1]
    x = normal(seed, rows, width) * torch.linspace(0.25, 4.0, max(rows, 1), device="cuda")[:rows, None]
    x += normal(seed + 1, rows, 1)
    if rows > 2:
        x[1] = 1.5
        x[2] *= 1e-3
    return x


@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("split,width,begin,extra,offset", NORMS)
def test_layer_norm(split, width, begin, extra, offset, with_bias, params, act):
    say("layer_norm", split, width, begin, extra, offset, with_bias, params, act)
    ptr = SPLITS[split]
    n, rows = len(ptr) - 1, ptr[-1]
    r = Rows(n, 2 * width, begin, params, stepped=np.arange(n) % 2)
    gain = r.put(1 + 0.1 * normal(1, n, width))
    bias = r.put(0.1 * normal(2, n, width), at=width) if with_bias else np.zeros((n, width))
    x, xs, _ = rows_of(norm_inputs(ptr, width, 3), act, extra, offset=offset)
    out, buf = out_buffer(rows, width, act, extra, offset=offset)
    _, stats = r.run.layer_norm(begin, begin + width if with_bias else None, width, x, ptr, eps=1e-5, out=out)
    want, bound, want_stats, stats_bound = ref.layer_norm(xs, gain, bias, np.asarray(ptr), np.float64(np.float32(1e-5)),
                                                          act)
    close(read_rows(out, buf, rows), want, bound, "out")
    close(stats.double().cpu().numpy(), want_stats, stats_bound, "stats")


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("split,width,begin,extra,offset", NORMS)
def test_layer_norm_grad(split, width, begin, extra, offset, params, act, accumulate):
    import torch

    say("layer_norm_grad", split, width, begin, extra, offset, params, act, accumulate)
    ptr = SPLITS[split]
    n, rows = len(ptr) - 1, ptr[-1]
    with_bias = split != "edges"
    r = Rows(n, 2 * width, begin, params, stepped=np.arange(n) % 2)
    gain = r.put(1 + 0.1 * normal(1, n, width))
    x, xs, _ = rows_of(norm_inputs(ptr, width, 3), act, extra, offset=offset)
    dout, d, _ = rows_of(normal(5, rows, width), act, extra, offset=offset)
    _, _, stats, _ = ref.layer_norm(xs, gain, gain, np.asarray(ptr), 1e-5, act)
    stats = torch.as_tensor(stats, dtype=torch.float32, device="cuda")
    dx, buf = out_buffer(rows, width, act, extra, offset=offset)
    r.run.layer_norm_grad(begin, begin + width if with_bias else None, width, x, ptr, stats, dout, r.grads, dx=dx,
                          accumulate=accumulate)
    want = ref.layer_norm_grad(xs, stats.double().cpu().numpy(), gain, d, np.asarray(ptr), act)
    close(read_rows(dx, buf, rows), want[0], want[1], "dx")
    got = r.gradient(2 * width if with_bias else width)
    for at, w, bound, what in ((0, want[2], want[3], "dgain"), (width, want[4], want[5], "dbias")):
        if at == 0 or with_bias:
            if accumulate:
                w = w + 7.0
                bound = bound + ref.U * np.abs(w) * 1.01
            close(got[:, at:at + width], w, bound, what)


def test_layer_norm_gradient_against_differences():
    """d sum(out * d) / d(x, gain, bias) by central differences of the formula in fp64."""
    import torch

    ptr = np.array([0, 3, 3, 8])
    n, width, rows = 3, 24, 8
    r = Rows(n, 2 * width, 0, "f32")
    gain = r.put(1 + 0.1 * normal(1, n, width))
    bias = r.put(0.1 * normal(2, n, width), at=width)
    x, xs, _ = rows_of(normal(3, rows, width), "f32")
    dout, d, _ = rows_of(normal(4, rows, width), "f32")
    out, stats = r.run.layer_norm(0, width, width, x, ptr)
    dx = r.run.layer_norm_grad(0, width, width, x, ptr, stats, dout, r.grads)
    got = r.gradient()

    def loss(xs, gain, bias):
        return float((ref.layer_norm(xs, gain, bias, ptr, 1e-5, "f32")[0] * d).sum())

    step = 2.0 ** -16
    rng = np.random.default_rng(0)
    for name, at, grad in (("x", 0, dx[:rows].double().cpu().numpy()), ("gain", 1, got[:, :width]),
                           ("bias", 2, got[:, width:])):
        for _ in range(12):
            args = [xs.copy(), gain.copy(), bias.copy()]
            where = tuple(rng.integers(0, s) for s in args[at].shape)
            args[at][where] += step
            up = loss(*args)
            args[at][where] -= 2 * step
            slope = (up - loss(*args)) / (2 * step)
            # third derivatives of order 10 times step^2, and fp64 rounding of the loss over the step
            assert abs(slope - grad[where]) < 2e-5 * (1 + abs(slope)), (name, where, slope, grad[where])


def test_layer_norm_in_place():
    import torch

    ptr = [0, 5, 17]
    r = Rows(2, 2 * 96, 0, "f32")
    r.put(1 + 0.1 * normal(1, 2, 96))
    r.put(0.1 * normal(2, 2, 96), at=96)
    x = normal(3, 17, 96)
    d = normal(4, 17, 96)
    out, stats = r.run.layer_norm(0, 96, 96, x, ptr)
    same = x.clone()
    r.run.layer_norm(0, 96, 96, same, ptr, out=same)
    assert torch.equal(out, same)
    dx = r.run.layer_norm_grad(0, 96, 96, x, ptr, stats, d, r.grads)
    for target in ("dout", "x"):
        x2, d2 = x.clone(), d.clone()
        got = r.run.layer_norm_grad(0, 96, 96, x2, ptr, stats, d2, r.grads, dx=d2 if target == "dout" else x2)
        assert torch.equal(got, dx), target


# --------------------------------------------------------------------------
# linear
# --------------------------------------------------------------------------

LINEARS = [("one", 1, 1, 0, 0, 0), ("each1", 64, 64, 0, 0, 0), ("empty", 8, 24, 8, 0, 0), ("none", 16, 16, 0, 0, 0),
           ("ragged", 320, 192, 16, 8, 0), ("ragged", 129, 65, 3, 1, 1), ("edges", 256, 512, 0, 0, 0),
           ("edges", 264, 72, 8, 0, 0), ("ragged", 33, 1000, 2, 0, 1), ("each1", 1000, 2056, 0, 0, 0),
           ("ragged", 1, 300, 0, 0, 0), ("ragged", 300, 1, 0, 0, 0), ("one", 4096, 72, 0, 8, 0),
           ("edges", 40, 4104, 0, 0, 0)]
# (split, out_features, in_features, begin, extra, offset)


def linear_case(split, m, k, begin, params, act, whole, stepped=True):
    ptr = SPLITS[split]
    n, rows = len(ptr) - 1, ptr[-1]
    r = Rows(n, m * k, begin, params, stepped=np.arange(n) % 2 if stepped else None)
    make = (lambda s, *shape: integers(s, -3, 3, *shape)) if whole else normal
    w = r.put(make(1, n, m * k)).reshape(n, m, k)
    if act == "bf16":
        w = ref.to_bf16(w)
    return np.asarray(ptr), rows, r, w, make


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("split,m,k,begin,extra,offset", LINEARS)
def test_linear(split, m, k, begin, extra, offset, params, act, whole):
    say("linear", split, m, k, begin, extra, offset, params, act, whole)
    ptr, rows, r, w, make = linear_case(split, m, k, begin, params, act, whole)
    x, xs, _ = rows_of(make(2, rows, k), act, extra, offset=offset)
    out, buf = out_buffer(rows, m, act, extra, offset=offset)
    r.run.linear(begin, m, k, x, ptr, out=out)
    want, bound = ref.linear(w, xs, ptr, act)
    got = read_rows(out, buf, rows)
    if whole:  # whole numbers: nothing is rounded before the store
        want, bound = (ref.to_bf16(want) if act == "bf16" else want), np.zeros_like(bound)
    close(got, want, bound, "linear")


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("split,m,k,begin,extra,offset", LINEARS)
def test_linear_grad_input(split, m, k, begin, extra, offset, params, act, whole):
    say("linear_grad_input", split, m, k, begin, extra, offset, params, act, whole)
    ptr, rows, r, w, make = linear_case(split, m, k, begin, params, act, whole)
    dout, d, _ = rows_of(make(2, rows, m), act, extra, offset=offset)
    dx, buf = out_buffer(rows, k, act, extra, offset=offset)
    r.run.linear_grad_input(begin, m, k, dout, ptr, dx=dx)
    want, bound = ref.linear_grad_input(w, d, ptr, act)
    got = read_rows(dx, buf, rows)
    if whole:
        want, bound = (ref.to_bf16(want) if act == "bf16" else want), np.zeros_like(bound)
    close(got, want, bound, "linear_grad_input")


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("params,act", TYPES)
@pytest.mark.parametrize("split,m,k,begin,extra,offset", LINEARS)
def test_linear_grad_weight(split, m, k, begin, extra, offset, params, act, whole):
    say("linear_grad_weight", split, m, k, begin, extra, offset, params, act, whole)
    ptr, rows, r, w, make = linear_case(split, m, k, begin, params, act, whole)
    x, xs, _ = rows_of(make(2, rows, k), act, extra, offset=offset)
    dout, d, _ = rows_of(make(3, rows, m), act, extra, offset=offset)
    r.run.linear_grad_weight(begin, m, k, x, dout, ptr, r.grads, accumulate=whole)
    want, bound = ref.linear_grad_weight(xs, d, ptr)
    want, bound = want.reshape(len(ptr) - 1, -1), bound.reshape(len(ptr) - 1, -1)
    if whole:
        want, bound = want + 7.0, np.zeros_like(bound)
    close(r.gradient(), want, bound, "linear_grad_weight")


@pytest.mark.parametrize("kind", ["linear", "linear_grad_input", "linear_grad_weight"])
@pytest.mark.parametrize("params,act", TYPES)
def test_linear_long_sums(kind, params, act):
    """The dimension that is summed over is long: thousands of features or of rows."""
    say("long", kind, params, act)
    m, k, rows = {"linear": (72, 12_296, 40), "linear_grad_input": (12_296, 72, 40),
                  "linear_grad_weight": (72, 40, 30_011)}[kind]
    ptr = np.array([0, rows - rows // 3, rows])
    r = Rows(2, m * k, 0, params)
    w = r.put(integers(1, -2, 2, 2, m * k)).reshape(2, m, k)
    x, xs, _ = rows_of(integers(2, -2, 2, rows, k), act)
    dout, d, _ = rows_of(integers(3, -2, 2, rows, m), act)
    if kind == "linear":
        got, want = r.run.linear(0, m, k, x, ptr)[:rows].double().cpu().numpy(), ref.linear(w, xs, ptr, act)[0]
    elif kind == "linear_grad_input":
        got = r.run.linear_grad_input(0, m, k, dout, ptr)[:rows].double().cpu().numpy()
        want = ref.linear_grad_input(w, d, ptr, act)[0]
    else:
        r.run.linear_grad_weight(0, m, k, x, dout, ptr, r.grads)
        got, want = r.gradient(), ref.linear_grad_weight(xs, d, ptr)[0].reshape(2, -1)
        assert np.array_equal(got, want)
        return
    assert np.array_equal(got, ref.to_bf16(want) if act == "bf16" else want)


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("kind,params,act,split", [(k, p, a, s) for k, a, s in ref.LARGE for p, b in TYPES if a == b])
def test_linear_large_tiles(kind, params, act, split, odd):
    """Tiles of 128 outputs, whole and in parts; odd: sizes and columns that no vector fits.  Whole numbers, whose
    sums (at most 4 * 80000) are exact."""
    say("large", kind, params, act, split, odd)
    ptr, m, k = ref.LARGE[kind, act, split]
    ptr, rows, m, k, begin = np.array(ptr), ptr[-1], m - odd, k - odd, int(odd)
    r = Rows(2, m * k, begin, params, stepped=[0, 1])
    w = r.put(integers(1, -2, 2, 2, m * k)).reshape(2, m, k)
    x, xs, _ = rows_of(integers(2, -2, 2, rows, k), act)
    dout, d, _ = rows_of(integers(3, -2, 2, rows, m), act)
    if kind == "linear":
        got, want = r.run.linear(begin, m, k, x, ptr)[:rows].double().cpu().numpy(), ref.linear(w, xs, ptr, act)[0]
    elif kind == "linear_grad_input":
        got = r.run.linear_grad_input(begin, m, k, dout, ptr)[:rows].double().cpu().numpy()
        want = ref.linear_grad_input(w, d, ptr, act)[0]
    else:
        r.run.linear_grad_weight(begin, m, k, x, dout, ptr, r.grads, accumulate=odd)
        got, want = r.gradient(), ref.linear_grad_weight(xs, d, ptr)[0].reshape(2, -1) + 7.0 * odd
        assert np.array_equal(got, want)
        return
    assert np.array_equal(got, ref.to_bf16(want) if act == "bf16" else want)


def test_linear_infinities_and_nan_stay_in_their_rows():
    """What is not finite in one worker's rows, or in the rows behind a ragged end, reaches no other worker."""
    import torch

    ptr = np.array([0, 37, 90, 90, 101])
    n, m, k = 4, 136, 72
    for params, act in TYPES:
        say("not finite", params, act)
        r = Rows(n, m * k, 0, params)
        w = r.put(integers(1, -3, 3, n, m * k)).reshape(n, m, k)
        values = integers(2, -3, 3, 101, k)
        grads = integers(3, -3, 3, 101, m)
        clean_x, clean_d = values.double().cpu().numpy(), grads.double().cpu().numpy()
        values[37:90] = NAN
        grads[37:90] = float("inf")
        x, _, _ = rows_of(values, act)
        dout, _, _ = rows_of(grads, act)
        out = r.run.linear(0, m, k, x, ptr).double().cpu().numpy()[:101]
        dx = r.run.linear_grad_input(0, m, k, dout, ptr).double().cpu().numpy()[:101]
        r.run.linear_grad_weight(0, m, k, x, dout, ptr, r.grads)
        gw = r.gradient().reshape(n, m, k)
        keep = np.r_[0:37, 90:101]
        q = ref.to_bf16 if act == "bf16" else (lambda a: a)
        assert np.array_equal(out[keep], q(ref.linear(w, clean_x, ptr, act)[0])[keep])
        assert np.array_equal(dx[keep], q(ref.linear_grad_input(w, clean_d, ptr, act)[0])[keep])
        assert np.isnan(out[37:90]).all() and np.isnan(gw[1]).all()
        want = ref.linear_grad_weight(clean_x, clean_d, ptr)[0]
        assert np.array_equal(gw[[0, 2, 3]], want[[0, 2, 3]]) and not gw[2].any()
