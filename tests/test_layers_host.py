"""The host side of the layer calls (no GPU): refusals of every entry point,
workspace sizes, and how calls are cut into workgroups.  A shim compiles
layers.cpp with a context made by hand and launchers that only record."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2606_11081_amd as g
from tests import layers_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
BAD, OK, STATE = g.gasloc.GASLOC_EINVAL, g.gasloc.GASLOC_OK, g.gasloc.GASLOC_ESTATE
P0 = 0x30000000  # an aligned address that nothing reads
F32, BF16 = 0, 1
CUS = 256


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no g++")
    so = str(tmp_path_factory.mktemp("shim") / "layers_shim.so")
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-shared", "-fPIC", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-include", "cstdarg", "-include", "cstdlib",
                    "-I" + os.path.join(ROCM, "include"), "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2606_11081_amd", "csrc"),
                    os.path.join(ROOT, "tests", "layers_shim.cpp"), "-L" + os.path.join(ROCM, "lib"), "-lamdhip64",
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", so], check=True, capture_output=True)
    lib = ctypes.CDLL(so)
    for name, (res, args) in g.gasloc._SIGNATURES.items():
        if re.match(r"gasloc_(embedding|layer_norm|linear)", name):
            getattr(lib, name).restype, getattr(lib, name).argtypes = res, args
    lib.shim_context.restype = ctypes.c_void_p
    lib.shim_context.argtypes = [ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    for name in ("shim_fail", "shim_free"):
        getattr(lib, name).argtypes = [ctypes.c_void_p]
    lib.shim_step.argtypes = [ctypes.c_void_p, ctypes.c_int]
    lib.shim_error.restype = ctypes.c_char_p
    lib.shim_linear_stepped.restype = ctypes.c_uint64
    return lib


class Context:
    def __init__(self, shim, n=4, P=100_000, dtype=F32):
        self.shim, self.n = shim, n
        self.c = shim.shim_context(n, P, dtype, CUS)

    def __del__(self):
        self.shim.shim_free(self.c)


def rp(*rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)


# every call with good arguments, as (name, argument list); {k: v} replaces argument k
def calls(ptr, act=F32):
    p = ptr.ctypes.data
    big = 1 << 40
    return {
        "gasloc_embedding": dict(begin=0, vocab=100, width=64, scale=1.0, row_ptr=p, tokens=P0, dtype=act, out=P0,
                                 out_ld=64),
        "gasloc_embedding_grad": dict(begin=0, vocab=100, width=64, scale=1.0, row_ptr=p, tokens=P0, dtype=act,
                                      dout=P0, dout_ld=64, grads=P0, grad_ld=100_000, accumulate=0, workspace=P0,
                                      workspace_bytes=big),
        "gasloc_layer_norm": dict(gain=0, bias=64, width=64, eps=1e-5, row_ptr=p, x=P0, x_ld=64, dtype=act, out=P0,
                                  out_ld=64, stats=P0),
        "gasloc_layer_norm_grad": dict(gain=0, bias=64, width=64, row_ptr=p, x=P0, x_ld=64, stats=P0, dout=P0,
                                       dout_ld=64, dtype=act, dx=P0, dx_ld=64, grads=P0, grad_ld=100_000,
                                       accumulate=0, workspace=P0, workspace_bytes=big),
        "gasloc_linear": dict(weight=0, out_features=64, in_features=32, row_ptr=p, x=P0, x_ld=32, dtype=act, out=P0,
                              out_ld=64, workspace=P0, workspace_bytes=big),
        "gasloc_linear_grad_input": dict(weight=0, out_features=64, in_features=32, row_ptr=p, dout=P0, dout_ld=64,
                                         dtype=act, dx=P0, dx_ld=32, workspace=P0, workspace_bytes=big),
        "gasloc_linear_grad_weight": dict(weight=0, out_features=64, in_features=32, row_ptr=p, x=P0, x_ld=32,
                                          dout=P0, dout_ld=64, dtype=act, grads=P0, grad_ld=100_000, accumulate=0,
                                          workspace=P0, workspace_bytes=big),
    }


NAMES = sorted(calls(rp(1, 1, 1, 1)))


def call(ctx, name, **changes):
    args = calls(changes.pop("ptr", rp(3, 0, 2, 1)), changes.pop("act", F32))[name]
    assert set(changes) <= set(args), (name, changes)
    args.update(changes)
    return getattr(ctx.shim, name)(ctx.c, *args.values())


@pytest.mark.parametrize("name", NAMES)
def test_good_calls_launch(shim, name):
    for dtype, act in ((F32, F32), (F32, BF16), (BF16, BF16)):
        ctx = Context(shim, dtype=dtype)
        shim.shim_launches()
        assert call(ctx, name, act=act) == OK, shim.shim_error()
        assert shim.shim_launches() >= 1


@pytest.mark.parametrize("name", NAMES)
def test_no_rows(shim, name):
    """Nothing to compute: no activation is needed, and gradients that are not added to become zero."""
    ctx = Context(shim)
    empty = {k: None for k in ("tokens", "out", "dout", "x", "dx", "stats") if k in calls(rp(1, 1, 1, 1))[name]}
    shim.shim_launches()
    assert call(ctx, name, ptr=rp(0, 0, 0, 0), **empty) == OK, shim.shim_error()
    writes = name.endswith(("embedding_grad", "norm_grad", "grad_weight"))
    assert (shim.shim_launches() > 0) == writes
    if writes:
        assert call(ctx, name, ptr=rp(0, 0, 0, 0), accumulate=1, **empty) == OK
        assert shim.shim_launches() == 0


REFUSALS = [
    ("gasloc_*", dict(row_ptr=None), "row_ptr must not be NULL"),
    ("gasloc_*", dict(ptr=np.array([1, 2, 3, 4, 5], np.int64)), "start at 0"),
    ("gasloc_*", dict(ptr=np.array([0, 4, 3, 4, 5], np.int64)), "decreases at worker 1"),
    ("gasloc_*", dict(ptr=rp(1 << 27, 0, 1, 0)), "more than 2^27 rows"),
    ("gasloc_*", dict(dtype=2), "dtype must be"),
    ("gasloc_*", dict(dtype=-1), "dtype must be"),
    ("gasloc_embedding*", dict(begin=-1), "table: columns"),
    ("gasloc_embedding*", dict(begin=100_000 - 6399), "table: columns"),
    ("gasloc_embedding*", dict(vocab=0), "vocab must be"),
    ("gasloc_embedding*", dict(vocab=(1 << 24) + 1), "vocab must be"),
    ("gasloc_embedding*", dict(width=0), "width must be"),
    ("gasloc_embedding*", dict(width=(1 << 31) - 1), "table: columns"),
    ("gasloc_embedding*", dict(scale=float("nan")), "scale must be finite"),
    ("gasloc_embedding*", dict(scale=float("inf")), "scale must be finite"),
    ("gasloc_embedding*", dict(tokens=None), "tokens must be"),
    ("gasloc_embedding*", dict(tokens=P0 + 2), "tokens must be"),
    ("gasloc_layer_norm*", dict(width=0), "width must be"),
    ("gasloc_layer_norm*", dict(width=16385), "width must be"),
    ("gasloc_layer_norm*", dict(gain=-1), "gain: columns"),
    ("gasloc_layer_norm*", dict(gain=100_000 - 63), "gain: columns"),
    ("gasloc_layer_norm*", dict(bias=100_000 - 63), "bias: columns"),
    ("gasloc_layer_norm*", dict(bias=63), "overlap"),
    ("gasloc_layer_norm", dict(eps=0.0), "eps must be"),
    ("gasloc_layer_norm", dict(eps=-1.0), "eps must be"),
    ("gasloc_layer_norm", dict(eps=float("nan")), "eps must be"),
    ("gasloc_layer_norm*", dict(stats=P0 + 4), "stats must be"),
    ("gasloc_layer_norm_grad", dict(stats=None), "stats must be"),
    ("gasloc_layer_norm", dict(out_ld=72), "rows of another length"),
    ("gasloc_layer_norm_grad", dict(dx_ld=72, dout=P0 + 0x1000), "rows of another length"),
    ("gasloc_layer_norm_grad", dict(dx_ld=72, x=P0 + 0x1000), "rows of another length"),
    ("gasloc_linear*", dict(weight=-1), "weight: columns"),
    ("gasloc_linear*", dict(weight=100_000 - 2047), "weight: columns"),
    ("gasloc_linear*", dict(out_features=0), "features must be"),
    ("gasloc_linear*", dict(in_features=(1 << 20) + 1), "features must be"),
    ("gasloc_*grad", dict(accumulate=2), "accumulate must be"),
    ("gasloc_*grad*", dict(grads=None), "grads must be"),
    ("gasloc_*grad*", dict(grads=P0 + 8), "grads must be"),
    ("gasloc_*grad*", dict(grad_ld=99_996), "grad_ld must be"),
    ("gasloc_*grad*", dict(grad_ld=100_002), "grad_ld must be"),
    ("gasloc_*grad", dict(workspace=None), "workspace must be"),
    ("gasloc_*grad", dict(workspace=P0 + 128), "workspace must be"),
    ("gasloc_*grad", dict(workspace_bytes=100), "needed"),
]
for _k in ("x", "dout", "dx", "out"):
    REFUSALS += [
        ("gasloc_*", {_k: None}, _k + " must not be NULL"),
        ("gasloc_*", {_k: P0 + 2}, _k + " is not aligned"),
        ("gasloc_*", {_k + "_ld": 31}, _k + ": row length"),
        ("gasloc_*", {_k + "_ld": 1 << 21}, _k + ": row length"),
        ("gasloc_*", {_k + "_ld": -64}, _k + ": row length"),
    ]


@pytest.mark.parametrize("pattern,changes,message", REFUSALS)
def test_refusals(shim, pattern, changes, message):
    ctx = Context(shim)
    hit = 0
    for name in NAMES:
        if not re.fullmatch(pattern.replace("*", ".*"), name):
            continue
        if not set(changes) - {"ptr"} <= set(calls(rp(1, 1, 1, 1))[name]):
            continue
        hit += 1
        shim.shim_launches()
        assert call(ctx, name, **changes) == BAD, (name, changes)
        assert message in shim.shim_error().decode(), (name, shim.shim_error())
        assert shim.shim_launches() == 0
    assert hit


@pytest.mark.parametrize("name", NAMES)
def test_types_that_do_not_go_together(shim, name):
    ctx = Context(shim, dtype=BF16)
    assert call(ctx, name, act=F32) == BAD
    assert b"F32 activations need F32 parameters" in shim.shim_error()


@pytest.mark.parametrize("name", NAMES)
def test_context_unusable_after_a_device_error(shim, name):
    ctx = Context(shim)
    shim.shim_fail(ctx.c)
    assert call(ctx, name) == STATE


@pytest.mark.parametrize("name", NAMES)
def test_null_context(shim, name):
    for lib in (shim, g.library()):
        fn = getattr(lib, name)
        assert fn(None, *calls(rp(1, 1, 1, 1))[name].values()) == BAD


def test_workspace_refusals(shim):
    size = ctypes.c_size_t()
    ctx = Context(shim)
    ptr = rp(1, 2, 3, 4)
    for args in ((None, 8, ptr.ctypes.data, ctypes.byref(size)), (ctx.c, 0, ptr.ctypes.data, ctypes.byref(size)),
                 (ctx.c, 8, None, ctypes.byref(size)), (ctx.c, 8, ptr.ctypes.data, None)):
        assert shim.gasloc_embedding_grad_workspace(*args) == BAD
        assert shim.gasloc_layer_norm_grad_workspace(*args) == BAD
    at, out = ptr.ctypes.data, ctypes.byref(size)
    for args in ((None, 8, 8, at, 0, out), (ctx.c, 0, 8, at, 0, out), (ctx.c, 8, 1 << 21, at, 0, out),
                 (ctx.c, 8, 8, None, 0, out), (ctx.c, 8, 8, at, 5, out), (ctx.c, 8, 8, at, 0, None)):
        assert shim.gasloc_linear_workspace(*args) == BAD


def test_the_live_iterate_is_chosen_per_worker(shim):
    ctx = Context(shim)
    shim.shim_step(ctx.c, 2)
    assert call(ctx, "gasloc_linear") == OK
    assert shim.shim_linear_stepped() == 1 << 2


@pytest.mark.parametrize("longest,merges", [(8192, 0), (8193, 1), (65_536, 1), (65_537, 2), (530_000, 3)])
def test_sorted_runs_are_merged_by_eights(shim, longest, merges):
    ctx = Context(shim)
    shim.shim_merges()
    assert call(ctx, "gasloc_embedding_grad", ptr=rp(5, longest, 0, 9)) == OK
    assert shim.shim_merges() == merges


def random_rows(rng, n):
    kind = rng.integers(4)
    rows = [rng.integers(0, 5, n), rng.integers(0, 300, n), rng.integers(0, 20_000, n), np.zeros(n, int)][kind]
    rows[rng.integers(n)] += rng.integers(1, 50)
    return rp(*rows)


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("kind,act,split", ref.LARGE)
def test_large_products_take_large_tiles(shim, kind, act, split, odd):
    """The cases that the GPU tests mean for tiles of 128 are such, in parts or not."""
    ptr, m, k = ref.LARGE[kind, act, split]
    m, k, ptr, act = m - odd, k - odd, np.array(ptr, np.int64), F32 if act == "f32" else BF16
    ctx = Context(shim, n=2, P=m * k + 8, dtype=F32)
    size = ctypes.c_size_t()
    assert shim.gasloc_linear_workspace(ctx.c, m, k, ptr.ctypes.data, act, ctypes.byref(size)) == OK
    changes = dict(weight=0, out_features=m, in_features=k, workspace_bytes=size.value)
    for key in calls(ptr)["gasloc_" + kind]:
        changes.update({"x_ld": dict(x_ld=k), "dx_ld": dict(dx_ld=k), "out_ld": dict(out_ld=m),
                        "dout_ld": dict(dout_ld=m), "grad_ld": dict(grad_ld=(m * k + 11) // 4 * 4)}.get(key, {}))
    assert call(ctx, "gasloc_" + kind, ptr=ptr, act=act, **changes) == OK, shim.shim_error()
    plan = np.zeros(3 + 3 * 2 + 2, np.int64)
    shim.shim_linear_plan(2, plan.ctypes.data_as(ctypes.c_void_p))
    assert plan[0] == 128 and bool(plan[1]) == (not odd) and (plan[2] > 0) == split


@pytest.mark.parametrize("seed", range(60))
def test_linear_plans_cover_every_product_once(shim, seed):
    """Tiles of each worker times its parts, the parts long enough for the sums, and the workspace that the size
    call gave is enough for what each of the three passes uses."""
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 9))
    m, k = (int(np.exp(rng.uniform(0, np.log(5000)))) for _ in range(2))
    act = int(rng.integers(2))
    ctx = Context(shim, n=n, P=m * k + 8, dtype=F32)
    ptr = random_rows(rng, n)
    size = ctypes.c_size_t()
    assert shim.gasloc_linear_workspace(ctx.c, m, k, ptr.ctypes.data, act, ctypes.byref(size)) == OK
    for name in ("gasloc_linear", "gasloc_linear_grad_input", "gasloc_linear_grad_weight"):
        changes = dict(weight=0, out_features=m, in_features=k, workspace_bytes=size.value)
        for key in calls(ptr)[name]:
            if key in ("x_ld", "dx_ld"):
                changes[key] = k
            if key in ("dout_ld", "out_ld"):
                changes[key] = m
            if key == "grad_ld":
                changes[key] = (m * k + 11) // 4 * 4
        assert call(ctx, name, ptr=ptr, act=act, **changes) == OK, shim.shim_error()
        plan = np.zeros(3 + 3 * n + 2, np.int64)
        shim.shim_linear_plan(n, plan.ctypes.data_as(ctypes.c_void_p))
        tile, vec, chunk = (int(v) for v in plan[:3])
        starts, parts, order = plan[3:4 + n], plan[4 + n:5 + 2 * n], plan[5 + 2 * n:]
        assert sorted(order) == list(range(n))
        assert tile in (16, 64, 128, 256) and (tile != 256 or (vec and act == BF16))
        step = 32 if act == BF16 else 16
        assert chunk % (4 * step) == 0
        used = 0
        cut = lambda v, t: -(-v // t)
        for s in range(n):
            w = order[s]
            rows = int(ptr[w + 1] - ptr[w])
            if name == "gasloc_linear_grad_weight":
                tiles, depth = cut(m, tile) * cut(k, tile), rows
            elif name == "gasloc_linear":
                tiles, depth = cut(rows, tile) * cut(m, tile), k
            else:
                tiles, depth = cut(rows, tile) * cut(k, tile), m
            count = int(parts[s + 1] - parts[s])
            assert count >= 1 and starts[s + 1] - starts[s] == tiles * count
            if chunk == 0:
                assert count == 1
            else:
                assert (count - 1) * chunk < max(depth, 1) <= max(count * chunk, 1)
        if chunk:
            used = (int(parts[n]) * m * k if name == "gasloc_linear_grad_weight"
                    else int(parts[1]) * int(ptr[-1]) * (m if name == "gasloc_linear" else k))
        assert 4 * used <= size.value


@pytest.mark.parametrize("seed", range(40))
def test_norm_and_embedding_workspaces_hold_their_partial_sums(shim, seed):
    rng = np.random.default_rng(100 + seed)
    n = int(rng.integers(1, 9))
    width = int(np.exp(rng.uniform(0, np.log(16_384))))
    ctx = Context(shim, n=n, P=4 * width + 100)
    ptr = random_rows(rng, n)
    size = ctypes.c_size_t()
    assert shim.gasloc_layer_norm_grad_workspace(ctx.c, width, ptr.ctypes.data, ctypes.byref(size)) == OK
    gld = (4 * width + 100 + 3) // 4 * 4
    lds = dict(x_ld=width, dout_ld=width, dx_ld=width)
    assert call(ctx, "gasloc_layer_norm_grad", ptr=ptr, width=width, gain=0, bias=width, grad_ld=gld,
                workspace_bytes=size.value, **lds) == OK, shim.shim_error()
    if size.value:
        assert call(ctx, "gasloc_layer_norm_grad", ptr=ptr, width=width, gain=0, bias=width, grad_ld=gld,
                    workspace_bytes=size.value - 256, **lds) == BAD
    plan = np.zeros(n + 2, np.int64)
    shim.shim_norm_plan(n, plan.ctypes.data_as(ctypes.c_void_p))
    rows = np.diff(ptr)
    assert np.array_equal(np.diff(plan[1:]), -(-rows // plan[0]))
    assert 2 * 4 * int(plan[-1]) * width <= size.value
    assert shim.gasloc_embedding_grad_workspace(ctx.c, width, ptr.ctypes.data, ctypes.byref(size)) == OK
    assert call(ctx, "gasloc_embedding_grad", ptr=ptr, vocab=3, width=width, dout_ld=width, grad_ld=gld,
                workspace_bytes=size.value) == OK, shim.shim_error()
    plan = np.zeros(n + 3, np.int64)
    shim.shim_sums_plan(n, plan.ctypes.data_as(ctypes.c_void_p))
    assert 1 <= plan[0] <= 256 and 1 <= plan[1] <= 256
    assert np.array_equal(np.diff(plan[2:]), -(-rows // plan[0]))
    sorts = 2 if rows.max() > 8192 else 1
    assert 8 * int(ptr[-1]) * sorts + 2 * 4 * int(plan[-1]) * width <= size.value


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no gcc")
    src = tmp_path / "use.c"
    src.write_text('#include "gasloc_layers.h"\nint main(void) { return gasloc_linear == 0; }\n')
    subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"),
                    "-fsyntax-only", "-Wno-address", str(src)], check=True, capture_output=True)


# --------------------------------------------------------------------------
# the binding
# --------------------------------------------------------------------------

def test_activation_types():
    import torch

    assert g.gasloc._act("bf16") == g.gasloc._act(torch.bfloat16) == BF16
    assert g.gasloc._act("f32") == g.gasloc._act(torch.float32) == F32
    with pytest.raises(ValueError):
        g.gasloc._act(torch.float16)


def test_tensor_checks():
    import torch

    rows = g.gasloc._rows_of
    cpu = torch.device("cpu")
    x = torch.zeros(6, 8)
    assert rows("x", x, 6, 8, torch.float32, cpu) == 8
    assert rows("x", x[:, :5], 4, 5, torch.float32, cpu) == 8
    assert rows("x", x[:1, :5], 1, 5, torch.float32, cpu) == 5
    assert rows("x", x[:0], 0, 8, torch.float32, cpu) == 8
    assert rows("x", x[::2, :1], 3, 1, torch.float32, cpu) == 16
    for bad in ((x, 7, 8, torch.float32), (x, 6, 7, torch.float32), (x, 6, 8, torch.bfloat16),
                (x.t(), 8, 6, torch.float32), (x[0], 1, 8, torch.float32), (x[:, ::2], 6, 4, torch.float32)):
        with pytest.raises(ValueError):
            rows("x", *bad, cpu)
    with pytest.raises(ValueError):
        rows("x", x, 6, 8, torch.float32, torch.device("meta"))
