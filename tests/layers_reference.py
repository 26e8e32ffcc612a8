"""The layer operators written out in fp64 with numpy, and how far fp32
arithmetic may be off (tests only).

U = 2^-24 is half a step of fp32 relative to the value, 2^-8 of bf16.  A sum of
m terms in fp32, whatever its order, is off by at most m U times the sum of the
terms' magnitudes (to first order; every bound below has a spare term for the
rest).  Additions inside a matrix instruction may be off by a whole step, so
products count 2 U each.
"""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 2.0 ** -126


def to_bf16(a):
    """fp64 holding fp32 values -> the nearest bf16 values (ties to even), as fp64."""
    b = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


def spans(row_ptr):
    return list(zip(row_ptr[:-1], row_ptr[1:]))


def embedding(tables, tokens, row_ptr, scale):
    """tables: [n, vocab, width]"""
    vocab, width = tables.shape[1:]
    out = np.zeros((row_ptr[-1], width))
    for i, (a, b) in enumerate(spans(row_ptr)):
        for t in range(a, b):
            if 0 <= tokens[t] < vocab:
                out[t] = scale * tables[i, tokens[t]]
    return out


def embedding_grad(n, vocab, tokens, row_ptr, dout, scale):
    """(gradient, bound)"""
    width = dout.shape[1]
    out, size, count = np.zeros((n, vocab, width)), np.zeros((n, vocab, width)), np.zeros((n, vocab, 1))
    for i, (a, b) in enumerate(spans(row_ptr)):
        k = tokens[a:b]
        real = (k >= 0) & (k < vocab)
        np.add.at(out[i], k[real], dout[a:b][real])
        np.add.at(size[i], k[real], np.abs(dout[a:b][real]))
        np.add.at(count[i], k[real], 1.0)
    return scale * out, (count + 3) * U * abs(scale) * size


def layer_norm(x, gain, bias, row_ptr, eps, act):
    """x [T, W], gain and bias [n, W]: (out, its bound, stats, their bound)"""
    worker = np.repeat(np.arange(len(row_ptr) - 1), np.diff(row_ptr))
    width = x.shape[1]
    mean = x.mean(1)
    d = x - mean[:, None]
    var = (d * d).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    hat = d * rstd[:, None]
    out = hat * gain[worker] + bias[worker]
    # a lane adds up to 32 values, a row of lanes 4 times, then 4 rows and up to 8 waves: at most 64 roundings
    e_mean = 68 * U * np.abs(x).mean(1)
    e_var = 2 * e_mean * np.abs(d).mean(1) + e_mean ** 2 + 72 * U * var
    e_rstd = e_var / (2 * (var + eps)) + 4 * U  # relative
    e = rstd[:, None] * (e_mean[:, None] + U * np.abs(d)) + np.abs(hat) * (e_rstd[:, None] + 4 * U)
    e = np.abs(gain[worker]) * e
    e = 1.01 * e + 2 * U * np.abs(out)
    e += (HALF_STEP[act] if act == "bf16" else 0) * (np.abs(out) + e) + TINY
    e_stats = np.stack((1.01 * e_mean, 1.01 * e_rstd * rstd), 1) + TINY
    return out, e, np.stack((mean, rstd), 1), e_stats


def layer_norm_grad(x, stats, gain, dout, row_ptr, act):
    """(dx, bound, dgain, bound, dbias, bound)"""
    n = len(row_ptr) - 1
    worker = np.repeat(np.arange(n), np.diff(row_ptr))
    mean, rstd = stats[:, :1], stats[:, 1:]
    hat = (x - mean) * rstd
    h = dout * gain[worker]
    m1, m2 = h.mean(1, keepdims=True), (h * hat).mean(1, keepdims=True)
    dx = rstd * (h - m1 - hat * m2)
    size = np.abs(h) + np.abs(h).mean(1, keepdims=True) + np.abs(hat) * np.abs(h * hat).mean(1, keepdims=True)
    e = 80 * U * rstd * size  # 64 roundings in a sum, as above, and those of the terms
    e += (HALF_STEP[act] if act == "bf16" else 0) * (np.abs(dx) + e) + TINY
    dgain, dbias = np.zeros((n, x.shape[1])), np.zeros((n, x.shape[1]))
    e_gain, e_bias = np.zeros_like(dgain), np.zeros_like(dbias)
    for i, (a, b) in enumerate(spans(row_ptr)):
        dgain[i], dbias[i] = (dout[a:b] * hat[a:b]).sum(0), dout[a:b].sum(0)
        e_gain[i] = (b - a + 8) * U * np.abs(dout[a:b] * hat[a:b]).sum(0)
        e_bias[i] = (b - a + 4) * U * np.abs(dout[a:b]).sum(0)
    return dx, e, dgain, e_gain + TINY, dbias, e_bias + TINY


def linear(w, x, row_ptr, act):
    """w [n, out, in] as the products take it: (out, bound)"""
    out = np.zeros((x.shape[0], w.shape[1]))
    size = np.zeros_like(out)
    for i, (a, b) in enumerate(spans(row_ptr)):
        out[a:b] = x[a:b] @ w[i].T
        size[a:b] = np.abs(x[a:b]) @ np.abs(w[i]).T
    e = 2 * (w.shape[2] + 4) * U * size
    return out, e + (HALF_STEP[act] if act == "bf16" else 0) * (np.abs(out) + e) + TINY


def linear_grad_input(w, dout, row_ptr, act):
    return linear(np.ascontiguousarray(w.transpose(0, 2, 1)), dout, row_ptr, act)


def linear_grad_weight(x, dout, row_ptr):
    n = len(row_ptr) - 1
    out = np.zeros((n, dout.shape[1], x.shape[1]))
    e = np.zeros_like(out)
    for i, (a, b) in enumerate(spans(row_ptr)):
        out[i] = dout[a:b].T @ x[a:b]
        e[i] = 2 * (b - a + 4) * U * (np.abs(dout[a:b]).T @ np.abs(x[a:b]))
    return out, e + TINY


# Products whose tiles are 128 outputs a side, on 256 CUs: with many outputs, and with sums long enough to be split.
# (pass, activations, split) -> row_ptr, out_features, in_features
LARGE = {
    ("linear", "f32", False): ([0, 1400, 2100], 4104, 72),
    ("linear", "bf16", False): ([0, 700, 1100], 4104, 72),
    ("linear_grad_input", "f32", False): ([0, 1400, 2100], 72, 4104),
    ("linear_grad_input", "bf16", False): ([0, 700, 1100], 72, 4104),
    ("linear_grad_weight", "f32", False): ([0, 50, 77], 2056, 2064),
    ("linear_grad_weight", "bf16", False): ([0, 50, 77], 2056, 1032),
}
for _act in ("f32", "bf16"):
    LARGE["linear", _act, True] = ([0, 400, 528], 264, 72_008)
    LARGE["linear_grad_input", _act, True] = ([0, 400, 528], 72_008, 264)
    LARGE["linear_grad_weight", _act, True] = ([0, 50_011, 80_000], 264, 520)
