"""CPU oracle of the layer operators: dropout, norms with gate and residual, products in 8-bit integers.

TEST INFRASTRUCTURE, NOT A PRODUCT PATH.  Plain double-precision numpy, written from the definitions; the gradients are written out by the
chain rule, one step per line.  Pins in tests/test_oracle_layers.py: finite differences, known generator words, values worked by hand.
"""
from __future__ import annotations

import numpy as np

from .cutoff_oracle import philox4x32_10, sigmoid

STREAM_DROPOUT = 0x400


def kept(rows: int, cols: int, p: float, seed: int, step: int, stream: int = STREAM_DROPOUT, first_row: int = 0) -> np.ndarray:
    """Which elements dropout keeps: sixteen bits of the generator each, eight columns to a counter."""
    border = int(np.rint(p * 65536))
    i = first_row + np.arange(rows, dtype=np.uint64)[:, None]
    j = np.arange(cols, dtype=np.uint64)[None, :]
    words = np.stack(np.broadcast_arrays(*philox4x32_10(j >> np.uint64(3), i, stream, step, seed & 0xFFFFFFFF, seed >> 32)))
    word = np.take_along_axis(words, np.broadcast_to((j % np.uint64(8) // np.uint64(2)).astype(np.int64), (rows, cols))[None], 0)[0]
    bits = np.where(j % np.uint64(2) == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    return bits >= border


def dropout(x, p, seed, step, stream=STREAM_DROPOUT, first_row=0, residual=None):
    dropped = int(np.rint(p * 65536))
    keep = kept(*x.shape, p, seed, step, stream, first_row)
    y = np.where(keep, x, 0.0) * (65536 / (65536 - dropped) if dropped < 65536 else 0.0)
    return y if residual is None else residual + y


def normalised(v, kind, eps):
    """(v - mean) / deviation of each row, and 1 / deviation."""
    if kind is None:
        return v, np.ones((len(v), 1))
    if kind == "layer":
        v = v - v.mean(1, keepdims=True)
    inv = 1.0 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return v * inv, inv


def gate_value(g, kind):
    """act(g) and its derivative."""
    s = sigmoid(g)
    return {"linear": (g, np.ones_like(g)), "sigmoid": (s, s * (1 - s)), "silu": (g * s, s * (1 + g * (1 - s)))}[kind]


def _parts(x, h, gate, gate_rows, gate_kind, scale, post, post_weight, post_bias, pre, pre_weight, pre_bias, eps):
    one, zero = np.ones(x.shape[1]), np.zeros(x.shape[1])
    d = {"scale": one if scale is None else scale, "w": one if post_weight is None else post_weight, "b": zero if post_bias is None else post_bias,
         "w2": one if pre_weight is None else pre_weight, "b2": zero if pre_bias is None else pre_bias}
    d["r"] = x
    if h is not None:
        d["hat"], d["inv"] = normalised(h, post, eps)
        d["p"] = d["hat"] * d["w"] + d["b"]
        d["a"], d["slope"] = np.ones_like(x), np.zeros_like(x)
        if gate is not None:
            d["group"] = np.arange(len(x)) // gate_rows
            d["a"], d["slope"] = (t[d["group"]] for t in gate_value(gate, gate_kind))
        d["r"] = x + d["scale"] * d["a"] * d["p"]
    d["r_hat"], d["r_inv"] = normalised(d["r"], pre, eps)
    d["n"] = d["r_hat"] * d["w2"] + d["b2"]
    return d


def residual_norm(x, h=None, gate=None, gate_rows=1, gate_kind="linear", scale=None, post="rms", post_weight=None, post_bias=None, pre="rms",
                  pre_weight=None, pre_bias=None, eps=1e-6):
    """(r, n): r = x + scale act(gate) post(h), n = pre(r)."""
    d = _parts(x, h, gate, gate_rows, gate_kind, scale, post, post_weight, post_bias, pre, pre_weight, pre_bias, eps)
    return d["r"], d["n"]


def _through_norm(g, hat, inv, kind):
    """The gradient at v, given the one at hat = (v - mean) inv."""
    if kind is None:
        return g
    if kind == "layer":
        g = g - g.mean(1, keepdims=True)
    return inv * (g - hat * (g * hat).mean(1, keepdims=True))


def residual_norm_grad(x, h, d_residual, d_norm, gate=None, gate_rows=1, gate_kind="linear", scale=None, post="rms", post_weight=None, post_bias=None,
                       pre="rms", pre_weight=None, pre_bias=None, eps=1e-6, sizes=False):
    """Gradients of residual_norm's inputs.  With sizes, of the sums among them also what their terms' magnitudes add up to."""
    d = _parts(x, h, gate, gate_rows, gate_kind, scale, post, post_weight, post_bias, pre, pre_weight, pre_bias, eps)
    zero = np.zeros_like(x)
    d_n = zero if d_norm is None else d_norm
    d_r = (zero if d_residual is None else d_residual) + _through_norm(d_n * d["w2"], d["r_hat"], d["r_inv"], pre)
    terms = {"pre_weight": d_n * d["r_hat"], "pre_bias": d_n}
    out = {"x": d_r}
    if h is not None:
        e = d_r * d["a"]
        terms.update(scale=e * d["p"], post_weight=e * d["scale"] * d["hat"], post_bias=e * d["scale"])
        out["h"] = _through_norm(e * d["scale"] * d["w"], d["hat"], d["inv"], post)
        if gate is not None:
            each = d_r * d["scale"] * d["p"] * d["slope"]
            out["gate"], magnitude = np.zeros_like(gate), np.zeros_like(gate)
            np.add.at(out["gate"], d["group"], each)
            np.add.at(magnitude, d["group"], np.abs(each))
    have = {"scale": scale, "post_weight": post_weight, "post_bias": post_bias, "pre_weight": pre_weight, "pre_bias": pre_bias}
    out.update({k: terms[k].sum(0) for k in have if have[k] is not None})
    if not sizes:
        return out
    size = {k: np.abs(terms[k]).sum(0) for k in have if have[k] is not None}
    if "gate" in out:
        size["gate"] = magnitude
    return out, size


def quantize_rows(x):
    """8-bit integers and scales of the rows of fp32 values x.  The single-precision steps are the definition's."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(x), axis=1)                     # NaN if there is one
        small = top < np.float32(2.0 ** -100)
        scale = np.where(small, np.float32(0), top / np.float32(127))
        inverse = np.where(small, np.float32(0), np.float32(127) / top)
        q = np.rint(x * inverse[:, None])
        q[~np.isfinite(q)] = 0
    return q.astype(np.int8), scale.astype(np.float32)


def quantized_product(a, a_scale, b, b_scale, bias=None):
    total = a.astype(np.int64) @ b.astype(np.int64).T
    with np.errstate(all="ignore"):
        y = total * a_scale.astype(np.float64)[:, None] * b_scale.astype(np.float64)
    return y if bias is None else y + bias
