"""Pins of the layer operators' oracle: finite differences, known generator words, values worked by hand."""
import itertools

import numpy as np
import pytest

from oracle import cutoff_oracle as O
from oracle import layers as L


def test_kept_bits_are_the_half_words_of_the_generator():
    seed, step, stream, row0 = 0x1122334455667788, 7, 0x400, 1000
    keep = L.kept(3, 21, 0.5, seed, step, stream, row0)
    for i, j in itertools.product(range(3), range(21)):
        words = [int(w) for w in O.philox4x32_10(j // 8, row0 + i, stream, step, seed % 2 ** 32, seed >> 32)]
        bits = words[j % 8 // 2] >> 16 * (j % 2) & 0xFFFF
        assert keep[i, j] == (bits >= 32768)


def test_dropout_keeps_the_mean_and_honours_the_ends():
    x = np.ones((400, 1000))
    for p in (0.0, 0.1, 0.37, 0.9):
        y = L.dropout(x, p, 3, 4)
        scale = 65536 / (65536 - round(p * 65536))
        assert set(np.unique(y)) <= {0.0, scale}
        # 400000 draws: five deviations
        assert abs(np.mean(y == 0) - p) <= 5 * np.sqrt(p * (1 - p) / x.size) + 2.0 ** -17
    assert np.all(L.dropout(np.full((2, 9), np.nan), 1.0, 0, 0, residual=np.full((2, 9), 2.0)) == 2.0)


def test_rows_can_be_drawn_in_parts():
    whole = L.kept(10, 33, 0.3, 5, 6)
    assert np.array_equal(whole[4:], L.kept(6, 33, 0.3, 5, 6, first_row=4))


def test_norms_of_a_row_worked_by_hand():
    x, h = np.array([[1.0, 3.0]]), np.array([[3.0, -4.0]])
    r, n = L.residual_norm(x, h, gate=np.array([[2.0, 0.5]]), scale=np.array([1.0, 2.0]), post="rms", post_weight=np.array([1.0, 3.0]), pre="layer", eps=1e-300)
    # rms(h) = sqrt(12.5); r = x + scale * gate * weight * h / rms
    want = np.array([[1 + 2 * 3 / 12.5 ** 0.5, 3 - 2 * 0.5 * 3 * 4 / 12.5 ** 0.5]])
    np.testing.assert_allclose(r, want, rtol=1e-14)
    # a layer norm of two values gives +-1
    np.testing.assert_allclose(n, [[1.0, -1.0]] if want[0, 0] > want[0, 1] else [[-1.0, 1.0]], rtol=1e-12)


@pytest.mark.parametrize("post,pre", list(itertools.product([None, "rms", "layer"], repeat=2)))
@pytest.mark.parametrize("gate_rows,gate_kind", [(None, "linear"), (1, "silu"), (2, "sigmoid"), (5, "linear")])
def test_gradients_against_central_differences(post, pre, gate_rows, gate_kind):
    rng = np.random.default_rng(1)
    rows, cols = 5, 4
    v = {"x": rng.standard_normal((rows, cols)), "h": rng.standard_normal((rows, cols)), "scale": rng.standard_normal(cols),
         "post_weight": rng.standard_normal(cols), "post_bias": rng.standard_normal(cols), "pre_weight": rng.standard_normal(cols),
         "pre_bias": rng.standard_normal(cols)}
    rest = {"post": post, "pre": pre, "eps": 1e-3}
    if gate_rows:
        v["gate"] = rng.standard_normal((-(-rows // gate_rows), cols))
        rest.update(gate_rows=gate_rows, gate_kind=gate_kind)
    d_r, d_n = rng.standard_normal((2, rows, cols))

    def loss():
        r, n = L.residual_norm(**v, **rest)
        return np.sum(r * d_r) + np.sum(n * d_n)
    grads = L.residual_norm_grad(v["x"], v["h"], d_r, d_n, **{k: t for k, t in v.items() if k not in ("x", "h")}, **rest)
    assert set(grads) == set(v)
    for name, t in v.items():
        flat, step = t.reshape(-1), 1e-6
        for i in range(flat.size):
            keep = flat[i]
            flat[i] = keep + step
            up = loss()
            flat[i] = keep - step
            down = loss()
            flat[i] = keep
            assert abs((up - down) / (2 * step) - grads[name].reshape(-1)[i]) <= 1e-6 * max(1.0, abs(grads[name]).max())


def test_quantised_rows_worked_by_hand():
    q, s = L.quantize_rows(np.array([[1.0, -2.0, 0.5, 127.0], [0, 0, 0, 0], [1e-38, 0, 0, 0], [np.nan, 1, 2, 3], [np.inf, 1, -2, 3]], np.float32))
    assert q[:3].tolist() == [[1, -2, 0, 127], [0, 0, 0, 0], [0, 0, 0, 0]]        # 0.5 ties to even
    assert s[:3].tolist() == [1.0, 0.0, 0.0] and np.isnan(s[3]) and np.isinf(s[4])
    y = L.quantized_product(q, s, q[:1], s[:1], bias=np.array([3.0]))
    assert y[0, 0] == 1 + 4 + 127 * 127 + 3 and y[1, 0] == 3 and np.isnan(y[3, 0]) and np.isnan(y[4, 0])
