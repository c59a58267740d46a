"""What the layer operators refuse before they touch a device."""
import ctypes as C

import numpy as np
import pytest

from paper_1803_04209_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


P = 4096                     # an address that nothing may look at


def _dropout(lib, **kw):
    a = dict(device=0, type=0, rows=4, cols=8, x=P, x_ld=8, residual=None, residual_ld=0, y=P, y_ld=8, p=0.5, seed=1, step=0, noise_stream=0, first_row=0, stream=None)
    a.update(kw)
    return lib.cutoff_dropout(*a.values())


@pytest.mark.parametrize("kw", [dict(device=-1), dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=0), dict(x=None), dict(y=None), dict(x_ld=7), dict(y_ld=7),
                                dict(residual=P, residual_ld=7), dict(x=P + 2), dict(y=P + 1), dict(type=1, x=P + 1), dict(x_ld=2 ** 39), dict(p=-1e-9), dict(p=1.0000001), dict(p=float("nan")), dict(first_row=-1),
                                dict(first_row=2 ** 32 - 3), dict(rows=2 ** 32 + 1)])
def test_dropout(lib, kw):
    assert _dropout(lib, **kw) == binding.ERR_BAD_ARG


def test_no_rows_need_no_device(lib):
    assert _dropout(lib, rows=0) == binding.OK
    assert lib.cutoff_quantize_rows(0, 0, 0, 8, P, 8, P, 16, P, None) == binding.OK
    assert lib.cutoff_quantized_product(0, 0, 8, 16, P, 16, P, P, 16, P, None, 0, P, 8, None) == binding.OK
    assert lib.cutoff_residual_norm(0, C.byref(_layer(rows=0)), P, 8, P, 8, None, None) == binding.OK


def _layer(**kw):
    a = dict(rows=4, cols=8, type=0, x=P, x_ld=8, h=P, h_ld=8, gate=None, gate_ld=0, gate_rows=1, gate_kind=0, post=1, pre=1, eps=1e-6, scale=None,
             post_weight=None, post_bias=None, pre_weight=None, pre_bias=None)
    a.update(kw)
    return binding.NormLayer(*a.values())


BAD_LAYERS = [dict(rows=-1), dict(rows=2 ** 30 + 1), dict(x=P + 2), dict(h=P + 1), dict(scale=P + 2), dict(pre_bias=P + 1), dict(x_ld=2 ** 39), dict(cols=0), dict(type=7), dict(x=None), dict(x_ld=7), dict(h_ld=7), dict(gate=P, gate_ld=7), dict(gate=P, gate_ld=8, gate_rows=0),
              dict(gate_kind=3), dict(gate_kind=-1), dict(post=3), dict(pre=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
              dict(h=None, scale=P), dict(h=None, gate=P, gate_ld=8), dict(h=None, post_weight=P), dict(h=None, post_bias=P)]


@pytest.mark.parametrize("kw", BAD_LAYERS)
def test_norm_layers(lib, kw):
    r, r_ld = (None, 0) if kw.get("h", P) is None else (P, 8)
    assert lib.cutoff_residual_norm(0, C.byref(_layer(**kw)), r, r_ld, P, 8, None, None) == binding.ERR_BAD_ARG
    ws = 1 << 30
    assert lib.cutoff_residual_norm_grad(0, C.byref(_layer(**kw)), P, 8, P, 8, C.byref(binding.NormGrads()), P, ws, None) == binding.ERR_BAD_ARG


def test_norms(lib):
    def call(layer, *args):
        return lib.cutoff_residual_norm(0, layer, *args, None)
    ok = C.byref(_layer())
    assert call(None, P, 8, P, 8, None) == binding.ERR_BAD_ARG
    assert call(ok, None, 0, None, 0, None) == binding.ERR_BAD_ARG                      # nothing wanted
    assert call(ok, P, 7, P, 8, None) == binding.ERR_BAD_ARG
    assert call(ok, P, 8, P, 7, None) == binding.ERR_BAD_ARG
    assert call(ok, P, 8, None, 0, P) == binding.ERR_BAD_ARG                            # scales of rows that are not wanted
    assert call(C.byref(_layer(h=None)), P, 8, P, 8, None) == binding.ERR_BAD_ARG       # r without a block
    assert call(C.byref(_layer(cols=8193, x_ld=8193, h_ld=8193)), P, 8193, None, 0, None) == binding.ERR_TOO_LARGE


def test_norm_gradients(lib):
    G = binding.NormGrads
    need = lib.cutoff_residual_norm_grad_workspace_bytes(4, 8)
    assert need > 0 and lib.cutoff_residual_norm_grad_workspace_bytes(-1, 8) < 0 and lib.cutoff_residual_norm_grad_workspace_bytes(4, 8193) < 0
    ok = C.byref(_layer())

    def call(layer=ok, dr=P, dr_ld=8, dn=P, dn_ld=8, grads=C.byref(G()), ws=P, size=need):
        return lib.cutoff_residual_norm_grad(0, layer, dr, dr_ld, dn, dn_ld, grads, ws, size, None)
    for kw in (dict(layer=None), dict(dr=None, dn=None), dict(dr_ld=7), dict(dn_ld=7), dict(grads=None), dict(ws=None), dict(ws=P + 4), dict(size=need - 1),
               dict(grads=C.byref(G(x=P, x_ld=7))), dict(grads=C.byref(G(h=P, h_ld=7))), dict(grads=C.byref(G(gate=P, gate_ld=8))), dict(grads=C.byref(G(scale=P))),
               dict(grads=C.byref(G(post_weight=P))), dict(grads=C.byref(G(post_bias=P))), dict(grads=C.byref(G(pre_weight=P))), dict(grads=C.byref(G(pre_bias=P))),
               dict(layer=C.byref(_layer(h=None)), grads=C.byref(G(h=P, h_ld=8)))):
        assert call(**kw) == binding.ERR_BAD_ARG, kw
    assert call(layer=C.byref(_layer(cols=8193, x_ld=8193, h_ld=8193)), dr_ld=8193, dn_ld=8193) == binding.ERR_TOO_LARGE


def test_products(lib):
    def quantize(device=0, type=0, rows=4, cols=8, x=P, x_ld=8, q=P, q_ld=8, scale=P):
        return lib.cutoff_quantize_rows(device, type, rows, cols, x, x_ld, q, q_ld, scale, None)
    for kw in (dict(device=-1), dict(type=3), dict(rows=-1), dict(rows=2 ** 31), dict(cols=0), dict(x=None), dict(q=None), dict(scale=None), dict(x_ld=7), dict(q_ld=7), dict(x=P + 2), dict(scale=P + 2)):
        assert quantize(**kw) == binding.ERR_BAD_ARG, kw

    def product(device=0, m=4, n=8, k=16, a=P, a_ld=16, a_scale=P, b=P, b_ld=16, b_scale=P, bias=None, type=0, y=P, y_ld=8):
        return lib.cutoff_quantized_product(device, m, n, k, a, a_ld, a_scale, b, b_ld, b_scale, bias, type, y, y_ld, None)
    for kw in (dict(device=-1), dict(m=-1), dict(m=2 ** 31), dict(n=0), dict(k=0), dict(a=None), dict(a_scale=None), dict(b=None), dict(b_scale=None), dict(type=5), dict(y=None),
               dict(a_ld=15), dict(b_ld=24), dict(y_ld=7), dict(a=P + 8), dict(b=P + 1), dict(y=P + 2), dict(bias=P + 2), dict(b_ld=2 ** 39)):
        assert product(**kw) == binding.ERR_BAD_ARG, kw
    assert product(k=131072, a_ld=131072, b_ld=131072) == binding.ERR_TOO_LARGE
    assert product(n=2 ** 30 + 1, y_ld=2 ** 31) == binding.ERR_TOO_LARGE
    assert quantize(cols=2 ** 30 + 1, x_ld=2 ** 31, q_ld=2 ** 31) == binding.ERR_TOO_LARGE
    assert _dropout(lib, cols=2 ** 30 + 1, x_ld=2 ** 31, y_ld=2 ** 31) == binding.ERR_TOO_LARGE


def test_longest_sum_fits_32_bits():
    assert binding.PRODUCT_MAX_K * 128 * 128 <= np.iinfo(np.int32).max
