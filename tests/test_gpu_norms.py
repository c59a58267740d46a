"""Norms before and after a block with gate and residual scale, and their gradients, through the C ABI, against the oracle in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from oracle import layers as L
from paper_1803_04209_b200 import binding, build
from layer_tools import TYPES, U, close, half_step, host, matrix, rounding, vector

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    build.build()
    return binding.load_library()


# A sum over a row is at most 16 additions in a thread and 10 across threads: 32 u of the magnitudes' mean, u = 2^-24.
def _norm_bound(v, hat, inv, kind, moved=0.0):
    """How far the normalised values may be off, the values themselves being off by `moved` (per element)."""
    if kind is None:
        return np.broadcast_to(moved, hat.shape)
    spread = np.abs(v) + np.abs(v).mean(1, keepdims=True)
    moved = np.max(np.broadcast_to(moved, hat.shape), 1, keepdims=True)
    return 40 * U * (np.abs(hat) + inv * spread) + 2 * inv * moved * (1 + np.abs(hat))


def _forward_bounds(x, h, o, dtype):
    """Bounds of r and n: the rounding of what is stored, and what the steps before it cost."""
    d = L._parts(x, h, **o)
    d_r = 0.0
    if h is not None:
        d_hat = _norm_bound(h, d["hat"], d["inv"], o["post"])
        branch = np.abs(d["scale"] * d["a"])
        # exp of a gate of up to 5: 8 steps of its own, the division and the products a few more
        d_r = branch * (np.abs(d["w"]) * d_hat + 30 * U * (np.abs(d["hat"] * d["w"]) + np.abs(d["b"]))) + 2 * U * (np.abs(x) + np.abs(d["r"]))
    d_n = _norm_bound(d["r"], d["r_hat"], d["r_inv"], o["pre"], d_r) * np.abs(d["w2"]) + 3 * U * (np.abs(d["r_hat"] * d["w2"]) + np.abs(d["b2"]))
    return d, d_r + rounding(d["r"], dtype) * 1.001, d_n + rounding(d["n"], dtype) * 1.001


def _case(rng, rows, cols, dt, post="rms", pre="rms", gate_rows=None, gate_kind="linear", bias=True, scale=True, weight=True, eps=1e-5, pad=0, offset=0,
          mean=0.0, block=True):
    """Arguments of the library and of the oracle."""
    x, x64 = matrix(rng, rows, cols, dt, pad, offset, mean=mean)
    h, h64 = matrix(rng, rows, cols, dt, pad, offset, std=2.0, mean=mean) if block else (None, None)
    dev, ref = {}, {}
    names = ["pre_weight"] * weight + ["pre_bias"] * bias
    if block:
        names += ["post_weight"] * weight + ["post_bias"] * bias + ["scale"] * scale
    for name in names:
        dev[name], ref[name] = vector(rng, cols, mean=0.0 if "bias" in name else 0.5)
    if gate_rows:
        dev["gate"], ref["gate"] = matrix(rng, -(-rows // gate_rows), cols, dt, pad, offset)
        dev["gate"].clamp_(-5, 5)
        ref["gate"] = host(dev["gate"])
    rest = {"post": post, "pre": pre, "gate_rows": gate_rows or 1, "gate_kind": gate_kind, "eps": eps}
    none = {k: None for k in ("gate", "scale", "post_weight", "post_bias", "pre_weight", "pre_bias")}
    return (x, h, {**dev, **rest}), (x64, h64, {**none, **ref, **rest})


SIZES = [(1, 1), (3, 5), (2, 32), (70, 33), (5, 128), (9, 129), (3, 256), (40, 257), (2, 512), (6, 513), (3, 1000), (600, 1024), (2, 2175), (1, 4096), (3, 8192), (2, 8191),
         (520, 2175), (513, 8192), (900, 1001), (2100, 100), (1500, 516)]


# both sides of every length at which another number of threads takes a row
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(dtype, rows, cols):
    rng = np.random.default_rng(rows * 10007 + cols)
    dt = TYPES[dtype]
    kind = ["rms", "layer", None][cols % 3]
    (x, h, o), (x64, h64, o64) = _case(rng, rows, cols, dt, post=kind, pre="layer" if cols % 2 else "rms", gate_rows=1 + cols % 2, gate_kind=["sigmoid", "silu"][cols % 2])
    d, b_r, b_n = _forward_bounds(x64, h64, o64, dt)
    r, n = binding.residual_norm(x, h, **o)
    close(r, d["r"], b_r, "r")
    close(n, d["n"], b_n, "n")


@pytest.mark.parametrize("post,pre", list(itertools.product([None, "rms", "layer"], repeat=2)))
@pytest.mark.parametrize("gate_rows,gate_kind", [(None, "linear"), (1, "sigmoid"), (3, "silu"), (100, "linear")])
@pytest.mark.parametrize("weights", [False, True])
def test_forward_kinds(post, pre, gate_rows, gate_kind, weights):
    rng = np.random.default_rng(5)
    (x, h, o), (x64, h64, o64) = _case(rng, 11, 136, torch.float32, post, pre, gate_rows, gate_kind, bias=weights, scale=weights, weight=weights)
    d, b_r, b_n = _forward_bounds(x64, h64, o64, torch.float32)
    r, n = binding.residual_norm(x, h, **o)
    close(r, d["r"], b_r, "r")
    close(n, d["n"], b_n, "n")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (0, 1), (3, 5)])
def test_strides_and_alignment(dtype, pad, offset):
    rng = np.random.default_rng(pad * 7 + offset)
    dt, rows, cols = TYPES[dtype], 13, 520
    (x, h, o), (x64, h64, o64) = _case(rng, rows, cols, dt, gate_rows=2, pad=pad, offset=offset)
    d, b_r, b_n = _forward_bounds(x64, h64, o64, dt)
    bufs = [torch.full((rows * (cols + pad) + offset,), -5.0, dtype=dt, device="cuda") for _ in range(2)]
    r, n = (b[offset:].view(rows, cols + pad)[:, :cols] for b in bufs)
    binding.residual_norm(x, h, residual_out=r, norm_out=n, **o)
    close(r, d["r"], b_r, "r")
    close(n, d["n"], b_n, "n")
    for b in bufs:
        assert torch.all(b[offset:].view(rows, cols + pad)[:, cols:] == -5.0) and torch.all(b[:offset] == -5.0)


def test_rows_far_from_zero_keep_their_deviations():
    rng = np.random.default_rng(2)
    (x, h, o), (x64, h64, o64) = _case(rng, 4, 777, torch.float32, post="layer", pre="layer", mean=1000.0)
    d, b_r, b_n = _forward_bounds(x64, h64, o64, torch.float32)
    r, n = binding.residual_norm(x, h, **o)
    close(r, d["r"], b_r)
    close(n, d["n"], b_n)
    assert b_n.max() < 0.05                                  # the bound itself says something


def test_without_a_block_and_without_a_norm():
    rng = np.random.default_rng(3)
    (x, _, o), (x64, _, o64) = _case(rng, 9, 300, torch.bfloat16, pre="layer", block=False)
    d, _, b_n = _forward_bounds(x64, None, o64, torch.bfloat16)
    r, n = binding.residual_norm(x, **o)
    assert r is x
    close(n, d["n"], b_n)
    (x, h, o), (x64, h64, o64) = _case(rng, 9, 300, torch.bfloat16)
    d, b_r, _ = _forward_bounds(x64, h64, o64, torch.bfloat16)
    r, n = binding.residual_norm(x, h, want_norm=False, **o)
    assert n is None
    close(r, d["r"], b_r)


def test_zero_rows_masked_values_and_nan():
    x = torch.zeros(4, 600, device="cuda")
    x[1, 3], x[2, 5], x[3] = float("nan"), float("inf"), torch.finfo(torch.float32).max
    r, n = binding.residual_norm(x, torch.zeros_like(x), pre="rms")
    assert torch.all(n[0] == 0) and bool(torch.isnan(n[1]).all()) and bool(torch.isnan(n[2, 5])) and torch.equal(n[2, :5], torch.zeros(5, device="cuda"))
    assert torch.all(n[3] == 0)                              # the squares overflow, as they would in any fp32 evaluation
    assert torch.equal(torch.nan_to_num(r), torch.nan_to_num(x))
    assert binding.residual_norm(torch.empty(0, 7, device="cuda"), torch.empty(0, 7, device="cuda"))[1].shape == (0, 7)


def test_in_place():
    rng = np.random.default_rng(4)
    for cols in (96, 520, 1000):
        (x, h, o), _ = _case(rng, 50, cols, torch.float16)
        r, n = binding.residual_norm(x, h, **o)
        x2, h2 = x.clone(), h.clone()
        binding.residual_norm(x2, h2, residual_out=x2, norm_out=h2, **o)
        assert torch.equal(x2, r) and torch.equal(h2, n)


# the 8-bit rows are those that quantising the unrounded fp32 rows gives, up to values that lie on a border between two integers
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 16), (7, 100), (3, 300), (2, 1000), (1, 4096), (5, 8192), (4, 2175), (700, 1024), (600, 1001), (3000, 48)])
def test_rows_in_8_bits(dtype, rows, cols):
    rng = np.random.default_rng(cols)
    dt = TYPES[dtype]
    (x, h, o), (x64, h64, o64) = _case(rng, rows, cols, dt, gate_rows=1, gate_kind="sigmoid")
    d, b_r, b_n = _forward_bounds(x64, h64, o64, torch.float32)
    r, q = binding.residual_norm(x, h, quantize=True, **o)
    close(r, d["r"], _forward_bounds(x64, h64, o64, dt)[1], "r")
    top = np.abs(d["n"]).max(1)
    close(q.scale, top / 127, b_n.max(1) / 127 + 4 * U * top / 127)
    values = host(q.values)
    assert np.all(np.abs(values).max(1) == 127)
    # value / scale is off by n's bound and by the scale's; rounding adds half a step
    at = d["n"] * (127 / top)[:, None]
    off = (b_n + np.abs(d["n"]) * (b_n.max(1) / top)[:, None]) * (127 / top)[:, None] + 8 * U * 127
    assert np.all(np.abs(values - at) <= 0.5 + off)


# ---- gradients ----------------------------------------------------------------------------------------------------------
# A value goes through at most ten steps of 40 u each, relative to the magnitudes that meet in it; the inputs are of order one and their
# deviation is no smaller than their mean.
STEPS = 400 * U


def _through(mag, hat, inv, kind):
    if kind is None:
        return mag
    return inv * (mag + mag.mean(1, keepdims=True) + np.abs(hat) * (mag * np.abs(hat)).mean(1, keepdims=True))


def _grad_check(x, h, o, x64, h64, o64, dt, with_r=True, with_n=True, seed=0, pad=0, offset=0):
    rng = np.random.default_rng(seed)
    rows, cols = x64.shape
    dr, dr64 = matrix(rng, rows, cols, dt, pad, offset) if with_r else (None, None)
    dn, dn64 = matrix(rng, rows, cols, dt, pad, offset) if with_n else (None, None)
    got = binding.residual_norm_grad(x, h, dr, dn, **o)
    want, size = L.residual_norm_grad(x64, h64, dr64, dn64, sizes=True, **o64)
    assert set(got) == set(want)
    d = L._parts(x64, h64, **o64)
    zero = np.zeros_like(x64)
    m_r = np.abs(dr64 if with_r else zero) + _through(np.abs((dn64 if with_n else zero) * d["w2"]), d["r_hat"], d["r_inv"], o64["pre"])
    spread = 1 + (d["r_inv"] * (np.abs(d["r"]).mean(1, keepdims=True) + np.abs(d["r"])).max(1, keepdims=True) if o64["pre"] else 0)
    b_x = STEPS * m_r * spread
    close(got["x"], want["x"], b_x + rounding(want["x"], dt) * 1.001, "x")
    extra = {}
    if h64 is not None:
        m_e = m_r * np.abs(d["a"] * d["scale"] * d["w"])
        spread2 = spread * (1 + (d["inv"] * (np.abs(h64).mean(1, keepdims=True) + np.abs(h64)).max(1, keepdims=True) if o64["post"] else 0))
        close(got["h"], want["h"], STEPS * _through(m_e, d["hat"], d["inv"], o64["post"]) * spread2 + rounding(want["h"], dt) * 1.001, "h")
        # p = hat w + b near zero: hat is off by 40 u (|hat| + inv (|h| + mean |h|)) <= 40 u (1 + |hat|) spread2, however small hat itself is,
        # so that what p is off by goes with |w| (1 + |hat|) + |b| and not with |p|
        m_p = np.abs(d["w"]) * (1 + np.abs(d["hat"])) + np.abs(d["b"])
        extra = {"scale": m_r * np.abs(d["a"]) * m_p, "post_weight": m_r * np.abs(d["a"] * d["scale"]) * (1 + np.abs(d["hat"])),
                 "post_bias": m_r * np.abs(d["a"] * d["scale"])}
        extra = {k: (v * spread2).sum(0) for k, v in extra.items()}
        if "gate" in want:
            each = m_r * spread2 * np.abs(d["scale"]) * m_p * (np.abs(d["slope"]) + 0.3)
            extra["gate"] = np.zeros_like(want["gate"])
            np.add.at(extra["gate"], d["group"], each)
    extra["pre_weight"] = (np.abs(dn64 if with_n else zero) * (1 + np.abs(d["r_hat"])) * spread).sum(0)
    extra["pre_bias"] = np.zeros(cols)
    for name, total in size.items():
        # a sum over the rows: chains of at most 256 additions, of terms that are off by STEPS of their magnitudes
        bound = 256 * U * total + STEPS * extra[name]
        if name == "gate":
            bound = bound + rounding(want[name], dt) * 1.001
        close(got[name], want[name], bound, name)
    return got, (dr, dn)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_gradients(dtype, rows, cols):
    rng = np.random.default_rng(rows * 10009 + cols)
    dt = TYPES[dtype]
    kind = ["rms", "layer", None][cols % 3]
    dev, ref = _case(rng, rows, cols, dt, post=kind, pre="layer" if cols % 2 else "rms", gate_rows=1 + cols % 2, gate_kind=["sigmoid", "silu"][cols % 2], eps=1e-2)
    _grad_check(*dev, *ref, dt)


@pytest.mark.parametrize("post,pre", list(itertools.product([None, "rms", "layer"], repeat=2)))
@pytest.mark.parametrize("gate_rows,gate_kind", [(None, "linear"), (1, "sigmoid"), (4, "silu"), (1000, "linear")])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cols", [40, 516])
def test_gradients_of_all_kinds(post, pre, gate_rows, gate_kind, bias, cols):
    rng = np.random.default_rng(6)
    dev, ref = _case(rng, 67, cols, torch.float32, post, pre, gate_rows, gate_kind, bias=bias, scale=bias or cols == 40)
    _grad_check(*dev, *ref, torch.float32)


# groups that end inside a team's rows, span several teams and CTAs, are all the rows; more rows than teams, and fewer
@pytest.mark.parametrize("rows,cols", [(5000, 24), (3000, 512), (2500, 520), (700, 1024)])
@pytest.mark.parametrize("gate_rows", [2, 7, 100, 999, 100000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_of_shared_gates(rows, cols, gate_rows, dtype):
    rng = np.random.default_rng(rows + gate_rows)
    dev, ref = _case(rng, rows, cols, TYPES[dtype], gate_rows=gate_rows, gate_kind="sigmoid", bias=False)
    _grad_check(*dev, *ref, TYPES[dtype])


# the most shared memory that a row takes: every operand, bias and group at the largest widths
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(5, 8192), (700, 8184), (3, 8190)])
@pytest.mark.parametrize("gate_rows", [1, 3])
def test_widest_rows(dtype, rows, cols, gate_rows):
    rng = np.random.default_rng(cols + gate_rows)
    dt = TYPES[dtype]
    dev, ref = _case(rng, rows, cols, dt, post="layer", gate_rows=gate_rows, gate_kind="silu", eps=1e-2)
    d, b_r, b_n = _forward_bounds(*ref, dt)
    r, n = binding.residual_norm(*dev[:2], **dev[2])
    close(r, d["r"], b_r, "r")
    close(n, d["n"], b_n, "n")
    _grad_check(*dev, *ref, dt)


@pytest.mark.parametrize("with_r,with_n", [(True, False), (False, True)])
@pytest.mark.parametrize("cols", [100, 1024])
def test_one_of_the_gradients_may_be_absent(with_r, with_n, cols):
    rng = np.random.default_rng(9)
    dev, ref = _case(rng, 30, cols, torch.bfloat16, gate_rows=1)
    _grad_check(*dev, *ref, torch.bfloat16, with_r, with_n)


@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradients_with_strides(pad, offset, dtype):
    rng = np.random.default_rng(10)
    dev, ref = _case(rng, 21, 528, TYPES[dtype], gate_rows=5, pad=pad, offset=offset)
    _grad_check(*dev, *ref, TYPES[dtype], pad=pad, offset=offset)


def test_gradients_without_a_block():
    rng = np.random.default_rng(11)
    dev, ref = _case(rng, 30, 1000, torch.float32, block=False, pre="layer")
    _grad_check(*dev, *ref, torch.float32)


def test_gradients_of_no_rows():
    x = torch.empty(0, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    g = binding.residual_norm_grad(x, x, x, x, gate=x, scale=w, pre_weight=w)
    assert g["x"].shape == (0, 40) and torch.all(g["scale"] == 0) and torch.all(g["pre_weight"] == 0)


# the library's gradient in single precision against differences of the oracle's forward pass in double
def test_gradients_against_differences():
    rng = np.random.default_rng(12)
    (x, h, o), (x64, h64, o64) = _case(rng, 6, 10, torch.float32, post="layer", pre="rms", gate_rows=4, gate_kind="silu")
    dr, dr64 = matrix(rng, 6, 10, torch.float32)
    dn, dn64 = matrix(rng, 6, 10, torch.float32)
    got = binding.residual_norm_grad(x, h, dr, dn, **o)

    def loss():
        r, n = L.residual_norm(x64, h64, **o64)
        return np.sum(r * dr64) + np.sum(n * dn64)
    for name, grad in got.items():
        flat = {"x": x64, "h": h64, **o64}[name].reshape(-1)
        grad, step = host(grad).reshape(-1), 1e-5
        for i in range(flat.size):
            keep = flat[i]
            flat[i] = keep + step
            up = loss()
            flat[i] = keep - step
            down = loss()
            flat[i] = keep
            # the difference's own error is of the order of step^2, the gradient's some hundred u
            assert abs((up - down) / (2 * step) - grad[i]) <= 1e-4 * (1 + abs(grad).max()), name


def test_same_bits_on_every_run_on_other_streams_and_replayed():
    rng = np.random.default_rng(13)
    for rows, cols in ((1500, 200), (800, 1536)):
        (x, h, o), _ = _case(rng, rows, cols, torch.bfloat16, gate_rows=77, gate_kind="sigmoid")
        dr, dn = torch.randn_like(x), torch.randn_like(x)
        want = binding.residual_norm_grad(x, h, dr, dn, **o)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                        # two calls at once, each with a workspace of its own
            other = binding.residual_norm_grad(x, h, dr, dn, **o)
        again = binding.residual_norm_grad(x, h, dr, dn, **o)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r, n = binding.residual_norm(x, h, **o)
            held = binding.residual_norm_grad(x, h, r, n, **o)
        graph.replay()
        r2, n2 = binding.residual_norm(x, h, **o)
        assert torch.equal(r, r2) and torch.equal(n, n2)
        for name, t in binding.residual_norm_grad(x, h, r2, n2, **o).items():
            assert torch.equal(held[name], t), name
        for name, t in want.items():
            assert torch.equal(t, other[name]) and torch.equal(t, again[name]), name


def test_refusals():
    x = torch.ones(4, 8, device="cuda")
    v = torch.ones(8, device="cuda")
    for kw in (dict(h=x.half()), dict(h=x[:3]), dict(h=x, gate=x[:3]), dict(h=x, gate=x, gate_rows=2), dict(h=x, gate_rows=0), dict(h=x, post="batch"),
               dict(h=x, scale=v[:7]), dict(h=x, scale=v.half()), dict(h=x, pre_weight=torch.ones(16, device="cuda")[::2]), dict(h=x.t()),
               dict(h=x, gate_kind="tanh"), dict(h=x, residual_out=torch.empty(4, 9, device="cuda")), dict(h=x, norm_out=x.bfloat16())):
        with pytest.raises(ValueError):
            binding.residual_norm(x, **kw)
    for kw in (dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        with pytest.raises(binding.CutoffError) as e:
            binding.residual_norm(x, x, **kw)
        assert e.value.code == binding.ERR_BAD_ARG
    for kw in (dict(scale=v), dict(post_weight=v), dict(gate=x)):                       # a block's parameters without a block
        with pytest.raises(binding.CutoffError) as e:
            binding.residual_norm(x, **kw)
        assert e.value.code == binding.ERR_BAD_ARG
    wide = torch.ones(1, 8193, device="cuda")
    with pytest.raises(binding.CutoffError) as e:
        binding.residual_norm(wide, wide)
    assert e.value.code == binding.ERR_TOO_LARGE
    with pytest.raises(binding.CutoffError) as e:
        binding.residual_norm_grad(wide, wide, wide, wide)
    assert e.value.code == binding.ERR_TOO_LARGE
    with pytest.raises(binding.CutoffError) as e:
        binding.residual_norm_grad(x, x, None, None)
    assert e.value.code == binding.ERR_BAD_ARG
