"""Dropout from the counter-based generator, through the C ABI, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from paper_1803_04209_b200 import binding, build
from layer_tools import TYPES, U, close, matrix, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    build.build()
    return binding.load_library()


def _bound(want, x, scale, residual, dtype):
    # the factor and the product are rounded once each, the sum once more, then the result
    terms = np.abs(x) * scale + (0 if residual is None else np.abs(residual))
    return 3 * U * terms + rounding(want, dtype) * (1 + 4 * U)


# one column to many, both sides of every width at which lanes share rows or columns fall into tiles; one row and many
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (1, 16), (33, 17), (2, 64), (9, 65), (7, 256), (4, 257), (1, 2175), (3, 4096), (1000, 24), (130, 1000)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_values_and_mask(dtype, rows, cols, with_residual):
    rng = np.random.default_rng(rows * 10007 + cols)
    dt, p, seed, step = TYPES[dtype], 0.3, 0x0123456789ABCDEF, 41
    x, x64 = matrix(rng, rows, cols, dt, std=2.0)
    res, res64 = matrix(rng, rows, cols, dt) if with_residual else (None, None)
    want = L.dropout(x64, p, seed, step, residual=res64)
    got = binding.dropout(x, p, seed, step, residual=res)
    close(got, want, _bound(want, x64, 65536 / (65536 - round(p * 65536)), res64, dt))
    if not with_residual:
        assert np.array_equal(got.cpu().numpy() == 0 if dt != torch.bfloat16 else (got == 0).cpu().numpy(), ~L.kept(rows, cols, p, seed, step) | (x64 == 0))


# rows further apart than they are long, starts that are not on 16 bytes; what lies between the rows stays
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (0, 1), (3, 5), (64, 8)])
def test_strides_and_alignment(dtype, pad, offset):
    rng = np.random.default_rng(pad * 31 + offset)
    dt, rows, cols = TYPES[dtype], 37, 264
    x, x64 = matrix(rng, rows, cols, dt, pad, offset)
    buf = torch.full((rows * (cols + pad) + offset,), -5.0, dtype=dt, device="cuda")
    out = buf[offset:].view(rows, cols + pad)[:, :cols]
    got = binding.dropout(x, 0.25, 9, 2, out=out)
    assert got.data_ptr() == out.data_ptr()
    want = L.dropout(x64, 0.25, 9, 2)
    close(out, want, _bound(want, x64, 4 / 3, None, dt))
    assert torch.all(buf[offset:].view(rows, cols + pad)[:, cols:] == -5.0) and torch.all(buf[:offset] == -5.0)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 0.5, 1 - 2.0 ** -16, 1.0])
def test_ends_of_the_range(p):
    rng = np.random.default_rng(3)
    x, x64 = matrix(rng, 64, 100, torch.float32)
    want = L.dropout(x64, p, 77, 1)
    close(binding.dropout(x, p, 77, 1), want, 3 * U * np.abs(want))


def test_a_dropped_value_is_not_looked_at():
    x = torch.full((8, 300), float("nan"), device="cuda", dtype=torch.bfloat16)
    x[::2] = float("inf")
    res = torch.full_like(x, 2.0)
    assert torch.all(binding.dropout(x, 1.0, 1, 1, residual=res) == 2.0)
    half = binding.dropout(x, 0.5, 1, 1)
    keep = L.kept(8, 300, 0.5, 1, 1)
    assert np.array_equal((half == 0).cpu().numpy(), ~keep)
    assert bool(torch.isnan(half[1]).any()) and bool(torch.isinf(half[0]).any())


def test_rows_in_parts_and_in_any_type_share_one_mask():
    x = torch.ones(1000, 515, device="cuda")
    whole = binding.dropout(x, 0.4, 5, 6) != 0
    for dt in TYPES.values():
        parts = [binding.dropout(x[i: i + 300].to(dt), 0.4, 5, 6, first_row=i) != 0 for i in range(0, 1000, 300)]
        assert torch.equal(torch.cat(parts), whole)
    last = binding.dropout(x[:1], 0.4, 5, 6, first_row=2 ** 32 - 1) != 0
    assert np.array_equal(last.cpu().numpy(), L.kept(1, 515, 0.4, 5, 6, first_row=2 ** 32 - 1))
    for other in (dict(seed=6), dict(step=7), dict(noise_stream=0x401)):
        kw = {"seed": 5, "step": 6, **other}
        assert not torch.equal(binding.dropout(x, 0.4, **kw) != 0, whole)


def test_gradient_is_the_same_call_and_agrees_with_differences():
    rng = np.random.default_rng(8)
    x, x64 = matrix(rng, 6, 50, torch.float32)
    dy, dy64 = matrix(rng, 6, 50, torch.float32)
    grad = binding.dropout(dy, 0.3, 11, 12)
    # the map is linear: a step of 1 in one value changes the loss by its gradient
    base = L.dropout(x64, 0.3, 11, 12)
    for i, j in ((0, 0), (2, 17), (5, 49), (3, 8), (1, 33)):
        moved = x64.copy()
        moved[i, j] += 1.0
        want = np.sum((L.dropout(moved, 0.3, 11, 12) - base) * dy64)
        assert abs(grad[i, j].item() - want) <= 1e-6


def test_in_place_and_on_another_stream_and_replayed():
    x = torch.randn(513, 1024, device="cuda", dtype=torch.bfloat16)
    want = binding.dropout(x, 0.2, 1, 2, residual=x)
    y = x.clone()
    assert torch.equal(binding.dropout(y, 0.2, 1, 2, residual=y, out=y), want) and torch.equal(y, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = x.clone()
        for _ in range(5):
            torch.cuda._sleep(200000)
            z = binding.dropout(z, 0.0, 1, 2)
        got = binding.dropout(z, 0.2, 1, 2, residual=z)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    fixed = x.clone()
    with torch.cuda.graph(graph):
        out = binding.dropout(fixed, 0.2, 1, 2, residual=fixed)
    for k in range(3):
        fixed.copy_(x + k)
        graph.replay()
        assert torch.equal(out, binding.dropout(x + k, 0.2, 1, 2, residual=x + k))


def test_no_rows():
    assert binding.dropout(torch.empty(0, 5, device="cuda"), 0.5, 1).shape == (0, 5)


def test_refusals():
    x = torch.ones(4, 8, device="cuda")
    with pytest.raises(ValueError):
        binding.dropout(x.double(), 0.1, 1)
    with pytest.raises(ValueError):
        binding.dropout(x.t(), 0.1, 1)
    with pytest.raises(ValueError):
        binding.dropout(x[:1].expand(4, 8), 0.1, 1)
    with pytest.raises(ValueError):
        binding.dropout(x.cpu(), 0.1, 1)
    with pytest.raises(ValueError):
        binding.dropout(x, 0.1, 1, residual=x.half())
    with pytest.raises(ValueError):
        binding.dropout(x, 0.1, 1, out=torch.empty(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        binding.dropout(x, 0.1, 1 << 64)
    for kw in (dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(p=0.1, first_row=-1), dict(p=0.1, first_row=2 ** 32 - 3)):
        with pytest.raises(binding.CutoffError) as e:
            binding.dropout(x, seed=1, **kw)
        assert e.value.code == binding.ERR_BAD_ARG
