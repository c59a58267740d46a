"""Quantised rows and products in 8-bit integers, through the C ABI, against exact integer sums."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from paper_1803_04209_b200 import binding, build
from layer_tools import TYPES, U, close, host, matrix, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (5, 16, 0), (2, 1000, 3), (7, 2048, 0), (4, 2175, 0), (1, 20001, 0), (300, 64, 8)])
def test_quantised_rows(dtype, rows, cols, pad):
    rng = np.random.default_rng(cols)
    x, x64 = matrix(rng, rows, cols, TYPES[dtype], pad)
    q = binding.quantize_rows(x)
    want, scale = L.quantize_rows(x64)
    assert np.array_equal(q.values.cpu().numpy(), want) and np.array_equal(q.scale.cpu().numpy(), scale)
    assert q.values.stride(0) % 16 == 0 or rows == 1


def test_quantised_rows_at_the_ends_of_the_range():
    x = torch.zeros(8, 100, device="cuda")
    x[1, 3], x[2, 4], x[3, 99], x[4, 0], x[5, :] = 1e-38, float("nan"), float("inf"), 2.0 ** -100, torch.finfo(torch.float32).max
    x[6, :2] = torch.tensor([127.0, 0.5])
    x[7, :3] = torch.tensor([-127.0, 1.5, 2.5])
    q = binding.quantize_rows(x)
    want, scale = L.quantize_rows(host(x))
    finite = np.isfinite(scale)
    assert finite.sum() == 6 and np.array_equal(q.values.cpu().numpy()[finite], want[finite])
    np.testing.assert_array_equal(q.scale.cpu().numpy(), scale)


def _operand(rng, rows, k, full=False):
    """8-bit rows 16 bytes apart from one another, what lies behind them set to values that would show, and scales."""
    ld = (k + 15) // 16 * 16
    v = rng.integers(-127, 128, (rows, ld), dtype=np.int64)
    if full:
        v[:, :k] = np.where(rng.random((rows, 1)) < 0.5, 127, -127)
    v = v.astype(np.int8)
    scale = rng.uniform(0.01, 0.1, rows).astype(np.float32)
    return (torch.from_numpy(v).cuda()[:, :k], torch.from_numpy(scale).cuda()), v[:, :k], scale


def _bound(want, total, a_scale, b_scale, bias, dt):
    # the sum becomes a float, is scaled twice and added to: four roundings of their magnitudes, then the result's
    mag = np.abs(total) * a_scale.astype(np.float64)[:, None] * b_scale + (0 if bias is None else np.abs(bias))
    return 4 * U * mag + rounding(want, dt) * 1.001


# one token to many, both sides of every border between kernels and tiles, inner lengths that end inside a chunk of 16, 32, 64 and 128
SIZES = [(1, 1, 1), (1, 8, 16), (2, 5, 17), (1, 300, 4096), (3, 129, 130), (8, 128, 512), (9, 64, 100), (16, 256, 128), (17, 200, 1000), (33, 130, 33),
         (64, 1024, 256), (64, 9600, 384), (65, 127, 129), (128, 128, 128), (129, 257, 640), (200, 513, 1001), (256, 256, 2048), (257, 600, 96), (300, 8, 48), (1000, 130, 272),
         (2, 2048, 8192), (48, 640, 8192), (100, 2175, 513), (1024, 1024, 512), (300, 512, 4096), (200, 5000, 640),
         (1300, 2300, 200), (4000, 2000, 129), (20, 6000, 300), (31, 5000, 2000), (100, 4000, 1024), (5, 1, 40), (128, 128, 4096)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_products(m, n, k, dtype):
    rng = np.random.default_rng(m * 101 + n * 11 + k)
    a, av, a_s = _operand(rng, m, k)
    b, bv, b_s = _operand(rng, n, k)
    with_bias = (m + n) % 2 == 0
    bias = rng.standard_normal(n).astype(np.float32) if with_bias else None
    dt = TYPES[dtype]
    total = (av.astype(np.float64) @ bv.astype(np.float64).T)             # exact: below 2^53
    # the scales bring fp16 results into its range
    fix = np.float32(1.0 / max(1.0, np.abs(total).max() * 0.01 / 3e4))
    a_s = (a_s * fix).astype(np.float32)
    a = (a[0], torch.from_numpy(a_s).cuda())
    want = total * a_s.astype(np.float64)[:, None] * b_s.astype(np.float64) + (0 if bias is None else bias.astype(np.float64))
    got = binding.quantized_product(a, b, None if bias is None else torch.from_numpy(bias).cuda(), dtype=dt)
    close(got, want, _bound(want, total, a_s, b_s, bias, dt))


# sums at the largest magnitude: 127 * 127 * k needs 31 bits at the longest rows, and differs from its neighbours in the last one
@pytest.mark.parametrize("m", [1, 40, 300])
@pytest.mark.parametrize("k", [binding.PRODUCT_MAX_K, 65536])
def test_the_longest_sums_are_exact(m, k):
    rng = np.random.default_rng(k)
    a, av, _ = _operand(rng, m, k, full=True)
    b, bv, _ = _operand(rng, 24, k, full=True)
    one = torch.ones(max(m, 24), device="cuda")
    got = binding.quantized_product((a[0], one[:m].contiguous()), (b[0], one[:24].contiguous()), dtype=torch.float32)
    want = av[:, 0].astype(np.int64)[:, None] * bv[:, 0].astype(np.int64) * k
    assert np.array_equal(got.cpu().numpy(), want.astype(np.float32))


def test_strided_results_leave_what_is_between_the_rows():
    rng = np.random.default_rng(1)
    for m, n, k, pad in ((5, 100, 64, 3), (70, 100, 64, 1), (300, 300, 192, 8), (130, 256, 128, 64)):
        a, av, a_s = _operand(rng, m, k)
        b, bv, b_s = _operand(rng, n, k)
        buf = torch.full((m, n + pad), -5.0, device="cuda", dtype=torch.bfloat16)
        binding.quantized_product(a, b, out=buf[:, :n])
        total = av.astype(np.float64) @ bv.astype(np.float64).T
        want = total * a_s.astype(np.float64)[:, None] * b_s
        close(buf[:, :n], want, _bound(want, total, a_s, b_s, None, torch.bfloat16))
        assert torch.all(buf[:, n:] == -5.0)


def test_operands_further_apart_than_they_are_long():
    rng = np.random.default_rng(2)
    for m, n, k in ((3, 70, 200), (150, 70, 200), (40, 300, 1024)):
        big_a = torch.from_numpy(rng.integers(-127, 128, (m, k + 64)).astype(np.int8)).cuda()
        big_b = torch.from_numpy(rng.integers(-127, 128, (n + 2, k + 48)).astype(np.int8)).cuda()
        a, b = big_a[:, 16: 16 + k] if k % 16 == 0 else big_a[:, :k], big_b[2:, :k]
        if a.stride(0) % 16 or b.stride(0) % 16:
            a = torch.nn.functional.pad(a, (0, -k % 16))[:, :k]
            b = torch.nn.functional.pad(b, (0, -k % 16))[:, :k]
        one = torch.ones(max(m, n), device="cuda")
        got = binding.quantized_product((a, one[:m].contiguous()), (b, one[:n].contiguous()), dtype=torch.float32)
        assert np.array_equal(host(got), a.cpu().numpy().astype(np.float64) @ b.cpu().numpy().astype(np.float64).T)


def test_rows_that_hold_nan_or_infinity_stay_to_themselves():
    x = torch.randn(70, 256, device="cuda")
    x[3, 5], x[40, 0] = float("nan"), float("inf")
    x[50] = 0
    w = binding.quantize_rows(torch.randn(130, 256, device="cuda"))
    for rows in (slice(0, 4), slice(0, 70)):
        y = binding.quantized_product(binding.quantize_rows(x[rows]), w, dtype=torch.float32)
        bad = ~torch.isfinite(y).all(1)
        assert torch.equal(bad.nonzero().flatten().cpu(), torch.tensor([i for i in (3, 40) if i < len(y)]))
        assert bool(torch.isnan(y[3]).all())
    assert torch.all(y[50] == 0)


def test_same_bits_on_every_run_on_other_streams_and_replayed():
    rng = np.random.default_rng(3)
    for m, n, k in ((1, 2048, 4096), (48, 1024, 4096), (300, 700, 512)):
        x = torch.randn(m, k, device="cuda", dtype=torch.bfloat16)
        w = binding.quantize_rows(torch.randn(n, k, device="cuda"))
        want = binding.quantized_product(binding.quantize_rows(x), w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = []
        with torch.cuda.stream(side):
            for _ in range(10):
                got.append(binding.quantized_product(binding.quantize_rows(x), w))
        for _ in range(10):                                  # at the same time
            got.append(binding.quantized_product(binding.quantize_rows(x), w))
        side.synchronize()
        assert all(torch.equal(g, want) for g in got)
        graph = torch.cuda.CUDAGraph()
        fixed = x.clone()
        with torch.cuda.graph(graph):
            y = binding.quantized_product(binding.quantize_rows(fixed), w)
        for s in (1.0, -2.0):
            fixed.copy_(x * s)
            graph.replay()
            assert torch.equal(y, binding.quantized_product(binding.quantize_rows(x * s), w))


def test_no_rows():
    a = binding.Quantized(torch.empty(0, 32, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"))
    w = binding.quantize_rows(torch.randn(9, 32, device="cuda"))
    assert binding.quantized_product(a, w).shape == (0, 9)
    assert binding.quantize_rows(torch.empty(0, 5, device="cuda")).values.shape == (0, 5)


def test_refusals():
    a = binding.quantize_rows(torch.randn(4, 32, device="cuda"))
    w = binding.quantize_rows(torch.randn(9, 32, device="cuda"))
    one = torch.ones(9, device="cuda")
    for bad in (lambda: binding.quantized_product(a, (w.values[:, :31], w.scale)), lambda: binding.quantized_product((a.values.short(), a.scale), w),
                lambda: binding.quantized_product(a, (w.values, w.scale[:8])), lambda: binding.quantized_product(a, w, bias=one[:8]),
                lambda: binding.quantized_product(a, w, out=torch.empty(4, 8, device="cuda")), lambda: binding.quantized_product(a, w, dtype=torch.float64),
                lambda: binding.quantize_rows(torch.ones(3, 4, device="cuda", dtype=torch.int8)), lambda: binding.quantize_rows(torch.ones(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros(9, 40, dtype=torch.int8, device="cuda")[:, :32]                    # rows 40 bytes apart
    off = torch.zeros(9, 64, dtype=torch.int8, device="cuda")[:, 8:40]                   # rows that start 8 bytes off
    for b in (odd, off):
        with pytest.raises(binding.CutoffError) as e:
            binding.quantized_product(a, (b, one))
        assert e.value.code == binding.ERR_BAD_ARG
    k = binding.PRODUCT_MAX_K + 1
    long = torch.zeros(1, k, dtype=torch.int8, device="cuda")
    with pytest.raises(binding.CutoffError) as e:
        binding.quantized_product((long, one[:1]), (long, one[:1]))
    assert e.value.code == binding.ERR_TOO_LARGE
