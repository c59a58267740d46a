"""The layer operators in calls that their users may make and that values alone do not cover: warps of which some lanes have no work, launches that the
runtime refuses, several host threads, tensors that autograd knows; gates far from zero, and of very many rows."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

from paper_1803_04209_b200 import binding, build
from layer_tools import TYPES, U, close, host, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    build.build()
    return binding.load_library()


# Tiles whose sums are split over a cluster, with 1 to 31 channels in their last warp: its lanes part at the stores, before the cluster's barrier.
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m", [2, 15, 31, 50, 64])
@pytest.mark.parametrize("n", [1, 31, 33, 97, 127, 129, 1023])
def test_split_tiles_with_channels_that_fill_no_warp(m, n, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m * 1000 + n)
    for k in (512, 1040, 4096):
        a, b = (torch.randint(-127, 128, (rows, k), dtype=torch.int8, device="cuda", generator=gen) for rows in (m, n))
        a_scale, b_scale = torch.full((m,), 2.0 ** -9, device="cuda"), torch.full((n,), 2.0 ** -9, device="cuda")
        total = a.cpu().numpy().astype(np.int64) @ b.cpu().numpy().astype(np.int64).T       # below 2^26
        # sums and powers of two: one rounding to fp32 where a sum takes more than 24 bits, and the result's own
        want = torch.from_numpy(total.astype(np.float32) * np.float32(2.0 ** -18)).to(dtype)
        for _ in range(3):
            y = binding.quantized_product((a, a_scale), (b, b_scale), dtype=dtype)
            assert torch.equal(y.cpu(), want)


# ---- launches that the runtime refuses -------------------------------------------------------------------------------------------
class _Capture:
    """While it is open, a launch on the legacy default stream is refused: a blocking stream is being captured.  Host errors only."""

    def __enter__(self):
        self.cuda, self.stream = C.CDLL("libcuda.so.1"), C.c_void_p()
        assert self.cuda.cuStreamCreate(C.byref(self.stream), 0) == 0
        assert self.cuda.cuStreamBeginCapture_v2(self.stream, 2) == 0           # relaxed: torch may allocate meanwhile
        return self

    def __exit__(self, *_):
        graph = C.c_void_p()
        self.cuda.cuStreamEndCapture(self.stream, C.byref(graph))                # the refused launch has ended the capture: no graph
        assert not graph.value and self.cuda.cuStreamDestroy_v2(self.stream) == 0


def _calls():
    """The calls by name, their outputs fixed, so that nothing but the launches can fail."""
    x = torch.randn(40, 640, device="cuda", dtype=torch.bfloat16)
    many = binding.quantize_rows(torch.randn(2600, 256, device="cuda"))
    q, w = binding.quantize_rows(x), binding.quantize_rows(torch.randn(200, 640, device="cuda"))
    v = torch.ones(640, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    out, one, large = (torch.empty(m, n, device="cuda", dtype=torch.bfloat16) for m, n in ((40, 200), (1, 200), (2600, 2600)))
    return {
        "dropout": lambda: binding.dropout(x, 0.5, 1, out=y),
        "norm": lambda: binding.residual_norm(x, x, residual_out=y, norm_out=z),
        "gradients": lambda: binding.residual_norm_grad(x, x, x, x, scale=v),
        "quantise": lambda: binding.quantize_rows(x),
        "product of one token": lambda: binding.quantized_product((q.values[:1], q.scale[:1]), w, out=one),
        "product": lambda: binding.quantized_product(q, w, out=out),
        "large product": lambda: binding.quantized_product(many, many, out=large),
    }


def test_a_refused_launch_is_an_error_of_its_own_call_alone():
    calls = _calls()
    for call in calls.values():                                                  # warm: the allocator has its blocks
        call()
    torch.cuda.synchronize()
    for name, call in calls.items():
        with _Capture():
            with pytest.raises(binding.CutoffError) as e:
                call()
            assert e.value.code == binding.ERR_CUDA, name
        for after in calls.values():
            after()                                                              # raises if it is told of the refused one
    torch.cuda.synchronize()


def test_an_unknown_device_is_an_error_of_its_own_call_alone():
    lib, x = binding.load_library(), torch.ones(4, 16, device="cuda")
    at = x.data_ptr()
    assert lib.cutoff_dropout(1000, 0, 4, 16, at, 16, None, 0, at, 16, 0.5, 1, 0, 0, 0, None) == binding.ERR_CUDA
    for call in _calls().values():
        call()


# ---- host threads ----------------------------------------------------------------------------------------------------------------
def _gradient_calls(cols, rounds, failed, written, barrier):
    """Gradients of rows of this width on a stream of this thread's own, through the C ABI; what calls returned, and what they had written."""
    lib = binding.load_library()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        x = torch.randn(64, cols, device="cuda", dtype=torch.bfloat16)
        w, got = torch.ones(cols, device="cuda"), torch.empty(cols, device="cuda")
        ws = torch.empty(lib.cutoff_residual_norm_grad_workspace_bytes(64, cols), dtype=torch.uint8, device="cuda")
        layer = binding.NormLayer(64, cols, binding.TYPE_BF16, x.data_ptr(), cols, x.data_ptr(), cols, None, 0, 1, 0, 1, 1, 1e-6, w.data_ptr())
        grads = binding.NormGrads(scale=got.data_ptr())
        args = (0, C.byref(layer), x.data_ptr(), cols, x.data_ptr(), cols, C.byref(grads), ws.data_ptr(), ws.numel(), stream.cuda_stream)
        stream.synchronize()
        barrier.wait()
        for i in range(rounds):
            if i % 256 == 0:
                stream.synchronize()
            got.fill_(-7.0)
            rc = lib.cutoff_residual_norm_grad(*args)
            if rc != binding.OK:
                failed.append(rc)
                stream.synchronize()
                if not bool((got == -7.0).all()):
                    written.append(rc)
        stream.synchronize()


def _in_threads(rounds=4000):
    failed, written, barrier = [], [], threading.Barrier(4)
    threads = [threading.Thread(target=_gradient_calls, args=(cols, rounds, failed, written, barrier)) for cols in (8192, 4096, 8192, 5120)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return failed, written


def test_a_call_that_fails_has_written_no_sums():
    failed, written = _in_threads()
    assert not written, (len(failed), len(written))


def test_threads_with_rows_of_several_widths_do_not_fail_one_another():
    failed, _ = _in_threads()
    assert not failed, len(failed)


def _forward_calls(cols, rounds, failed, barrier):
    lib = binding.load_library()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        x = torch.randn(2000, cols, device="cuda")
        n = torch.empty_like(x)
        layer = binding.NormLayer(2000, cols, binding.TYPE_FP32, x.data_ptr(), cols, x.data_ptr(), cols, None, 0, 1, 0, 1, 1, 1e-6)
        stream.synchronize()
        barrier.wait()
        for i in range(rounds):
            if i % 64 == 0:
                stream.synchronize()
            rc = lib.cutoff_residual_norm(0, C.byref(layer), None, 0, n.data_ptr(), cols, None, stream.cuda_stream)
            if rc != binding.OK:
                failed.append(rc)
        stream.synchronize()


def test_threads_with_norms_of_several_widths_do_not_fail_one_another():
    failed, barrier = [], threading.Barrier(4)
    threads = [threading.Thread(target=_forward_calls, args=(cols, 4000, failed, barrier)) for cols in (8192, 6144, 8192, 5120)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, len(failed)


# ---- gates far from zero ---------------------------------------------------------------------------------------------------------
def _gates(dtype, cols):
    """Gates of all sizes, the ends among them, as rows; and their values in 64 bits."""
    rng = np.random.default_rng(cols)
    g = np.concatenate([np.linspace(-110, 110, 2201), rng.standard_normal(2000) * 5, 10.0 ** rng.uniform(-30, 0, 500), -(10.0 ** rng.uniform(-30, 0, 500)),
                        [0.0, -0.0, 87.0, -87.0, 88.5, -88.5, 104.0, -104.0, 1e4, -1e4, np.inf, -np.inf, np.nan]])
    g = torch.from_numpy(np.resize(g, (-(-len(g) // cols), cols))).to(TYPES[dtype]).cuda()
    return g, host(g)


def _logistic(g):
    """Value and derivative of the sigmoid in 64 bits, neither of them a difference of neighbours."""
    u = np.exp(-np.abs(g))
    value = np.where(np.isnan(g), np.nan, np.where(g < 0, u / (1 + u), 1 / (1 + u)))
    return value, u / (1 + u) ** 2


def _gate_bounds(g, dtype):
    """How far value and derivative of the sigmoid may be off, relative to themselves, and absolutely.

    fp32: exp(-|g|) is off by 2 steps = 4 U; 1 + it is rounded (U), its reciprocal 1 step = 2 U off: 5 U with half of the exponential's error; their product is
    4 + 5 + 1 = 10 U off, and once more times the reciprocal 16 U.  16 bits: the exponent |g| log2(e) is rounded twice, by U each, which the exponential
    multiplies by |g|; results below 2^-126 may be 0."""
    if dtype == "fp32":
        return 10 * U, 16 * U, 2.0 ** -148
    steps = 2 * np.minimum(np.abs(np.nan_to_num(g, nan=0.0, posinf=200.0, neginf=-200.0)), 200.0) * U
    return 10 * U + steps, 16 * U + steps, 2.0 ** -126


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
@pytest.mark.parametrize("cols,gate_rows", [(24, 1), (25, 1), (512, 1), (1024, 1), (1001, 1), (1024, 2), (1001, 3), (40, 5)])
def test_gates_of_any_size(dtype, kind, cols, gate_rows):
    gate, g = _gates(dtype, cols)
    rows = len(g) * gate_rows
    x, h = torch.zeros(rows, cols, device="cuda", dtype=gate.dtype), torch.ones(rows, cols, device="cuda", dtype=gate.dtype)
    kw = dict(gate=gate, gate_rows=gate_rows, gate_kind=kind, post=None, pre=None)
    r, _ = binding.residual_norm(x, h, want_norm=False, **kw)                    # 0 + act(gate) * 1
    grads = binding.residual_norm_grad(x, h, h, None, **kw)                      # the gate's: the derivative, gate_rows times
    with np.errstate(invalid="ignore"):
        value, slope = _logistic(g)
        value_off, slope_off, least = _gate_bounds(g, dtype)
        value_off, slope_off = value_off * value, slope_off * slope
        if kind == "silu":
            value, slope, value_off, slope_off = g * value, value + g * slope, np.abs(g) * (value_off + U * value), value_off + np.abs(g) * (slope_off + U * slope)
            slope_off = slope_off + U * np.abs(slope)
            least = least * np.maximum(1, np.abs(g))
    value_off, slope_off = (np.where(np.isfinite(off), off, 0) for off in (value_off + least, slope_off + least))      # what is not finite is compared exactly
    each, bound = np.repeat(value, gate_rows, 0), np.repeat(value_off, gate_rows, 0)
    finite = np.isfinite(each)
    got = host(r)
    assert np.array_equal(got[~finite], each[~finite], equal_nan=True)           # infinities and NaN as the formula has them
    close(r.masked_fill(torch.from_numpy(~finite).cuda(), 0), np.where(finite, each, 0), bound + rounding(np.where(finite, each, 0), gate.dtype) * 1.001, "value")
    close(grads["h"].masked_fill(torch.from_numpy(~finite).cuda(), 0), np.where(finite, each, 0), bound + rounding(np.where(finite, each, 0), gate.dtype) * 1.001, "h")
    total = slope * gate_rows
    finite = np.isfinite(total)
    assert np.array_equal(host(grads["gate"])[~finite], total[~finite], equal_nan=True)
    total = np.where(finite, total, 0)
    bound = gate_rows * slope_off + gate_rows * U * np.abs(total) + rounding(total, gate.dtype) * 1.001
    close(grads["gate"].masked_fill(torch.from_numpy(~finite).cuda(), 0), total, bound, "gate")


# ---- tensors that autograd knows ---------------------------------------------------------------------------------------------------
def test_tensors_that_require_a_gradient_are_refused_and_taken_without_one():
    x = torch.randn(6, 64, device="cuda")
    leaf, w, q = x.clone().requires_grad_(), torch.ones(64, device="cuda").requires_grad_(), binding.quantize_rows(x)
    calls = [lambda t, w: binding.dropout(t, 0.5, 1), lambda t, w: binding.dropout(x, 0.5, 1, residual=t), lambda t, w: binding.residual_norm(t),
             lambda t, w: binding.residual_norm(x, t), lambda t, w: binding.residual_norm(x, x, gate=t), lambda t, w: binding.residual_norm(x, x, scale=w),
             lambda t, w: binding.residual_norm(x, pre_weight=w), lambda t, w: binding.residual_norm_grad(x, x, t, x),
             lambda t, w: binding.residual_norm_grad(x, x, x, x, post_bias=w), lambda t, w: binding.quantize_rows(t),
             lambda t, w: binding.quantized_product(q, q, bias=w[:6], dtype=torch.float32)]
    flat = lambda r: list(r.values()) if isinstance(r, dict) else list(r) if isinstance(r, tuple) else [r]
    for i, call in enumerate(calls):
        for t, v in ((leaf, w), (leaf * 1.0, w * 1.0)):
            with pytest.raises(ValueError, match="requires a gradient"):
                call(t, v)
        want = flat(call(x, w.detach()))
        with torch.no_grad():
            got = flat(call(leaf, w))
        with torch.inference_mode():
            inferred = flat(call(x, w))
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, inferred)), i


def test_autograd_learns_of_results_written_over_what_it_keeps():
    x = torch.randn(6, 64, device="cuda")
    writes = [lambda t: binding.dropout(x, 0.5, 1, out=t), lambda t: binding.residual_norm(x, x, residual_out=t), lambda t: binding.residual_norm(x, x, norm_out=t),
              lambda t: binding.quantized_product(binding.quantize_rows(x), binding.quantize_rows(torch.ones(64, 64, device="cuda")), out=t)]
    for write in writes:
        leaf = x.clone().requires_grad_()
        kept = leaf.exp()                                    # whose gradient needs it as it is
        write(kept.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.sum().backward()
    with torch.inference_mode():
        out = torch.empty_like(x)
        binding.dropout(x, 0.5, 1, out=out)
    assert torch.equal(out, binding.dropout(x, 0.5, 1))


# ---- gates that many rows share ----------------------------------------------------------------------------------------------------
# One gate for all rows, and terms of one sign whose sum takes more digits than fp32 has: an addition that follows on too many others rounds the same way
# over and over.  A sum of n terms in chains and trees of at most `depth` additions is off by depth u of the magnitudes, u = 2^-24.  Rows per team, then at
# most 32 teams of a CTA, then 16 parts of at most 592 CTAs, then the 16: 11 + 32 + 37 + 16 = 96 for the first case, 22 + 8 + 37 + 16 and 34 + 4 + 28 + 16.
@pytest.mark.parametrize("rows,cols", [(200000, 24), (100000, 128), (60000, 500)])
@pytest.mark.parametrize("value", [1 + 2.0 ** -10, 1 + 2.0 ** -9 + 2.0 ** -11])
def test_a_gate_of_very_many_rows(rows, cols, value):
    x, h, d = torch.zeros(rows, cols, device="cuda"), torch.ones(rows, cols, device="cuda"), torch.full((rows, cols), value, device="cuda")
    gate = torch.ones(1, cols, device="cuda")
    got = binding.residual_norm_grad(x, h, d, None, gate=gate, gate_rows=rows, post=None, pre=None)["gate"]
    want = rows * value
    assert np.abs(host(got) - want).max() <= (96 + 1) * U * want


# groups on both sides of a team's and of a CTA's rows: a group inside a team, across teams of one CTA, across two CTAs and many
@pytest.mark.parametrize("rows,cols", [(40000, 24), (9473, 32), (20011, 100), (7000, 512), (1201, 600)])
@pytest.mark.parametrize("gate_rows", [2, 3, 33, 64, 65, 337, 1000, 9472])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_sums_over_groups(rows, cols, gate_rows, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + gate_rows)
    dt, groups = TYPES[dtype], -(-rows // gate_rows)
    x, h = torch.zeros(rows, cols, device="cuda", dtype=dt), torch.ones(rows, cols, device="cuda", dtype=dt)
    # small whole numbers: every sum is exact in fp32, in any order
    d = torch.randint(-4, 5, (rows, cols), device="cuda", generator=gen).to(dt)
    gate = torch.randint(1, 4, (groups, cols), device="cuda", generator=gen).to(dt)
    kw = dict(gate=gate, gate_rows=gate_rows, post=None, pre=None)
    got = binding.residual_norm_grad(x, h, d, None, **kw)
    group = torch.arange(rows, device="cuda") // gate_rows
    want = torch.zeros(groups, cols, device="cuda").index_add_(0, group, d.float())
    assert torch.equal(got["gate"], want.to(dt)) and torch.equal(got["x"], d) and torch.equal(got["h"], (d.float() * gate.float()[group]).to(dt))
    again = binding.residual_norm_grad(x, h, d, None, **kw)
    assert all(torch.equal(got[k], again[k]) for k in got)


# ---- single rows -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("k", [1, 17, 513, 1001, 4095])
def test_the_distance_of_a_single_row_may_be_any(k):
    gen = torch.Generator(device="cuda").manual_seed(k)
    token = torch.randint(-127, 128, (1, k), dtype=torch.int8, device="cuda", generator=gen)               # contiguous, as its owner has it
    many = torch.randint(-127, 128, (40, (k + 15) // 16 * 16), dtype=torch.int8, device="cuda", generator=gen)[:, :k]
    one, scales = torch.ones(1, device="cuda"), torch.ones(40, device="cuda")
    want = (token.long().cpu() @ many.long().cpu().T).float()                                               # below 2^27: rounded once
    assert torch.equal(binding.quantized_product((token, one), (many, scales), dtype=torch.float32).cpu(), want)
    assert torch.equal(binding.quantized_product((many, scales), (token, one), dtype=torch.float32).cpu(), want.T)
    square = (token.long() ** 2).sum().float()
    assert torch.equal(binding.quantized_product((token, one), (token, one), dtype=torch.float32)[0, 0], square)
    with pytest.raises(binding.CutoffError) as e:                                                           # two rows are a distance apart
        binding.quantized_product((torch.zeros(2, 17, dtype=torch.int8, device="cuda"), scales[:2]), (torch.zeros(1, 17, dtype=torch.int8, device="cuda"), one))
    assert e.value.code == binding.ERR_BAD_ARG
