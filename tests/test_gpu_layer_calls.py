"""The layer operators in calls that their users may make and that values alone do not cover: warps of which some lanes have no work, launches that the
runtime refuses, several host threads."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

from paper_1803_04209_b200 import binding, build

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
