"""The layer operators in calls that their users may make and that values alone do not cover: warps of which some lanes have no work."""
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
