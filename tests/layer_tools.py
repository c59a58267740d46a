"""What the tests of the layer operators share: inputs, and how far a correctly rounded result may be off."""
import numpy as np
import torch

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24                                  # half a step of fp32


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def rounding(want, dtype):
    """What storing `want` in dtype may cost: half a step, absolute below the smallest normal number."""
    return half_step(dtype) * np.maximum(np.abs(want), torch.finfo(dtype).tiny)


def matrix(rng, rows, cols, dtype, pad=0, offset=0, std=1.0, mean=0.0):
    """A CUDA matrix and its values in 64 bits; rows `pad` values apart, the first value `offset` values into the buffer."""
    buf = torch.full((rows * (cols + pad) + offset + 16,), 7.0, dtype=dtype)
    view = buf[offset: offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] if rows else buf[:0].view(0, cols)
    view.copy_(torch.from_numpy(rng.standard_normal((rows, cols)) * std + mean))
    dev = buf.cuda()
    out = dev[offset: offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] if rows else dev[:0].view(0, cols)
    return out, view.double().numpy()


def vector(rng, cols, std=0.1, mean=1.0):
    v = (rng.standard_normal(cols) * std + mean).astype(np.float32)
    return torch.from_numpy(v).cuda(), v.astype(np.float64)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, bound, what=""):
    got = host(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    ok = ~np.isnan(want)
    off = np.abs(got - want)[ok]
    limit = np.broadcast_to(bound, want.shape)[ok]
    assert np.all(off <= limit), (what, float(off.max()), float((off / np.maximum(limit, 1e-300)).max()), int(np.argmax(off / np.maximum(limit, 1e-300))))
