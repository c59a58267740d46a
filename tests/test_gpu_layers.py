"""The layer operators together, as a residual block is trained and served, and at sizes and orders of calls that one operator's tests do not reach."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layers as L
from paper_1803_04209_b200 import binding, build
from layer_tools import U, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    build.build()
    return binding.load_library()


# ---- training: x -> pre-norm -> linear layer -> dropout -> post-norm, gate, scale -> residual stream -> final norm -> loss -------
def _block(ops, p, x, w, step):
    """Loss and gradients of one block; ops: the library's or the oracle's functions, on arrays of their kind."""
    _, n = ops["norm"](x, None, pre="rms", pre_weight=p["w0"], post=None)
    h = n @ w.T
    d = ops["dropout"](h, 0.25, 99, step)
    kw = dict(gate=p["gate"], gate_rows=8, gate_kind="sigmoid", scale=p["scale"], post="rms", post_weight=p["w1"], pre="layer", pre_weight=p["w2"], pre_bias=p["b2"])
    r, out = ops["norm"](x, d, **kw)
    loss = 0.5 * (out * out).sum() + (r * r).sum()
    g = ops["grad"](x, d, 2 * r, out, **kw)
    d_h = ops["dropout"](g["h"], 0.25, 99, step)
    first = ops["grad"](x, None, g["x"], d_h @ w, pre="rms", pre_weight=p["w0"], post=None)
    return loss, {"x": first["x"], "w": d_h.T @ n, "w0": first["pre_weight"], "gate": g["gate"], "scale": g["scale"], "w1": g["post_weight"], "w2": g["pre_weight"],
                  "b2": g["pre_bias"]}


GPU = {"norm": binding.residual_norm, "grad": binding.residual_norm_grad, "dropout": lambda v, p, seed, step: binding.dropout(v, p, seed, step)}
CPU = {"norm": L.residual_norm, "grad": L.residual_norm_grad, "dropout": lambda v, p, seed, step: L.dropout(v, p, seed, step)}


def _problem(seed=0, rows=32, cols=48):
    rng = np.random.default_rng(seed)
    p = {"w0": 1 + 0.1 * rng.standard_normal(cols), "gate": rng.standard_normal((rows // 8, cols)), "scale": 0.5 + 0.1 * rng.standard_normal(cols),
         "w1": 1 + 0.1 * rng.standard_normal(cols), "w2": 1 + 0.1 * rng.standard_normal(cols), "b2": 0.1 * rng.standard_normal(cols)}
    x, w = rng.standard_normal((rows, cols)), rng.standard_normal((cols, cols)) / cols ** 0.5
    as32 = {k: np.float32(v) for k, v in p.items()}
    dev = {k: torch.from_numpy(v).cuda() for k, v in as32.items()}
    return {k: v.astype(np.float64) for k, v in as32.items()}, np.float64(np.float32(x)), np.float64(np.float32(w)), dev, torch.from_numpy(np.float32(x)).cuda(), torch.from_numpy(np.float32(w)).cuda()


def test_a_blocks_gradients_against_the_oracle_and_differences():
    p, x, w, dp, dx, dw = _problem()
    want_loss, want = _block(CPU, p, x, w, 3)
    loss, got = _block(GPU, dp, dx, dw, 3)
    assert abs(loss.item() - want_loss) <= 1e-4 * abs(want_loss)
    for name in want:
        # a dozen steps of some 100 u each, relative to the largest value
        assert np.abs(host(got[name]) - want[name]).max() <= 2000 * U * np.abs(want[name]).max(), name
    rng = np.random.default_rng(1)
    for name, t in {**p, "x": x, "w": w}.items():
        flat, grad = t.reshape(-1), host(got[name]).reshape(-1)
        for i in rng.choice(flat.size, 5, replace=False):
            keep = flat[i]
            flat[i] = keep + 1e-5
            up, _ = _block(CPU, p, x, w, 3)
            flat[i] = keep - 1e-5
            down, _ = _block(CPU, p, x, w, 3)
            flat[i] = keep
            assert abs((up - down) / 2e-5 - grad[i]) <= 1e-3 * (1 + np.abs(grad).max()), (name, i)


def test_a_block_trains_with_the_librarys_adam_in_a_graph():
    _, _, _, p, x, w = _problem(2)
    names = ["w0", "scale", "w1", "w2", "b2"]
    cols = x.shape[1]
    flat = torch.cat([p[k] for k in names]).clone()
    grads, m, v = (torch.zeros_like(flat) for _ in range(3))
    norm, ws = torch.zeros(1, device="cuda"), torch.empty(4096, dtype=torch.uint8, device="cuda")
    lib = binding.load_library()

    def step(t):
        q = {**p, **{k: flat[i * cols: (i + 1) * cols] for i, k in enumerate(names)}}
        loss, g = _block(GPU, q, x, w, t)
        torch.cat([g[k] for k in names], out=grads)
        assert lib.cutoff_adam_step(0, flat.numel(), flat.data_ptr(), grads.data_ptr(), m.data_ptr(), v.data_ptr(), t, 1e-2, 0.9, 0.999, 1e-8, 10.0, 1.0, norm.data_ptr(),
                                    ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
        return loss
    start = flat.clone()
    losses = [step(t).item() for t in range(1, 6)]
    assert all(np.isfinite(losses)) and not torch.equal(flat, start)
    # the same five steps, the last of them replayed from a graph: the same bits
    want = flat.clone()
    flat.copy_(start), m.zero_(), v.zero_()
    for t in range(1, 5):
        step(t)
    keep = [s.clone() for s in (flat, m, v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(5)
    for s, k in zip((flat, m, v), keep):
        s.copy_(k)
    graph.replay()
    assert torch.equal(flat, want) and held.item() == losses[-1]


# ---- serving: norm -> 8-bit product -> norm -> 8-bit product, one token at a time and many ----------------------------------------
@pytest.mark.parametrize("cols,hidden", [(256, 1024), (250, 333)])
def test_a_served_block_gives_a_token_the_same_alone_and_in_a_batch(cols, hidden):
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((70, cols))).cuda().bfloat16()
    w_in = binding.quantize_rows(torch.from_numpy(rng.standard_normal((hidden, cols)) / cols ** 0.5).float().cuda())
    w_out = binding.quantize_rows(torch.from_numpy(rng.standard_normal((cols, hidden)) / hidden ** 0.5).float().cuda())
    weight = torch.from_numpy(np.float32(1 + 0.1 * rng.standard_normal(cols))).cuda()

    def block(x):
        _, n = binding.residual_norm(x, pre_weight=weight, quantize=True)
        h = torch.relu(binding.quantized_product(n, w_in))
        y = binding.quantized_product(binding.quantize_rows(h), w_out)
        return binding.residual_norm(x, y, post_weight=weight, pre_weight=weight)
    r, n = block(x)
    for i in (0, 1, 33, 69):
        ri, ni = block(x[i: i + 1])
        # integer sums are exact, and a row's norm takes the same steps whatever stands beside it
        assert torch.equal(ri[0], r[i]) and torch.equal(ni[0], n[i])
    # against the plain computation in 64 bits: 8-bit operands are half a step of 1/127 of a row's largest value off, over sums of
    # independent errors; a tenth of the result's spread is far more than they can add up to, and far less than a wrong channel
    x64 = host(x)
    _, n64 = L.residual_norm(x64, pre_weight=host(weight))
    y64 = np.maximum(n64 @ (host(w_in.values) * host(w_in.scale)[:, None]).T, 0) @ (host(w_out.values) * host(w_out.scale)[:, None]).T
    want, _ = L.residual_norm(x64, y64, post_weight=host(weight), pre_weight=host(weight))
    assert np.abs(host(r) - want).max() <= 0.1 * want.std() + 0.02 * np.abs(want).max()


# ---- offsets beyond 32 bits, on rows far apart -----------------------------------------------------------------------------------
def test_rows_far_apart():
    apart, cols = (1 << 31) + 64, 520                         # the third row starts behind 2^32 values
    buf = torch.empty(2 * apart + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, cols), (apart, 1))
    rng = np.random.default_rng(4)
    x64 = rng.standard_normal((3, cols))
    x.copy_(torch.from_numpy(x64))
    near = x.contiguous()
    assert torch.equal(binding.dropout(x, 0.5, 1, 2), binding.dropout(near, 0.5, 1, 2))
    for a, b in zip(binding.residual_norm(x, x), binding.residual_norm(near, near)):
        assert torch.equal(a, b)
    for a, b in zip(binding.residual_norm_grad(x, x, x, x).values(), binding.residual_norm_grad(near, near, near, near).values()):
        assert torch.equal(a, b)
    q, qn = binding.quantize_rows(x), binding.quantize_rows(near)
    assert torch.equal(q.values, qn.values) and torch.equal(q.scale, qn.scale)
    binding.quantized_product(qn, qn, out=x[:, :3])
    assert torch.equal(x[:, :3], binding.quantized_product(qn, qn))
    binding.dropout(near, 0.5, 1, 2, out=x)
    assert torch.equal(x, binding.dropout(near, 0.5, 1, 2))


# ---- in place where rows share 16-byte units --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("cols", [5, 37, 261, 997])
def test_in_place_on_odd_rows(dtype, cols):
    torch.manual_seed(cols)
    x, h, dr, dn = (torch.randn(3001, cols, device="cuda").to(dtype) for _ in range(4))
    r, n = binding.residual_norm(x, h)
    x2, h2 = x.clone(), h.clone()
    binding.residual_norm(x2, h2, residual_out=x2, norm_out=h2)
    assert torch.equal(x2, r) and torch.equal(h2, n)
    g = binding.residual_norm_grad(x, h, dr, dn)
    lib = binding.load_library()
    layer = binding.NormLayer(3001, cols, {torch.float32: 0, torch.float16: 1}[dtype], x.data_ptr(), cols, h.data_ptr(), cols, None, 0, 1, 0, 1, 1, 1e-6)
    ws = torch.empty(lib.cutoff_residual_norm_grad_workspace_bytes(3001, cols), dtype=torch.uint8, device="cuda")
    out = binding.NormGrads(dr.data_ptr(), cols, dn.data_ptr(), cols)                        # over the gradients that came in
    assert lib.cutoff_residual_norm_grad(0, C.byref(layer), dr.data_ptr(), cols, dn.data_ptr(), cols, C.byref(out), ws.data_ptr(), ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(dr, g["x"]) and torch.equal(dn, g["h"])


def test_two_graphs_and_an_eager_call_at_once():
    x = torch.randn(3000, 700, device="cuda")
    gate = torch.randn(30, 700, device="cuda")
    args = dict(gate=gate, gate_rows=100, gate_kind="silu")
    want = binding.residual_norm_grad(x, x, x, x, **args)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = binding.residual_norm_grad(x, x, x, x, **args)
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(5):
        for g, _, s in graphs:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        eager = binding.residual_norm_grad(x, x, x, x, **args)
        torch.cuda.synchronize()
        for out in (graphs[0][1], graphs[1][1], eager):
            assert all(torch.equal(out[k], want[k]) for k in want)


# ---- the very first calls of a process, captured: nothing is set up by them that a capture would not allow ---------------------------
FIRST = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_1803_04209_b200 import binding
x = torch.randn(100, 520, device="cuda", dtype=torch.bfloat16)
w = binding.Quantized(torch.randint(-127, 128, (640, 528), dtype=torch.int8, device="cuda")[:, :520], torch.rand(640, device="cuda"))
v = torch.ones(520, device="cuda")
torch.cuda.synchronize()
def calls():
    y = binding.dropout(x, 0.5, 1, residual=x)
    r, n = binding.residual_norm(x, y, scale=v, post_weight=v, pre_weight=v)
    g = binding.residual_norm_grad(x, y, r, n, scale=v, post_weight=v, pre_weight=v)
    _, q = binding.residual_norm(x, y, quantize=True)
    return [y, r, n, *g.values(), binding.quantized_product(q, w), binding.quantized_product(binding.quantize_rows(x[:1]), w)]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    held = calls()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(held, calls()))
print("captured")
"""


def test_first_calls_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST.format(root=root)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]
