"""The layer operators as timed and compared cases: dropout, norms with gate and residual, products in 8-bit integers.

    listed()             named cases
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  what a program holds before the call: inputs, weights (8-bit ones are quantised once), buffers
    run(state)           one pass: the framework's calls where `own` is true, else the plain form in elementary operations
    work(case)           bytes and operations one pass cannot do without
    exact(case, seed)    the same outputs from the definition in 64 bits

Four kinds of pass:
    dropout   y = [residual +] keep * x / (1 - p), the mask a function of (seed, step, stream, row, column) alone; the
              gradient with respect to x is the same pass over the gradient of y.
    norm      r = x + scale * gate * post(h), n = pre(r): the end of one residual block and the start of the next.
    grad      the gradients of `norm` with respect to all of its inputs, from those with respect to r and n.
    product   y = x w^T in 8-bit integers, x quantised row by row on the way (after `norm`, if the case has one).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                   # set from outside: whether run() calls the framework's operators

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
NOISE_STREAM = 0x400


def _dropout(name, rows, cols, type, p, residual, pad=0):
    return {"name": name, "kind": "dropout", "rows": rows, "cols": cols, "type": type, "p": p, "residual": residual, "pad": pad}


def _norm(name, kind, rows, cols, type, post="rms", pre="rms", gate="none", gate_rows=1, gate_kind="linear", bias=False, scale=True, pad=0):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "type": type, "post": post, "pre": pre, "gate": gate,
            "gate_rows": gate_rows, "gate_kind": gate_kind, "bias": bias, "scale": scale, "pad": pad}


def _product(name, rows, outputs, cols, type, bias=False, norm=False, pad=0):
    return {"name": name, "kind": "product", "rows": rows, "outputs": outputs, "cols": cols, "type": type, "bias": bias, "norm": norm, "pad": pad}


def listed():
    return [
        # training: the branch of a residual block, dropped out and added to the residual stream
        _dropout("dropout add 16384x4096 bf16", 16384, 4096, "bf16", 0.1, True),
        # the gradient through the dropout of a hidden layer as wide as the paper's larger cluster, rows of an odd length
        _dropout("dropout 8001x2175 fp32", 8001, 2175, "fp32", 0.3, False),
        # serving, one token: latency is all there is
        _norm("norm 1x4096 bf16", "norm", 1, 4096, "bf16"),
        # a long prompt or a training batch on its way forward, one gate value per feature and token
        _norm("norm 16384x4096 bf16 gate", "norm", 16384, 4096, "bf16", gate="rows", gate_kind="sigmoid"),
        # layer norms in fp32 over an odd width, one gate per sequence
        _norm("norm 5000x2175 fp32 layer", "norm", 5000, 2175, "fp32", post="layer", pre="layer", gate="groups", gate_rows=125, bias=True),
        # the same blocks on the way back
        _norm("grad 16384x4096 bf16 gate", "grad", 16384, 4096, "bf16", gate="rows", gate_kind="sigmoid"),
        _norm("grad 4001x1025 fp32 layer", "grad", 4001, 1025, "fp32", post="layer", pre="layer", gate="groups", gate_rows=200, bias=True),
        _norm("grad 100000x512 fp16", "grad", 100000, 512, "fp16", gate="groups", gate_rows=1000, gate_kind="silu"),
        # serving, one token: the weights are read once, in a quarter of their bytes
        _product("product 1x4096x4096 bf16", 1, 4096, 4096, "bf16"),
        # serving, a batch of sequences, the norm before the block quantises for its product
        _product("norm, product 48x8192x8192", 48, 8192, 8192, "bf16", norm=True),
        # an output layer of odd sizes
        _product("product 2175x1001x513 fp32", 2175, 1001, 513, "fp32", bias=True),
        # a long prompt through a wide layer
        _product("product 8192x8192x8192 bf16", 8192, 8192, 8192, "bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm", "grad", "grad", "product", "product"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    pad = rng.choice([0, 0, 0, 1, 8, 64])
    if kind == "product":
        rows = _log_uniform(rng, 1, 8192)
        even = rng.random() < 0.5                       # widths as networks have them, or any
        outputs, cols = (_log_uniform(rng, 1, 64) * 128 if even else _log_uniform(rng, 16, 8192) for _ in range(2))
        norm = type != "fp32" and rng.random() < 0.4    # what a norm leaves next to a border between two integers is decided by its last bit
        return _drawn(_product("", rows, outputs, cols, type, bias=rng.random() < 0.5, norm=norm, pad=pad))
    even = rng.random() < 0.6
    cols = _log_uniform(rng, 1, 64) * 128 if even else _log_uniform(rng, 16, 8192)
    rows = _log_uniform(rng, 1, min(200000, ((1 << 26) if type != "fp32" else (1 << 25)) // cols))
    if kind == "dropout":
        return _drawn(_dropout("", rows, cols, type, rng.choice([0.0, 0.05, 0.1, 0.2, 0.5, round(rng.random(), 3)]), rng.random() < 0.5, pad))
    gate = rng.choice(["none", "rows", "groups"])
    return _drawn(_norm("", kind, rows, cols, type, post=rng.choice(["rms", "layer", "none"]), pre=rng.choice(["rms", "layer"]), gate=gate,
                        gate_rows=_log_uniform(rng, 1, rows) if gate == "groups" else 1, gate_kind=rng.choice(["linear", "sigmoid", "silu"]),
                        bias=rng.random() < 0.4, scale=rng.random() < 0.7, pad=pad))


def _drawn(case):
    del case["name"]
    return case


# ---- inputs --------------------------------------------------------------------------------------------------------
class _Inputs:
    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, std=1.0, mean=0.0):
        return torch.randn(*shape, device="cuda", generator=self.gen) * std + mean

    def rows(self, rows, cols, type, pad, std=1.0):
        """[rows, cols] of `type`, rows `pad` values further apart than they are long."""
        buf = torch.empty(rows, cols + pad, device="cuda", dtype=TYPES[type])
        buf.normal_(std=std, generator=self.gen)
        return buf[:, :cols]


def _residual_stream(make, case):
    """Activations as a deep network's residual stream has them: a few features are many times larger than the others."""
    x = make.rows(case["rows"], case["cols"], case["type"], case["pad"])
    x[:, 5::97] *= 8
    return x


def _norm_state(make, case):
    rows, cols, type = case["rows"], case["cols"], case["type"]
    s = {"x": _residual_stream(make, case), "h": make.rows(rows, cols, type, case["pad"], std=2.0), "gate": None, "scale": None,
         "post_weight": None, "post_bias": None, "pre_weight": make.normal(cols, std=0.1, mean=1.0), "pre_bias": None}
    if case["gate"] == "rows":
        s["gate"] = make.rows(rows, cols, type, case["pad"])
    elif case["gate"] == "groups":
        s["gate"] = make.rows(-(-rows // case["gate_rows"]), cols, type, 0)
    if case["scale"]:
        s["scale"] = make.normal(cols, std=0.05, mean=0.3)
    if case["post"] != "none":
        s["post_weight"] = make.normal(cols, std=0.1, mean=1.0)
        if case["bias"]:
            s["post_bias"] = make.normal(cols, std=0.1)
    if case["bias"]:
        s["pre_bias"] = make.normal(cols, std=0.1)
    return s


def prepare(case, seed):
    make = _Inputs(seed)
    s = {"case": case}
    if case["kind"] == "dropout":
        s["x"] = make.rows(case["rows"], case["cols"], case["type"], case["pad"], std=2.0)
        s["residual"] = _residual_stream(make, case) if case["residual"] else None
        s["seed"], s["step"] = (seed * 0x9E3779B97F4A7C15 + 1) % (1 << 64), seed % 1000
    elif case["kind"] in ("norm", "grad"):
        s.update(_norm_state(make, case))
        if case["kind"] == "grad":
            s["d_residual"] = make.rows(case["rows"], case["cols"], case["type"], case["pad"], std=0.1)
            s["d_norm"] = make.rows(case["rows"], case["cols"], case["type"], case["pad"], std=0.1)
    else:
        if case["norm"]:
            s.update(_norm_state(make, _norm("", "norm", case["rows"], case["cols"], case["type"], pad=case["pad"])))
        else:
            s["x"] = _residual_stream(make, case)
        # the weights, quantised once: 8-bit rows on 16-byte boundaries and a scale per output
        w = make.normal(case["outputs"], case["cols"], std=case["cols"] ** -0.5)
        w *= 1.0 + make.normal(case["outputs"], 1, std=0.2).abs()
        w_scale = w.abs().amax(1) / 127.0
        buf = torch.zeros(case["outputs"], (case["cols"] + 15) // 16 * 16, device="cuda", dtype=torch.int8)
        buf[:, : case["cols"]] = torch.round(w / w_scale[:, None]).clamp(-127, 127).to(torch.int8)
        s["w"], s["w_scale"] = buf[:, : case["cols"]], w_scale
        s["bias"] = make.normal(case["outputs"], std=0.1) if case["bias"] else None
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["kind"] == "dropout":
        if own:
            from paper_1803_04209_b200 import binding
            return binding.dropout(s["x"], case["p"], s["seed"], s["step"], noise_stream=NOISE_STREAM, residual=s["residual"])
        return _plain_dropout(s)
    if case["kind"] == "norm":
        if own:
            from paper_1803_04209_b200 import binding
            r, n = binding.residual_norm(s["x"], s["h"], **_norm_options(s, case))
            return {"residual": r, "norm": n}
        r, n = _plain_norm(s, case)
        return {"residual": r.to(s["x"].dtype), "norm": n.to(s["x"].dtype)}
    if case["kind"] == "grad":
        if own:
            from paper_1803_04209_b200 import binding
            return binding.residual_norm_grad(s["x"], s["h"], s["d_residual"], s["d_norm"], **_norm_options(s, case))
        return _plain_grad(s)
    if own:
        from paper_1803_04209_b200 import binding
        if case["norm"]:
            r, a = binding.residual_norm(s["x"], s["h"], quantize=True, **_norm_options(s, _norm("", "norm", 0, 0, case["type"])))
            return {"residual": r, "y": binding.quantized_product(a, (s["w"], s["w_scale"]), s["bias"], dtype=r.dtype)}
        a = binding.quantize_rows(s["x"])
        return {"y": binding.quantized_product(a, (s["w"], s["w_scale"]), s["bias"], dtype=s["x"].dtype)}
    return _plain_product(s)


def _norm_options(s, case):
    return {"gate": s["gate"], "gate_rows": case["gate_rows"], "gate_kind": case["gate_kind"], "scale": s["scale"],
            "post": None if case["post"] == "none" else case["post"], "post_weight": s["post_weight"], "post_bias": s["post_bias"],
            "pre": case["pre"], "pre_weight": s["pre_weight"], "pre_bias": s["pre_bias"], "eps": EPS}


# ---- the plain form ------------------------------------------------------------------------------------------------
def _plain_round(c, k):
    """One round of Philox4x32 on 32-bit words held in 64-bit integers."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
    return ((b >> 32 & 0xFFFFFFFF) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32 & 0xFFFFFFFF) ^ c[3] ^ k[1], a & 0xFFFFFFFF)


def _plain_keep(rows, cols, p, seed, step):
    """Where an element stays: 16 bits for each of the eight columns that a counter (column / 8, row, stream, step) serves."""
    q = torch.arange((cols + 7) // 8, device="cuda")[None, :].expand(rows, -1)
    i = torch.arange(rows, device="cuda")[:, None].expand_as(q)
    c = (q, i, torch.full_like(q, NOISE_STREAM), torch.full_like(q, step))
    for r in range(10):
        c = _plain_round(c, ((seed + r * 0x9E3779B9) & 0xFFFFFFFF, ((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF))
    words = torch.stack(c, -1)
    bits = torch.stack((words & 0xFFFF, words >> 16), -1).reshape(rows, -1)[:, :cols]
    return bits >= round(p * 65536)


def _plain_dropout(s):
    case, x = s["case"], s["x"]
    dropped = round(case["p"] * 65536)
    keep = _plain_keep(case["rows"], case["cols"], case["p"], s["seed"], s["step"])
    y = torch.where(keep, x.float() * (65536.0 / max(1, 65536 - dropped)), 0.0)
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return y.to(x.dtype)


def _plain_normalised(v, kind):
    """The rows of v normalised, and the factor that did it."""
    if kind == "none":
        return v, None
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    inv = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * inv, inv


def _plain_gate(s, case):
    """The gate's value for each row, and its derivative."""
    if s["gate"] is None:
        return 1.0, None
    g = s["gate"].float()
    if case["gate_kind"] == "linear":
        a, d = g, torch.ones_like(g)
    else:
        sig = torch.sigmoid(g)
        a, d = (sig, sig * (1 - sig)) if case["gate_kind"] == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))
    if case["gate"] == "groups":
        group = torch.arange(s["x"].shape[0], device="cuda") // case["gate_rows"]
        a, d = a[group], d[group]
    return a, d


def _or(v, other):
    return other if v is None else v


def _plain_norm(s, case):
    hat, _ = _plain_normalised(s["h"].float(), case["post"])
    p = hat * _or(s["post_weight"], 1.0) + _or(s["post_bias"], 0.0)
    r = s["x"].float() + _or(s["scale"], 1.0) * _plain_gate(s, case)[0] * p
    return r, _plain_normalised(r, case["pre"])[0] * s["pre_weight"] + _or(s["pre_bias"], 0.0)


def _plain_back(d, hat, inv, kind):
    if kind == "none":
        return d
    if kind == "layer":
        d = d - d.mean(1, keepdim=True)
    return inv * (d - hat * (d * hat).mean(1, keepdim=True))


def _plain_grad(s):
    case, type = s["case"], s["x"].dtype
    hat, inv = _plain_normalised(s["h"].float(), case["post"])
    weight, scale = _or(s["post_weight"], 1.0), _or(s["scale"], 1.0)
    p = hat * weight + _or(s["post_bias"], 0.0)
    a, slope = _plain_gate(s, case)
    r_hat, r_inv = _plain_normalised(s["x"].float() + scale * a * p, case["pre"])
    d_norm = s["d_norm"].float()
    d_r = s["d_residual"].float() + _plain_back(d_norm * s["pre_weight"], r_hat, r_inv, case["pre"])
    e = d_r * a
    out = {"x": d_r.to(type), "h": _plain_back(e * scale * weight, hat, inv, case["post"]).to(type), "pre_weight": (d_norm * r_hat).sum(0)}
    if s["pre_bias"] is not None:
        out["pre_bias"] = d_norm.sum(0)
    if s["scale"] is not None:
        out["scale"] = (e * p).sum(0)
    if s["post_weight"] is not None:
        out["post_weight"] = (e * scale * hat).sum(0)
    if s["post_bias"] is not None:
        out["post_bias"] = (e * scale).sum(0)
    if s["gate"] is not None:
        d_gate = d_r * scale * p * slope
        if case["gate"] == "groups":
            rows, cols, each = case["rows"], case["cols"], case["gate_rows"]
            whole = rows // each * each
            parts = [d_gate[:whole].reshape(-1, each, cols).sum(1)]
            if whole < rows:
                parts.append(d_gate[whole:].sum(0, keepdim=True))
            d_gate = torch.cat(parts)
        out["gate"] = d_gate.to(type)
    return out


def _plain_quantised(x):
    """8-bit integers (as fp32) and the scale of each row."""
    top = x.abs().amax(1, keepdim=True)
    inv = torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)          # a division, not a reciprocal's product
    return torch.round(x * inv).clamp(-127, 127), top / 127.0


def _plain_product(s):
    case, type = s["case"], s["x"].dtype
    out = {}
    if case["norm"]:
        r, x = _plain_norm(s, _norm("", "norm", 0, 0, case["type"]))
        out["residual"] = r.to(type)
    else:
        x = s["x"].float()
    q, scale = _plain_quantised(x)
    y = q @ s["w"].float().t() * scale * s["w_scale"]
    out["y"] = (y + _or(s["bias"], 0.0)).to(type)
    return out


# ---- the definition in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        return _exact_dropout(s, case)
    if case["kind"] == "product":
        return _exact_product(s, case)
    names = ("x", "h", "gate", "scale", "post_weight", "post_bias", "pre_weight", "pre_bias")
    v = {k: None if s[k] is None else s[k].double().requires_grad_(case["kind"] == "grad") for k in names}
    r, n = _exact_norm(v, case)
    if case["kind"] == "norm":
        return {"residual": r, "norm": n}
    (r * s["d_residual"].double()).sum().add((n * s["d_norm"].double()).sum()).backward()
    return {k: v[k].grad for k in names if v[k] is not None}


def _exact_norm(v, case):
    def norm(t, kind, weight, bias):
        if kind != "none":
            centre = t.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(t[:, :1])
            t = (t - centre) / torch.sqrt(torch.mean((t - centre) ** 2, dim=1, keepdim=True) + EPS)
        t = t if weight is None else t * weight
        return t if bias is None else t + bias

    branch = norm(v["h"], case["post"], v["post_weight"], v["post_bias"])
    if v["gate"] is not None:
        g = {"linear": lambda t: t, "sigmoid": lambda t: 1 / (1 + torch.exp(-t)), "silu": lambda t: t / (1 + torch.exp(-t))}[case["gate_kind"]](v["gate"])
        if case["gate"] == "groups":
            g = g.repeat_interleave(case["gate_rows"], dim=0)[: len(branch)]
        branch = branch * g
    r = v["x"] + (branch if v["scale"] is None else branch * v["scale"])
    return r, norm(r, case["pre"], v["pre_weight"], v["pre_bias"])


def _exact_dropout(s, case):
    rows, cols, seed = case["rows"], case["cols"], s["seed"]
    low = np.uint64(0xFFFFFFFF)
    groups = (cols + 7) // 8
    c0 = np.tile(np.arange(groups, dtype=np.uint64), rows)
    c1 = np.repeat(np.arange(rows, dtype=np.uint64), groups)
    c2, c3 = np.full_like(c0, NOISE_STREAM), np.full_like(c0, s["step"])
    k0, k1 = seed % 2 ** 32, seed // 2 ** 32
    for _ in range(10):
        left, right = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (right >> np.uint64(32)) ^ c1 ^ np.uint64(k0), right & low, (left >> np.uint64(32)) ^ c3 ^ np.uint64(k1), left & low
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    halves = np.stack([c0, c1, c2, c3], 1).astype("<u4").view("<u2").reshape(rows, groups * 8)[:, :cols]
    border = int(round(case["p"] * 65536))
    keep = torch.from_numpy(halves >= border).cuda()
    y = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    y[keep] = s["x"].double()[keep] * (65536 / (65536 - border))
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_product(s, case):
    out = {}
    if case["norm"]:
        v = {k: None if s[k] is None else s[k].double() for k in ("x", "h", "gate", "scale", "post_weight", "post_bias", "pre_weight", "pre_bias")}
        r, x = _exact_norm(v, _norm("", "norm", 0, 0, case["type"]))
        out["residual"], x = r, x.float()
    else:
        x = s["x"].float()
    # the 8-bit values are part of the definition, with the single-precision steps that lead to them
    top = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)
    inverse = torch.full_like(top, 127.0) / top
    inverse[top == 0] = 0
    q = torch.round((x.double() * inverse.double()[:, None]).float()).double()
    y = torch.einsum("ik,jk->ij", q, s["w"].double()) * (top / 127.0).double()[:, None] * s["w_scale"].double()[None, :]
    out["y"] = y if s["bias"] is None else y + s["bias"].double()
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    size = 4 if case["type"] == "fp32" else 2
    if case["kind"] == "product":
        m, n, k = case["rows"], case["outputs"], case["cols"]
        bytes = size * m * k + n * k + 4 * n * (2 if case["bias"] else 1) + size * m * n
        flops = 2 * m * n * k + 4 * m * k + 3 * m * n
        if case["norm"]:                                  # the block's output in, the residual stream out
            bytes += 2 * size * m * k + 12 * k
            flops += 14 * m * k
        return {"bytes": bytes, "flops": flops}
    each = case["rows"] * case["cols"]
    if case["kind"] == "dropout":                         # ten rounds of eight operations serve eight elements
        return {"bytes": size * each * (3 if case["residual"] else 2), "flops": 13 * each}
    vectors = 1 + (case["post"] != "none") + case["scale"] + case["bias"] * (1 + (case["post"] != "none"))
    tensors = 4 if case["kind"] == "norm" else 6          # x, h in, r, n out; x, h, d_r, d_n in, d_x, d_h out
    gates = {"none": 0, "rows": each, "groups": -(-case["rows"] // case["gate_rows"]) * case["cols"]}[case["gate"]]
    if case["kind"] == "grad":
        vectors, gates = 2 * vectors, 2 * gates
    return {"bytes": size * (tensors * each + gates) + 4 * vectors * case["cols"], "flops": (14 if case["kind"] == "norm" else 40) * each}
