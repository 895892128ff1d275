"""Operators of a transformer layer over bird's-eye-view cells: the calls that a user makes of them, and their plain forms.

The spatial cross-attention of this package (`binding.sca`) is the core of such a layer.  Around it stand

* `linear`: the matrix products that make its value maps, sampling offsets and attention logits, take its output back into
  the cells' rows, and form the feed-forward part; with bias, activation and residual, and the gradients of them;
* `block_norm`: what joins one block of the layer to the next: the norm of the block's output, its gate and residual scale, the
  sum with the rows that passed it by, and the norm before the next block; with the gradients.

Sizes are those of this package's workloads and tests (200 x 200 cells, six cameras, 256 channels in the cross-attention, grids of
181 x 203 and 50 x 50 cells, 80 to 130 channels) or generic powers of two.  A run of `own = False` computes the plain form in
32 bits with elementary operations.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ACTS = ("none", "relu", "gelu", "silu")
_NORMS = ("none", "layer", "rms")
_EPS = 1e-5

#: Rows of the value maps of six cameras: 928 x 1600 images at strides 8 to 64.
_VALUE_ROWS = 6 * (116 * 200 + 58 * 100 + 29 * 50 + 15 * 25)


def _linear(name, **k):
    """rows x K times (N x K) transposed."""
    c = dict(name=name, op="linear", rows=40000, K=256, N=256, dtype="bf16", out="bf16", bias=True, act="none", residual=False, preact=False)
    c.update(k)
    return c


def _linear_backward(name, **k):
    c = dict(name=name, op="linear_backward", rows=40000, K=256, N=256, dtype="bf16", grad="bf16", bias=True, act="none")
    c.update(k)
    return c


def _norm(name, op="block_norm", **k):
    """stream, branch, params: number types of the rows that pass the block by, of the block's output and of the parameters.
    groups: how many gates there are, each for as many rows (0: no gate)."""
    c = dict(name=name, op=op, rows=40000, C=256, stream="bf16", branch="bf16", params="f32", after="none", before="layer", bias=True,
             groups=0, scale=1.0, keep=True)
    c.update(k)
    return c


def listed():
    return [
        # one query: a single token through a wide feed-forward layer, where latency counts
        _linear("linear_single", rows=1, K=1024, N=4096, act="gelu"),
        # the value maps of the cross-attention from the features of all cameras and levels
        _linear("linear_value_maps", rows=_VALUE_ROWS),
        # the way up in the feed-forward part of a training step, which keeps what went into the activation
        _linear("linear_feed_forward", N=1024, act="gelu", preact=True),
        # the cross-attention's float32 output back into float32 rows
        _linear("linear_output_f32", dtype="f32", out="f32", residual=True),
        # a grid and a channel count that nothing divides
        _linear("linear_ragged", rows=181 * 203, K=82, N=130, act="relu", residual=True),
        # a wide layer: bound by arithmetic
        _linear("linear_wide", rows=8192, K=4096, N=4096, act="silu"),
        # gradients of the way up in the feed-forward part
        _linear_backward("linear_backward_feed_forward", N=1024, act="gelu"),
        # gradients of the float32 output projection
        _linear_backward("linear_backward_f32", dtype="f32", grad="f32"),
        # the smallest grid, in single precision: the norm after the sum, as in BEV transformers
        _norm("norm_small", rows=2500, stream="f32", branch="f32", keep=False),
        # norms on both sides of the sum and a gate for each of two frames
        _norm("norm_gated", rows=80000, after="rms", before="rms", bias=False, groups=2, scale=0.5, params="bf16"),
        # gradients of the same
        _norm("norm_backward_gated", "block_norm_backward", rows=80000, after="rms", before="rms", bias=False, groups=2, scale=0.5, params="bf16"),
        # gradients with a float32 stream and rows that are no whole vectors
        _norm("norm_backward_ragged", "block_norm_backward", rows=181 * 203, C=82, stream="f32", groups=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of channels: half of them multiples of 32, the others any."""
    n = _log_int(rng, lo, hi)
    return max(32, n // 32 * 32) if rng.random() < 0.5 else n


def draw(rng):
    """One more call: sizes over the whole range of the listed ones, odd ones among them; not beyond the largest of them."""
    most = {"bytes": 0, "flops": 0}
    for c in listed():
        w = work(c)
        most = {k: max(most[k], w[k]) for k in most}
    while True:
        op = rng.choice(("linear", "linear", "linear_backward", "block_norm", "block_norm_backward"))
        rows = _log_int(rng, 1, _VALUE_ROWS)
        if op.startswith("linear"):
            dtype = rng.choice(("bf16", "bf16", "f32"))
            c = dict(rows=rows, K=_size(rng, 16, 4096), N=_size(rng, 16, 4096), dtype=dtype, bias=rng.random() < 0.75, act=rng.choice(_ACTS))
            if op == "linear":
                c.update(out=rng.choice(("bf16", "bf16", "f32")) if dtype == "bf16" else "f32", residual=rng.random() < 0.5, preact=rng.random() < 0.3)
                c = _linear("", **c)
            else:
                c = _linear_backward("", grad=rng.choice(("bf16", "bf16", "f32")) if dtype == "bf16" else "f32", **c)
        else:
            stream, branch = rng.choice((("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")))
            per = rng.choice((0, 0, 1, rows, 2 if rows % 2 == 0 else 1))
            c = _norm("", op, rows=rows, C=_size(rng, 16, 4096), stream=stream, branch=branch, params=rng.choice(("f32", branch)), groups=per,
                      after=rng.choice(_NORMS), before=rng.choice(_NORMS[1:]), bias=rng.random() < 0.5, scale=rng.choice((1.0, 0.5)),
                      keep=rng.random() < 0.75)
        w = work(c)
        # (single precision costs several times as much as bf16)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] / (8 if c.get("dtype") == "f32" else 1):
            break
    del c["name"]
    return c


def work(case):
    """Bytes: every input read once and every output written once.  Flops: two for each product and sum of the matrix products;
    about ten an element of a norm, twice that for its gradients."""
    size = {"f32": 4, "bf16": 2}
    R = case["rows"]
    if case["op"].startswith("linear"):
        K, N, e = case["K"], case["N"], size[case["dtype"]]
        weights = N * K * e + (N * e if case["bias"] else 0)
        if case["op"] == "linear":
            out = R * N * size[case["out"]]
            return {"bytes": R * K * e + weights + out * (2 if case["residual"] else 1) + (R * N * e if case["preact"] else 0), "flops": 2 * R * K * N}
        pre = R * N * e if case["act"] != "none" else 0
        return {"bytes": R * N * size[case["grad"]] + pre + 2 * (R * K + N * K) * e + (N * e if case["bias"] else 0), "flops": 4 * R * K * N}
    C = case["C"]
    stream, branch, p = R * C * size[case["stream"]], R * C * size[case["branch"]], size[case["params"]]
    vectors = sum((2 if case["bias"] else 1) for k in ("after", "before") if case[k] != "none") * C * p
    gate = case["groups"] * C * p
    if case["op"] == "block_norm":
        return {"bytes": stream * (2 if case["keep"] else 1) + 2 * branch + vectors + gate, "flops": 10 * R * C}
    return {"bytes": stream * (3 if case["keep"] else 2) + 3 * branch + 2 * (vectors + gate), "flops": 20 * R * C}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 11 + 5)

    def normal(*shape, dtype, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).to(_DTYPES[dtype])

    s = {k: v for k, v in case.items() if k != "name"}
    R = case["rows"]
    if case["op"].startswith("linear"):
        K, N, d = case["K"], case["N"], case["dtype"]
        s["x"] = normal(R, K, dtype=d)
        s["weight"] = normal(N, K, dtype=d, scale=K ** -0.5)
        if case["op"] == "linear":
            s["b"] = normal(N, dtype=d, scale=0.5) if case["bias"] else None
            s["r"] = normal(R, N, dtype=case["out"]) if case["residual"] else None
        else:
            s["grad_out"] = normal(R, N, dtype=case["grad"])
            # what the forward call kept: sums of about unit size
            s["z"] = normal(R, N, dtype=d, scale=1.1) if case["act"] != "none" else None
        return s
    C, p = case["C"], case["params"]
    s["x"] = normal(R, C, dtype=case["stream"], scale=2.0, shift=0.1)
    s["y"] = normal(R, C, dtype=case["branch"], shift=-0.05)
    s["g"] = normal(case["groups"], C, dtype=p, scale=0.3, shift=0.5) if case["groups"] else None
    for k in ("after", "before"):
        has = case[k] != "none"
        s[k + "_weight"] = normal(C, dtype=p, scale=0.2, shift=1.0) if has else None
        s[k + "_bias"] = normal(C, dtype=p, scale=0.2) if has and case["bias"] else None
    if case["op"] == "block_norm_backward":
        s["grad_h"] = normal(R, C, dtype=case["stream"]) if case["keep"] else None
        s["grad_n"] = normal(R, C, dtype=case["branch"])
    return s


# ---- the framework's calls -------------------------------------------------------------------------------------------------

def _run_own(s):
    from paper_2607_10071_b200 import binding as fb
    acts = dict(none=fb.ACT_NONE, relu=fb.ACT_RELU, gelu=fb.ACT_GELU, silu=fb.ACT_SILU)
    norms = dict(none=fb.NORM_NONE, layer=fb.NORM_LAYER, rms=fb.NORM_RMS)
    types = dict(f32=fb.F32, bf16=fb.BF16)
    if s["op"] == "linear":
        pre = torch.empty(s["rows"], s["N"], dtype=s["x"].dtype, device=s["x"].device) if s["preact"] else None
        out = fb.linear(s["x"], s["weight"], s["b"], act=acts[s["act"]], residual=s["r"], out_dtype=types[s["out"]], preact=pre)
        return (out, pre) if s["preact"] else (out,)
    if s["op"] == "linear_backward":
        grads = fb.linear_backward(s["grad_out"], s["x"], s["weight"], act=acts[s["act"]], preact=s["z"], grad_bias=s["bias"])
        return tuple(t for t in grads if t is not None)
    kw = dict(gate=s["g"], scale=s["scale"], after=norms[s["after"]], after_weight=s["after_weight"], after_bias=s["after_bias"],
              before=norms[s["before"]], before_weight=s["before_weight"], before_bias=s["before_bias"], eps=_EPS)
    if s["op"] == "block_norm":
        out = fb.block_norm(s["x"], s["y"], keep_h=s["keep"], **kw)
    else:
        out = fb.block_norm_backward(s["grad_h"], s["grad_n"], s["x"], s["y"], **kw)
    return tuple(t for t in out if t is not None)


# ---- the plain form ---------------------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _whiten(t, kind):
    """(t - mean) / deviation of every row, and 1 / deviation."""
    if kind == "layer":
        t = t - t.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((t * t).mean(-1, keepdim=True) + _EPS)
    return t * r, r


def _affine(t, w, b):
    t = t * w
    return t if b is None else t + b


def _whiten_back(g, t, r, kind):
    """Gradient at the input of `_whiten` from that at its result `t`."""
    g = g - t * (g * t).mean(-1, keepdim=True)
    if kind == "layer":
        g = g - g.mean(-1, keepdim=True)
    return g * r


def _gates(s, real):
    """The gate of every row, times the scale."""
    if s["g"] is None:
        return torch.full((1, 1), s["scale"], dtype=real, device=s["x"].device)
    return s["g"].to(real).repeat_interleave(s["rows"] // s["groups"], 0) * s["scale"]


def _run_plain(s):
    f = torch.float32

    def up(t):
        return None if t is None else t.to(f)

    if s["op"] == "linear":
        z = up(s["x"]) @ up(s["weight"]).t()
        if s["b"] is not None:
            z = z + up(s["b"])
        out = _act(z, s["act"])
        if s["r"] is not None:
            out = out + up(s["r"])
        out = out.to(_DTYPES[s["out"]])
        return (out, z.to(s["x"].dtype)) if s["preact"] else (out,)
    if s["op"] == "linear_backward":
        d, g = s["x"].dtype, up(s["grad_out"])
        if s["act"] != "none":
            g = g * _act_slope(up(s["z"]), s["act"])
        grads = ((g @ up(s["weight"])).to(d), (g.t() @ up(s["x"])).to(d))
        return grads + (g.sum(0).to(d),) if s["bias"] else grads
    x, y = up(s["x"]), up(s["y"])
    wa, wb = up(s["after_weight"]), up(s["before_weight"])
    gate = _gates(s, f)
    t, m = y, y
    if s["after"] != "none":
        t, ra = _whiten(y, s["after"])
        m = _affine(t, wa, up(s["after_bias"]))
    h = x + gate * m
    u, rb = _whiten(h, s["before"])
    if s["op"] == "block_norm":
        n = _affine(u, wb, up(s["before_bias"])).to(s["y"].dtype)
        return (h.to(s["x"].dtype), n) if s["keep"] else (n,)
    p = _DTYPES[s["params"]]
    gn = up(s["grad_n"])
    gh = _whiten_back(gn * wb, u, rb, s["before"])
    if s["grad_h"] is not None:
        gh = gh + up(s["grad_h"])
    gm = gh * gate
    out = [gh.to(s["x"].dtype)]
    gy = gm if s["after"] == "none" else _whiten_back(gm * wa, t, ra, s["after"])
    out.append(gy.to(s["y"].dtype))
    if s["groups"]:
        out.append(((gh * m).reshape(s["groups"], -1, s["C"]).sum(1) * s["scale"]).to(p))
    if s["after"] != "none":
        out.append((gm * t).sum(0).to(p))
        if s["bias"]:
            out.append(gm.sum(0).to(p))
    out.append((gn * u).sum(0).to(p))
    if s["bias"]:
        out.append(gn.sum(0).to(p))
    return tuple(out)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    """The values from the definitions, gradients by differentiating them."""
    s = prepare(case, seed)

    def leaf(t):
        return None if t is None else t.double().requires_grad_(case["op"].endswith("backward"))

    if case["op"].startswith("linear"):
        x, w = leaf(s["x"]), leaf(s["weight"])
        if case["op"] == "linear":
            z = torch.einsum("rk,nk->rn", x, w) + (0 if s["b"] is None else s["b"].double())
            out = _definition(z, case["act"]) + (0 if s["r"] is None else s["r"].double())
            return (out, z) if case["preact"] else (out,)
        # the activation's gradient at the kept sums, then those of the product and of the bias
        dz = s["grad_out"].double()
        if case["act"] != "none":
            z = leaf(s["z"])
            dz, = torch.autograd.grad(_definition(z, case["act"]), z, dz)
        bias = torch.zeros(case["N"], dtype=torch.float64, device="cuda", requires_grad=True)
        grads = torch.autograd.grad(torch.einsum("rk,nk->rn", x, w) + bias, (x, w, bias), dz)
        return grads if case["bias"] else grads[:2]

    leaves = [leaf(s[k]) for k in ("x", "y", "g", "after_weight", "after_bias", "before_weight", "before_bias")]
    x, y, gate, wa, ba, wb, bb = leaves

    def normed(v, kind, weight, bias):
        centre = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        power = (v - centre).pow(2).sum(1, keepdim=True) / v.shape[1]
        v = (v - centre) * (power + _EPS).pow(-0.5) * weight
        return v if bias is None else v + bias

    m = y if case["after"] == "none" else normed(y, case["after"], wa, ba)
    if gate is not None:
        m = (m.view(case["groups"], -1, case["C"]) * gate[:, None]).view_as(x)
    h = x + m * case["scale"]
    n = normed(h, case["before"], wb, bb)
    if case["op"] == "block_norm":
        return (h, n) if case["keep"] else (n,)
    ends = [(n, s["grad_n"].double())] + ([(h, s["grad_h"].double())] if case["keep"] else [])
    return torch.autograd.grad([a for a, _ in ends], [t for t in leaves if t is not None], [b for _, b in ends])


def _definition(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z
