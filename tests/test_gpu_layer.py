"""The operators of a transformer layer together, as they are used: values and gradients of a whole layer around the spatial cross-attention."""
import pytest

from paper_2607_10071_b200 import binding as fb
from paper_2607_10071_b200 import workloads as wl

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
HEADS, DIM, LEVELS, POINTS = 4, 16, 2, 4
C = HEADS * DIM


def relative(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm()).item()


@pytest.fixture(scope="module")
def scene():
    import numpy as np
    grid, img, levels = (30, 34, 4), (128, 352), ((16, 44), (8, 22))
    rig = wl.ring_rig(6, 70.0, img, np.zeros((1, 6)))
    gen = torch.Generator(device="cuda").manual_seed(11)

    def draw(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=gen, device="cuda") * scale + shift

    T = sum(h * w for h, w in levels)
    s = dict(grid=grid, img=img, levels=levels, rig=torch.from_numpy(rig).cuda(), range=(-25.0, 25.0, -25.0, 25.0, -3.0, 1.0),
             query=draw(1, grid[0] * grid[1], C), tokens=draw(1, 6, T, C), gate=draw(C, scale=0.2, shift=1.0))
    for name, rows, cols in (("value", C, C), ("offset", HEADS * LEVELS * POINTS * 2, C), ("logit", HEADS * LEVELS * POINTS, C), ("output", C, C),
                             ("up", 4 * C, C), ("down", C, 4 * C)):
        s[name + "_w"], s[name + "_b"] = draw(rows, cols, scale=cols ** -0.5), draw(rows, scale=0.2)
    for i in range(3):
        s[f"norm{i}_w"], s[f"norm{i}_b"] = draw(C, scale=0.1, shift=1.0), draw(C, scale=0.1)
    return s


def layer(s, dtype):
    """norm -> cross-attention (values, offsets, logits, output) -> sum and norm -> feed-forward -> gated sum and norm"""
    p = {k: (v.to(dtype) if torch.is_tensor(v) and k.endswith(("_w", "_b")) and not k.startswith("norm") else v) for k, v in s.items()}
    query, tokens = s["query"].to(dtype), s["tokens"].to(dtype)
    _, n = fb.block_norm(query, before_weight=s["norm0_w"], before_bias=s["norm0_b"])
    value = fb.linear(tokens, p["value_w"], p["value_b"]).reshape(1, 6, -1, HEADS, DIM)
    off = fb.linear(n, p["offset_w"], p["offset_b"], out_dtype=fb.F32)
    logit = fb.linear(n, p["logit_w"], p["logit_b"], out_dtype=fb.F32)
    Q = n.shape[1]
    weight = torch.softmax(logit.reshape(1, Q, HEADS, LEVELS * POINTS), -1).reshape(1, Q, HEADS, LEVELS, POINTS)
    off = off.reshape(1, Q, HEADS, LEVELS, POINTS, 2)
    seen = fb.sca(value, s["levels"], s["rig"], off, weight, s["img"], s["range"], s["grid"])
    out = fb.linear(seen.to(dtype), p["output_w"], p["output_b"])
    h, n = fb.block_norm(query, out, before_weight=s["norm1_w"], before_bias=s["norm1_b"])
    up = fb.linear(n, p["up_w"], p["up_b"], act=fb.ACT_GELU)
    down = fb.linear(up, p["down_w"], p["down_b"])
    return (seen, ) + fb.block_norm(h, down, gate=s["gate"], before=fb.NORM_RMS, before_weight=s["norm2_w"])


def plain_layer(s):
    d = {k: (v.double() if torch.is_tensor(v) else v) for k, v in s.items()}
    norm = lambda v, i, kind=fb.NORM_LAYER: ref.whiten(v, kind, 1e-5) * d[f"norm{i}_w"] + (d[f"norm{i}_b"] if kind == fb.NORM_LAYER else 0)  # noqa: E731
    lin = lambda v, k: v @ d[k + "_w"].T + d[k + "_b"]  # noqa: E731
    n = norm(d["query"], 0)
    Q = n.shape[1]
    value = lin(d["tokens"], "value").reshape(1, 6, -1, HEADS, DIM)
    weight = torch.softmax(lin(n, "logit").reshape(1, Q, HEADS, LEVELS * POINTS), -1).reshape(1, Q, HEADS, LEVELS, POINTS)
    off = lin(n, "offset").reshape(1, Q, HEADS, LEVELS, POINTS, 2)
    # (the cross-attention itself has tests of its own: here on the exact inputs, rounded once)
    seen = fb.sca(value.float(), s["levels"], s["rig"], off.float().contiguous(), weight.float().contiguous(), s["img"], s["range"], s["grid"])
    h = d["query"] + lin(seen.double(), "output")
    f = lin(ref.activation(lin(norm(h, 1), "up"), fb.ACT_GELU), "down")
    h = h + d["gate"] * f
    return seen, h, norm(h, 2, fb.NORM_RMS)


def test_layer(scene):
    want = plain_layer(scene)
    # float32: a dozen products and norms of 1e-7 each, and positions in the maps that move by as much of up to 44 texels
    got = layer(scene, F32)
    assert float(want[0].abs().sum()) > 0
    for a, b in zip(got, want):
        assert relative(a.reshape(b.shape), b) < 2e-5
    # bf16: every rounding is 2^-9 on the average and a dozen of them add up; the positions move by hundredths of a texel
    for a, b in zip(layer(scene, BF16)[1:], want[1:]):
        assert relative(a.reshape(b.shape), b) < 3e-2


@pytest.mark.parametrize("dtype,most", [(F32, 1e-5), (BF16, 3e-2)])
def test_gradients_of_the_feed_forward_block(scene, dtype, most):
    """h = x + gate * down(gelu(up(norm(x)))), n = norm(h), back from gradients at h and n to everything."""
    s = scene
    x = s["query"].to(dtype)[0]
    w = {k: s[k].to(dtype) for k in ("up_w", "up_b", "down_w", "down_b")}
    gen = torch.Generator(device="cuda").manual_seed(4)
    gh, gn = (torch.randn(x.shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    first = dict(before_weight=s["norm0_w"], before_bias=s["norm0_b"])
    second = dict(gate=s["gate"], scale=0.5, before_weight=s["norm1_w"], before_bias=s["norm1_b"])
    _, n0 = fb.block_norm(x, **first)
    z = torch.empty(x.shape[0], 4 * C, dtype=dtype, device="cuda")
    up = fb.linear(n0, w["up_w"], w["up_b"], act=fb.ACT_GELU, preact=z)
    y = fb.linear(up, w["down_w"], w["down_b"])
    h, n = fb.block_norm(x, y, **second)
    g_x, g_y, g_gate, _, _, g_w1, g_b1 = fb.block_norm_backward(gh, gn, x, y, **second)
    g_up, g_down_w, g_down_b = fb.linear_backward(g_y, up, w["down_w"])
    g_n0, g_up_w, g_up_b = fb.linear_backward(g_up, n0, w["up_w"], act=fb.ACT_GELU, preact=z)
    g_in, _, _, _, _, g_w0, g_b0 = fb.block_norm_backward(None, g_n0, x, **first)
    got = dict(x=g_x.double() + g_in.double(), gate=g_gate, norm1_w=g_w1, norm1_b=g_b1, down_w=g_down_w, down_b=g_down_b, up_w=g_up_w, up_b=g_up_b,
               norm0_w=g_w0, norm0_b=g_b0)
    leaf = {k: v.double().requires_grad_(True) for k, v in dict(x=x, gate=s["gate"], norm0_w=s["norm0_w"], norm0_b=s["norm0_b"], norm1_w=s["norm1_w"],
                                                                norm1_b=s["norm1_b"], **w).items()}
    m = ref.whiten(leaf["x"], fb.NORM_LAYER, 1e-5) * leaf["norm0_w"] + leaf["norm0_b"]
    f = ref.activation(m @ leaf["up_w"].T + leaf["up_b"], fb.ACT_GELU) @ leaf["down_w"].T + leaf["down_b"]
    hh = leaf["x"] + 0.5 * leaf["gate"] * f
    nn = ref.whiten(hh, fb.NORM_LAYER, 1e-5) * leaf["norm1_w"] + leaf["norm1_b"]
    want = torch.autograd.grad((hh * gh.double()).sum() + (nn * gn.double()).sum(), list(leaf.values()))
    assert relative(h, hh) < most and relative(n, nn) < most
    for k, t in zip(leaf, want):
        assert relative(got[k], t) < most, k


def test_layer_beside_the_view_transformation(scene):
    """A grid of the sampling operator through a 1 x 1 convolution with ReLU, channels last, bf16 cells."""
    w = wl.get("tiny")
    inp = wl.make_inputs(w)
    X, Y, Z = w.grid
    bev = fb.sampling_vt(torch.from_numpy(inp.features).cuda(), torch.from_numpy(inp.lidar2img).cuda(), w.img_hw, w.bev_range, w.grid)
    gen = torch.Generator(device="cuda").manual_seed(2)
    kernel = torch.randn(48, w.C, generator=gen, device="cuda")
    out = fb.linear(bev, kernel, act=fb.ACT_RELU, out_dtype=fb.BF16)
    assert out.shape == (1, X, Y, 48) and out.dtype == BF16
    want, _, off, _ = ref.linear(bev.reshape(-1, w.C), kernel, None, fb.ACT_RELU)
    ref.check(out.reshape(-1, 48), want, off)
