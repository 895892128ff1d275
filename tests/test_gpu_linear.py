"""Matrix products with their epilogue, and their gradients, against plain 64-bit forms."""
import ctypes

import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
ACTS = (fb.ACT_NONE, fb.ACT_RELU, fb.ACT_GELU, fb.ACT_SILU)


def draw(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def inputs(rows, K, N, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 131 * rows + 17 * K + N)
    return gen, draw(gen, rows, K, dtype=dtype), draw(gen, N, K, dtype=dtype, scale=K ** -0.5), draw(gen, N, dtype=dtype)


SHAPES = [(1, 1, 1), (1, 256, 96), (2, 7, 3), (5, 83, 130), (8, 512, 33), (9, 64, 64), (9, 65, 1), (17, 1, 257), (127, 63, 31), (128, 64, 128),
          (129, 128, 129), (300, 82, 130), (257, 264, 520), (64, 1024, 96), (33, 4096, 40), (1000, 385, 200), (20000, 32, 16), (4000, 256, 1024)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    rows, K, N = shape
    gen, x, w, b = inputs(rows, K, N, dtype)
    for i, act in enumerate(ACTS):
        out_type = (BF16, F32)[(i + rows) % 2]
        res = draw(gen, rows, N, dtype=out_type) if i % 2 else None
        pre = torch.full((rows, N), float("nan"), dtype=dtype, device="cuda") if i > 1 else None
        bias = b if i != 1 else None
        out = fb.linear(x, w, bias, act=act, residual=res, out_dtype=fb.F32 if out_type is F32 else fb.BF16, preact=pre)
        want, z, off, off_z = ref.linear(x, w, bias, act, res)
        low = 6e-6 if out_type is BF16 and act == fb.ACT_GELU else 0.0       # the formula of results that are rounded to bf16
        ref.check(out, want, off + low, (shape, act))
        if pre is not None:
            ref.check(pre, z, off_z, (shape, act, "z"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype):
    rows, K, N = shape
    gen, x, w, b = inputs(rows, K, N, dtype, 5)
    for i, act in enumerate(ACTS):
        g = draw(gen, rows, N, dtype=F32 if (i + rows) % 2 else dtype)
        z = draw(gen, rows, N, dtype=dtype) if act else None
        grads = fb.linear_backward(g, x, w, act=act, preact=z)
        want, bounds = ref.linear_backward(g, x, w, act, z)
        for got, a, off, what in zip(grads, want, bounds, ("x", "weight", "bias")):
            assert got.dtype == dtype
            ref.check(got, a, off, (shape, act, what))


def test_only_the_gradients_that_are_wanted():
    gen, x, w, b = inputs(200, 96, 72, BF16)
    g, z = draw(gen, 200, 72, dtype=BF16), draw(gen, 200, 72, dtype=BF16)
    full = fb.linear_backward(g, x, w, act=fb.ACT_SILU, preact=z)
    for wanted in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 0, 0)):
        part = fb.linear_backward(g, x, w, act=fb.ACT_SILU, preact=z, grad_x=wanted[0], grad_weight=wanted[1], grad_bias=wanted[2])
        for a, b_, want in zip(part, full, wanted):
            assert (a is not None) == bool(want) and (a is None or torch.equal(a, b_))


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """Directional derivatives of the float32 calls: steps of 2^-6 of unit directions make errors of the second order below 2^-12 of third derivatives
    of about 1, and differences of sums of 1e4 numbers of 1 that float32 rounds to 6e-8 each, over 2^-5: about 2e-4; both below 2e-3 of
    derivatives of about 100."""
    gen, x, w, b = inputs(160, 48, 56, F32)
    g = draw(gen, 160, 56, dtype=F32)
    z = torch.empty(160, 56, device="cuda")
    fb.linear(x, w, b, act=act, preact=z)
    if act == fb.ACT_RELU:       # no kink within a step
        b = b + 0.5
        z = torch.empty_like(z)
        fb.linear(x, w, b, act=act, preact=z)
    grads = fb.linear_backward(g, x, w, act=act, preact=z if act else None)
    h = 2.0 ** -6 if act != fb.ACT_RELU else 2.0 ** -14
    for i, (p, grad) in enumerate(zip((x, w, b), grads)):
        v = grad / grad.norm()
        ends = []
        for s in (h, -h):
            args = [x, w, b]
            args[i] = p + s * v
            ends.append((fb.linear(args[0], args[1], args[2], act=act).double() * g.double()).sum())
        slope = ((ends[0] - ends[1]) / (2 * h)).item()
        want = (grad.double() * v.double()).sum().item()
        assert abs(slope - want) <= (2e-3 if act != fb.ACT_RELU else 2e-2) * want, (i, slope, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_alignment_and_what_lies_around(dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    for off, pad, K, N in ((0, 8, 64, 48), (1, 3, 40, 24), (2, 6, 82, 130), (1, 1, 33, 65), (4, 4, 64, 128)):
        wide_x = draw(gen, 70, 4, K + pad, dtype=dtype)
        x = wide_x[:, :, off:off + K]
        w = draw(gen, N, K + pad, dtype=dtype, scale=K ** -0.5)[:, off:off + K]
        wide_r = draw(gen, 280, N + pad, dtype=dtype)
        frame = torch.full((281, N + pad), 7.0, dtype=dtype, device="cuda")
        pre = torch.full((281, N + pad), 7.0, dtype=dtype, device="cuda")
        out = frame[:280, off:off + N]
        got = fb.linear(x, w, act=fb.ACT_RELU, residual=wide_r[:, off:off + N], out=out, preact=pre[:280, off:off + N])
        assert got.data_ptr() == out.data_ptr()
        want, z, bound, bound_z = ref.linear(x.reshape(280, K), w, None, fb.ACT_RELU, wide_r[:, off:off + N])
        ref.check(out, want, bound, (off, pad, K, N))
        ref.check(pre[:280, off:off + N], z, bound_z)
        for f in (frame, pre):
            assert bool((f[280] == 7).all()) and bool((f[:, :off] == 7).all()) and bool((f[:, off + N:] == 7).all())
        g = draw(gen, 280, N + pad, dtype=dtype)[:, off:off + N]
        grads = fb.linear_backward(g, x, w, act=fb.ACT_RELU, preact=pre[:280, off:off + N])
        wants, bounds = ref.linear_backward(g, x.reshape(280, K), w, fb.ACT_RELU, pre[:280, off:off + N])
        assert grads[0].shape == x.shape
        for a, b, c in zip((grads[0].reshape(280, K),) + grads[1:], wants, bounds):
            ref.check(a, b, c, (off, pad, K, N))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [3, 500, 5000])
def test_residual_in_place(rows, dtype):
    gen, x, w, b = inputs(rows, 96, 160, dtype)
    r = draw(gen, rows, 160, dtype=dtype)
    want = fb.linear(x, w, b, act=fb.ACT_GELU, residual=r)
    assert fb.linear(x, w, b, act=fb.ACT_GELU, residual=r, out=r).data_ptr() == r.data_ptr()
    assert torch.equal(r, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_rows(dtype):
    gen, x, w, b = inputs(0, 40, 24, dtype)
    assert fb.linear(x, w, b, act=fb.ACT_GELU).shape == (0, 24)
    assert fb.linear(x.reshape(0, 5, 40), w).shape == (0, 5, 24)
    gx, gw, gb = fb.linear_backward(torch.empty(0, 24, dtype=dtype, device="cuda"), x, w)
    assert gx.shape == (0, 40) and gw.shape == (24, 40) and not bool(gw.any()) and gb.shape == (24,) and not bool(gb.any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [4, 300])
def test_what_is_not_finite_stays_in_its_row(rows, dtype):
    gen, x, w, b = inputs(rows, 130, 72, dtype)
    clean = fb.linear(x, w, b, act=fb.ACT_SILU)
    x[1, 77] = float("nan")
    x[2, 3] = float("inf")
    out = fb.linear(x, w, b, act=fb.ACT_SILU)
    assert bool(out[1].isnan().all()) and not bool(out[2].isfinite().all())
    keep = [i for i in range(rows) if i not in (1, 2)]
    assert torch.equal(out[keep], clean[keep])
    big = draw(gen, 16, 8, dtype=dtype)
    big[0, 0] = 3e38
    assert bool(fb.linear(big, torch.eye(8, device="cuda").to(dtype)).isfinite().all())


def test_extreme_values_of_the_activations():
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3.0, -3.0, 13.9, -13.9, 14.1, -14.1, 60.0, -60.0, 3e38, -3e38, 90.0, -90.0], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    for dtype in (BF16, F32):
        for act in (fb.ACT_RELU, fb.ACT_GELU, fb.ACT_SILU):
            v = z.to(dtype).reshape(-1, 1)
            out = fb.linear(v, one.to(dtype), act=act).double().flatten()
            want = ref.activation(v.double().flatten(), act)
            assert bool(out.isfinite().all())
            assert torch.allclose(out, want, rtol=2.0 ** -7, atol=1e-6), (dtype, act)


def test_results_are_the_same_bits_every_time():
    for rows, K, N, dtype in ((700, 2048, 96, BF16), (700, 2048, 96, F32), (4, 300, 200, BF16)):
        gen, x, w, b = inputs(rows, K, N, dtype)
        g = draw(gen, rows, N, dtype=dtype)
        first = (fb.linear(x, w, b),) + fb.linear_backward(g, x, w)
        for _ in range(3):
            for a, c in zip(first, (fb.linear(x, w, b),) + fb.linear_backward(g, x, w)):
                assert torch.equal(a, c)


def test_float32_sums_are_as_near_as_float32_is():
    """Long sums: tensor cores that cut off at every step would be off by 2^-24 for each; 1e-6 is what float32 sums in blocks reach."""
    for rows, K, N in ((2000, 4096, 256), (12, 4096, 700)):
        gen, x, w, b = inputs(rows, K, N, F32)
        out, want = fb.linear(x, w), x.double() @ w.double().T
        assert ((out - want).norm() / want.norm()).item() < 1e-6
        g = draw(gen, rows, N, dtype=F32)
        for got, a in zip(fb.linear_backward(g, x, w), (g.double() @ w.double(), g.double().T @ x.double())):
            assert ((got - a).norm() / a.norm()).item() < 2e-6


def test_rows_beyond_32_bit_offsets():
    rows, K, N = 9_000_000, 256, 16
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB")
    gen, _, w, b = inputs(1, K, N, BF16)
    x = torch.zeros(rows, K, dtype=BF16, device="cuda")
    at = torch.tensor([0, 8_388_607, 8_388_608, 8_388_609, rows - 1], device="cuda")
    x[at] = draw(gen, 5, K, dtype=BF16)
    out = fb.linear(x, w, b)
    want, _, off, _ = ref.linear(x[at], w, b)
    ref.check(out[at], want, off)
    assert torch.equal(out[1], b) and torch.equal(out[rows - 2], b)


def test_streams_and_graphs():
    gen, x, w, b = inputs(600, 1024, 96, BF16)
    g = draw(gen, 600, 96, dtype=BF16)
    z = torch.empty(600, 96, dtype=BF16, device="cuda")

    def step():
        out = fb.linear(x, w, b, act=fb.ACT_GELU, preact=z)
        return (out,) + fb.linear_backward(g, x, w, act=fb.ACT_GELU, preact=z)

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    named = fb.linear(x, w, b, act=fb.ACT_GELU, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(named, want[0])
    graphs = []
    for _ in range(2):           # two graphs, each with scratch of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        graphs.append((graph, outs))
    for turn in range(3):
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            for a, c in zip(outs, want):
                assert torch.equal(a, c)
        x.copy_(draw(gen, 600, 1024, dtype=BF16))
        want = [t.clone() for t in step()]
    # two calls at once on two streams
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for s in (first, second) * 4:
        with torch.cuda.stream(s):
            outs.append(fb.linear(x, w, b, act=fb.ACT_GELU))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) for o in outs)


def test_c_abi_without_scratch_and_its_error_word():
    """A call of few rows and a long sum without scratch gives the same numbers from one thread block per tile; the error word stays 0."""
    gen, x, w, b = inputs(40, 8192, 96, BF16)
    with_scratch = fb.linear(x, w, b)
    assert fb.flashbev_last_launch_count() == 2
    out = torch.empty_like(with_scratch)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = fb.LinearParams()
    p.struct_size = ctypes.sizeof(p)
    p.x, p.weight, p.bias, p.out, p.error_word = x.data_ptr(), w.data_ptr(), b.data_ptr(), out.data_ptr(), word.data_ptr()
    p.rows, p.in_features, p.out_features, p.dtype, p.out_dtype = 40, 8192, 96, fb.BF16, fb.BF16
    fb.flashbev_linear(p, torch.cuda.current_stream().cuda_stream)
    assert fb.flashbev_last_launch_count() == 1
    torch.cuda.synchronize()
    want, _, off, _ = ref.linear(x, w, b)
    ref.check(out, want, off)
    ref.check(with_scratch, want, off)
    assert int(word) == 0
    p.dtype = p.out_dtype = fb.F32   # float32 operands are laid out in scratch
    assert fb.flashbev_linear(p, None, check=False) == fb.TOO_SMALL


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(200, 256, 256), (320, 1024, 256), (900, 300, 256), (100, 264, 1000), (64, 1024, 1600), (16, 2048, 64), (2500, 48, 32)])
def test_sums_that_may_be_shared_and_need_not(shape, dtype):
    """Sizes on either side of where blocks begin to share sums: forward, both products of the backward, and again without scratch."""
    rows, K, N = shape
    gen, x, w, b = inputs(rows, K, N, dtype, 11)
    want, _, off, _ = ref.linear(x, w, b)
    ref.check(fb.linear(x, w, b), want, off, shape)
    g = draw(gen, rows, N, dtype=dtype)
    wants, bounds = ref.linear_backward(g, x, w, fb.ACT_NONE, None)
    for wanted in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1)):
        grads = fb.linear_backward(g, x, w, grad_x=wanted[0], grad_weight=wanted[1], grad_bias=wanted[2])
        for got, a, bound, asked in zip(grads, wants, bounds, wanted):
            assert (got is not None) == bool(asked)
            if asked:
                ref.check(got, a, bound, (shape, wanted))


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("off, pad, N", [(0, 0, 130), (0, 3, 130), (1, 0, 130), (2, 2, 130), (0, 1, 129), (1, 7, 8), (0, 8, 264), (2, 6, 264)])
def test_gradients_of_many_rows_at_any_alignment(off, pad, N, types):
    dtype, grad_type = types
    rows, K = 3001, 40
    gen, x, w, b = inputs(rows, K, N, dtype, 13)
    g = draw(gen, rows, off + N + pad, dtype=grad_type)[:, off:off + N]
    z = draw(gen, rows, N + 2, dtype=dtype)[:, :N]
    for act, pre in ((fb.ACT_NONE, None), (fb.ACT_GELU, z)):
        wants, bounds = ref.linear_backward(g, x, w, act, pre)
        for got, a, bound, what in zip(fb.linear_backward(g, x, w, act=act, preact=pre), wants, bounds, ("x", "weight", "bias")):
            ref.check(got, a, bound, (off, pad, N, act, what))
