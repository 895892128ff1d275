"""The norms and the sum between two residual blocks, and their gradients, against plain 64-bit forms."""
import itertools

import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
TYPES = [(F32, F32, F32), (BF16, BF16, BF16), (BF16, BF16, F32), (F32, BF16, F32), (F32, BF16, BF16)]
WIDTHS = [1, 2, 3, 8, 30, 31, 32, 82, 128, 136, 255, 256, 264, 510, 1000, 1024, 2049, 4096]
EPS = 1e-5


def case(rows, C, types, after, before, gates, bias, seed=0):
    stream, branch, param = types
    gen = torch.Generator(device="cuda").manual_seed(1000 * C + rows + seed)

    def draw(*shape, dtype, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)

    a = dict(x=draw(rows, C, dtype=stream, scale=2.0, shift=0.3), y=draw(rows, C, dtype=branch),
             gate=draw(gates, C, dtype=param, shift=0.5) if gates else None, scale=0.75, after=after,
             after_weight=draw(C, dtype=param, scale=0.3, shift=1.0) if after else None,
             after_bias=draw(C, dtype=param, scale=0.3) if after and bias else None, before=before,
             before_weight=draw(C, dtype=param, scale=0.3, shift=1.0) if before else None,
             before_bias=draw(C, dtype=param, scale=0.3) if before and bias else None, eps=EPS)
    return gen, draw, a


def plain(a, grad=False):
    """Leaves in 64 bits and the results."""
    keys = ("x", "y", "gate", "after_weight", "after_bias", "before_weight", "before_bias")
    d = {k: None if a[k] is None else a[k].double().requires_grad_(grad) for k in keys}
    h, n = ref.block_norm(d["x"], d["y"], d["gate"], a["scale"], a["after"], d["after_weight"], d["after_bias"], a["before"], d["before_weight"],
                          d["before_bias"], a["eps"])
    return d, h, n


def near(got, want, what, steps=32.0):
    """Statistics of float32 numbers: sums in trees of at most 16 levels, and a dozen roundings, of quantities up to the row's largest."""
    size = want.abs().amax(-1, keepdim=True) if want.dim() > 1 else want.abs().max()
    ref.check(got, want, steps * 2.0 ** -24 * (size + want.abs()) * 4, what)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_forward(C, types):
    for i, (after, before, gates) in enumerate(itertools.product((0, 1, 2), (0, 1, 2), (0, 1, 3))):
        if C == 1 and fb.NORM_LAYER in (after, before):
            continue             # (a row of one number has no deviation: 0 divided by the root of eps)
        gen, draw, a = case(39, C, types, after, before, (0, 1, 3)[gates % 3] if gates < 2 else (3, 39)[i % 2], i % 2)
        h, n = fb.block_norm(**a)
        _, wh, wn = plain(a)
        near(h, wh, (C, after, before, gates, "h"))
        assert (n is None) == (wn is None)
        if n is not None:
            # (a small deviation magnifies what h is off by)
            grow = 1.0 + float((wh.abs().amax(-1) / (wh - wh.mean(-1, keepdim=True)).pow(2).mean(-1).add(EPS).sqrt()).max()) if C > 1 else 8.0
            near(n, wn, (C, after, before, gates, "n"), 32.0 * grow)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_backward(C, types):
    for i, (after, before, gates) in enumerate(itertools.product((0, 1, 2), (0, 1, 2), (0, 1, 41, 82))):
        if C < 8 and fb.NORM_LAYER in (after, before) or C == 1:
            continue             # (deviations near 0)
        rows = 82
        gen, draw, a = case(rows, C, types, after, before, gates, i % 2, 9)
        gn = draw(rows, C, dtype=types[1]) if before else None
        gh = draw(rows, C, dtype=types[0]) if i % 3 or not before else None
        got = fb.block_norm_backward(gh, gn, **a)
        d, h, n = plain(a, True)
        ends = [(t, g.double()) for t, g in ((h, gh), (n, gn)) if g is not None]
        keys = [k for k in d if d[k] is not None]
        want = dict(zip(keys, torch.autograd.grad([t for t, _ in ends], [d[k] for k in keys], [g for _, g in ends], allow_unused=True)))
        for k, t in zip(d, got):
            assert (t is None) == (d[k] is None), k
            if t is None or want[k] is None:
                continue
            assert t.dtype == a[k].dtype and t.shape == a[k].shape
            # rows: as the forward call, a few times over; parameters: sums over the rows of numbers each so near
            spread = 1.0 if k in ("x", "y") else rows ** 0.5
            near(t, want[k], (C, after, before, gates, k), 256.0 * spread * (4 if C < 32 else 1))


@pytest.mark.parametrize("before", [fb.NORM_LAYER, fb.NORM_RMS])
def test_gradients_against_differences(before):
    """Central differences of float32 calls along the gradients: steps of 2^-7 of unit directions (errors of the second order about 6e-5) and sums of
    6400 numbers that float32 rounds to 6e-8 each, over 2^-6 (about 3e-4), of derivatives above 1."""
    gen, draw, a = case(100, 64, (F32, F32, F32), fb.NORM_RMS, before, 4, True)
    gh, gn = draw(100, 64, dtype=F32), draw(100, 64, dtype=F32)
    grads = fb.block_norm_backward(gh, gn, **a)
    step = 2.0 ** -7
    for k, grad in zip(("x", "y", "gate", "after_weight", "after_bias", "before_weight", "before_bias"), grads):
        v = grad / grad.norm()
        ends = []
        for s in (step, -step):
            h, n = fb.block_norm(**{**a, k: a[k] + s * v})
            ends.append((h.double() * gh.double()).sum() + (n.double() * gn.double()).sum())
        slope = ((ends[0] - ends[1]) / (2 * step)).item()
        assert abs(slope - grad.norm().item()) <= 5e-3 * grad.norm().item() + 5e-3, (k, slope, grad.norm().item())


def test_many_rows_share_gates_as_they_come():
    """Blocks per gate, teams that take whole gates, and a gate for every row give the same sums."""
    for rows, gates, C in ((6000, 2, 64), (6000, 3000, 64), (6000, 6000, 64), (4096, 1024, 40), (30000, 10, 256), (20000, 5000, 2050)):
        gen, draw, a = case(rows, C, (F32, F32, F32), fb.NORM_RMS, fb.NORM_LAYER, gates, True)
        gn = draw(rows, C, dtype=F32)
        got = fb.block_norm_backward(None, gn, **a)
        d, h, n = plain(a, True)
        want = torch.autograd.grad(n, list(d.values()), gn.double())
        for k, t, w in zip(d, got, want):
            near(t, w, (rows, gates, C, k), 256.0 * (1.0 if k in ("x", "y") else (rows / (gates if k == "gate" else 1)) ** 0.5))
        again = fb.block_norm_backward(None, gn, **a)
        assert all(torch.equal(s, t) for s, t in zip(got, again))


def test_first_norm_of_a_layer_and_rows_without_deviation():
    for types in TYPES:
        x = torch.randn(50, 96, device="cuda").to(types[0])
        h, n = fb.block_norm(x)
        assert h is None and n.dtype == types[0]
        near(n, ref.whiten(x.double(), fb.NORM_LAYER, EPS), "n")
        flat = torch.full((3, 96), 5.0, device="cuda").to(types[0])
        flat[1] = 0
        h, n = fb.block_norm(flat)
        assert bool((n == 0).all())
        (gx,) = [t for t in fb.block_norm_backward(None, torch.ones_like(n), flat) if t is not None]
        assert bool(gx.isfinite().all())


def test_what_is_not_finite_stays_in_its_row():
    gen, draw, a = case(64, 40, (F32, BF16, F32), fb.NORM_LAYER, fb.NORM_RMS, 0, True)
    clean = fb.block_norm(**a)
    a["y"][5, 7] = float("nan")
    a["x"][9, 1] = float("inf")
    h, n = fb.block_norm(**a)
    assert bool(h[5].isnan().all()) and bool(n[5].isnan().all()) and not bool(n[9].isfinite().all())
    keep = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(h[keep], clean[0][keep]) and torch.equal(n[keep], clean[1][keep])


@pytest.mark.parametrize("types", TYPES)
def test_strides_places_and_what_lies_around(types):
    for off, pad, C in ((0, 8, 64), (2, 6, 82), (1, 2, 33), (4, 4, 64), (3, 5, 520)):
        gen, draw, a = case(30, C, types, fb.NORM_LAYER, fb.NORM_RMS, 1, True)
        want = fb.block_norm(**a)
        b = dict(a)
        for k in ("x", "y"):
            wide = draw(30, C + pad, dtype=a[k].dtype)
            wide[:, off:off + C] = a[k]
            b[k] = wide[:, off:off + C].reshape(5, 6, C) if off == 0 and pad == 0 else wide[:, off:off + C]
        frames = [torch.full((31, C + pad), 7.0, dtype=t, device="cuda") for t in types[:2]]
        h, n = fb.block_norm(**b, h=frames[0][:30, off:off + C], n=frames[1][:30, off:off + C])
        for got, w, f in zip((h, n), want, frames):
            near(got, w.double(), (off, pad, C), 64.0) if got.dtype == F32 else ref.check(got, w.double(), w.double().abs() * 2.0 ** -8)
            assert bool((f[30] == 7).all()) and bool((f[:, :off] == 7).all()) and bool((f[:, off + C:] == 7).all())
        # in place
        x, y = b["x"].clone(), b["y"].clone()
        h, n = fb.block_norm(**{**b, "x": x, "y": y}, h=x, n=y)
        assert h.data_ptr() == x.data_ptr() and n.data_ptr() == y.data_ptr()
        for got, w in zip((x, y), want):
            near(got, w.double(), (off, pad, C), 64.0) if got.dtype == F32 else ref.check(got, w.double(), w.double().abs() * 2.0 ** -8)
        only = fb.block_norm(**a, keep_h=False)
        assert only[0] is None and torch.equal(only[1], want[1])


def test_no_rows():
    for types in TYPES:
        gen, draw, a = case(0, 24, types, fb.NORM_RMS, fb.NORM_LAYER, 1, True)
        h, n = fb.block_norm(**a)
        assert h.shape == n.shape == (0, 24)
        grads = fb.block_norm_backward(h, n, **a)
        assert grads[0].shape == (0, 24) and all(not bool(t.any()) for t in grads[2:])


def test_streams_and_graphs():
    gen, draw, a = case(3000, 256, (BF16, BF16, F32), fb.NORM_RMS, fb.NORM_RMS, 2, True)
    gn = draw(3000, 256, dtype=BF16)

    def step():
        return fb.block_norm(**a) + fb.block_norm_backward(gn, gn, **a)

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    named = fb.block_norm(**a, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(named[1], want[1])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        graphs.append((graph, outs))
    for graph, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, outs in graphs:
        assert all(torch.equal(s, t) for s, t in zip(outs, want))
