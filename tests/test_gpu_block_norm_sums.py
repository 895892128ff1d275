"""Gradients of the norms between residual blocks against bounds that are made of the numbers a sum has: nothing held in fewer bits than
float32, and no row left out, stays below them, however many rows there are."""
import itertools

import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402
from tests.test_gpu_block_norm import EPS, case, plain  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
KEYS = ("x", "y", "gate", "after_weight", "after_bias", "before_weight", "before_bias")


def bounds(a, gh, gn, chain):
    """What each gradient may be off by before its own rounding.

    Statistics are sums in trees of 8 numbers and up to 9 levels, a whitened number has about a dozen roundings more: 32 steps of 2^-24 of itself
    and of 1 (the mean's).  A gradient that went back through a norm is as near to the sum of its terms' sizes, which are all positive
    here; one that is a sum over rows adds a rounding for each of the `chain` sums on the way to a term."""
    d = {k: None if a[k] is None else a[k].double() for k in KEYS}
    rows, C = d["x"].shape
    step = 2.0 ** -24
    one = torch.ones(1, dtype=torch.float64, device="cuda")

    def weight(k):
        return one if d[k] is None else d[k].abs()

    def statistics(v, kind):
        if kind == fb.NORM_LAYER:
            v = v - v.mean(-1, keepdim=True)
        r = 1 / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        return (v * r).abs() + 1, r

    def back(g, t, r):
        return r * (g + g.mean(-1, keepdim=True) + t * (g * t).mean(-1, keepdim=True))

    gate = one if d["gate"] is None else d["gate"].reshape(-1, C).repeat_interleave(rows // d["gate"].reshape(-1, C).shape[0], 0).abs()
    gate = gate * abs(a["scale"])
    h, _ = ref.block_norm(d["x"], d["y"], d["gate"], a["scale"], a["after"], d["after_weight"], d["after_bias"], fb.NORM_NONE, None, None, EPS)
    off = {}
    size = torch.zeros_like(h) if gh is None else gh.double().abs()
    if a["before"]:
        u, r = statistics(h, a["before"])
        g = gn.double().abs()
        # (h is as near as its own size; a small deviation magnifies that)
        u = u + r * h.abs()
        off["before_weight"], off["before_bias"] = (g * u).sum(0), g.sum(0)
        size = size + back(g * weight("before_weight"), u, r)
    off["x"] = size
    branch = d["y"].abs()
    through = size * gate
    if a["after"]:
        v, r = statistics(d["y"], a["after"])
        branch = v * weight("after_weight") + (0 if d["after_bias"] is None else d["after_bias"].abs())
        off["after_weight"], off["after_bias"] = (through * v).sum(0), through.sum(0)
        through = back(through * weight("after_weight"), v, r)
    off["y"] = through
    if d["gate"] is not None:
        off["gate"] = (size * branch * abs(a["scale"])).reshape(-1, rows // d["gate"].reshape(-1, C).shape[0], C).sum(1).reshape(d["gate"].shape)
    return {k: v * step * (32 if k in ("x", "y") else 32 + chain) for k, v in off.items()}


def run(rows, C, types, after, before, gates, keep, seed=0):
    gen, draw, a = case(rows, C, types, after, before, gates, True, seed)
    gn = draw(rows, C, dtype=types[1]) if before else None
    gh = draw(rows, C, dtype=types[0]) if keep or not before else None
    got = dict(zip(KEYS, fb.block_norm_backward(gh, gn, **a)))
    d, h, n = plain(a, True)
    ends = [(t, g.double()) for t, g in ((h, gh), (n, gn)) if g is not None]
    keys = [k for k in KEYS if d[k] is not None]
    want = dict(zip(keys, torch.autograd.grad([t for t, _ in ends], [d[k] for k in keys], [g for _, g in ends])))
    # a register's sum over a team's rows, the teams of a block, and the blocks' sums: 16 threads, then their sums
    teams = max(1, 256 // max(4, 1 << max(0, (C - 1).bit_length() - 3)))
    chain = 2 * rows / (148 * teams) + 8 + max(296, gates) / 16 + 16
    what = (rows, C, after, before, gates)
    for k, off in bounds(a, gh, gn, chain).items():
        if want.get(k) is None:
            continue
        ref.check(got[k], want[k], off, what + (k,))
        # (roundings go either way; the bounds above do not count on it)
        if got[k].dtype == F32:
            assert ((got[k].double() - want[k]).norm() / want[k].norm()).item() < 1e-6, what + (k,)


TYPES = [(F32, F32, F32), (F32, BF16, F32), (BF16, BF16, F32)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", [8, 33, 82, 256, 264, 1000, 2050, 4096])
def test_rows_and_their_sums(C, types):
    for i, (after, before, gates) in enumerate(itertools.product((0, 1, 2), (0, 1, 2), (0, 1, 41, 82))):
        run(82, C, types, after, before, gates, i % 2)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows, gates, C", [
    (30000, 0, 256), (30000, 10, 256), (20000, 0, 82), (9000, 1, 2050),
    # a block for each of more gates than run at once; and teams that take whole gates, one or several after another
    (19200, 300, 32), (24000, 400, 256), (30000, 500, 1000), (64000, 1000, 33), (90000, 3000, 32),
    (6000, 1200, 256), (15000, 3000, 33), (60000, 12000, 32), (40000, 20000, 30), (9000, 3000, 264), (3000, 600, 4096)])
def test_many_rows_and_gates(rows, gates, C, types):
    for after, before in ((fb.NORM_RMS, fb.NORM_LAYER), (fb.NORM_NONE, fb.NORM_RMS)):
        run(rows, C, types, after, before, gates, True, 3)
