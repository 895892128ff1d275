"""The operators of a transformer layer on tensors of more than 2^31 elements, and called from two host threads at once."""
import threading

import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402
from tests.test_gpu_block_norm_sums import KEYS, bounds  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
ROWS = 9_000_000
#: The first and last rows, those around 2^31 elements of 256 to a row, and one of no particular place; the others are zeros.
AT = (0, 8_388_607, 8_388_608, 8_388_609, 5_000_011, ROWS - 1)


@pytest.fixture(autouse=True)
def memory_given_back():
    yield
    torch.cuda.empty_cache()


def some(gen, width, dtype, scale=1.0):
    """All rows, and those of them that are not zeros"""
    t = torch.zeros(ROWS, width, dtype=dtype, device="cuda")
    at = torch.tensor(AT, device="cuda")
    t[at] = (torch.randn(len(AT), width, generator=gen, device="cuda") * scale).to(dtype)
    return t, t[at]


def need(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip(f"needs {gigabytes} GB")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K, N", [(256, 16), (16, 256)])
def test_products_and_their_gradients(K, N, dtype):
    need(80)
    gen = torch.Generator(device="cuda").manual_seed(K)
    at = torch.tensor(AT, device="cuda")
    x, xs = some(gen, K, dtype)
    w = (torch.randn(N, K, generator=gen, device="cuda") * K ** -0.5).to(dtype)
    b = torch.randn(N, generator=gen, device="cuda").to(dtype)
    r, rs = some(gen, N, dtype)
    z = torch.empty(ROWS, N, dtype=dtype, device="cuda")
    out = fb.linear(x, w, b, act=fb.ACT_SILU, residual=r, preact=z)
    want, wz, off, off_z = ref.linear(xs, w, b, fb.ACT_SILU, rs)
    ref.check(out[at], want, off)
    ref.check(z[at], wz, off_z)
    zero = fb.linear(x[:1] * 0, w, b, act=fb.ACT_SILU)[0]                # what a row of zeros gives
    for i in (1, 8_388_606, 8_388_610, ROWS - 2):
        assert torch.equal(z[i], b) and torch.allclose(out[i].float(), zero.float(), rtol=2.0 ** -7, atol=0)
    del out, r
    g, gs = some(gen, N, dtype)
    gx, gw, gb = fb.linear_backward(g, x, w, act=fb.ACT_SILU, preact=z)
    want, off = ref.linear_backward(gs, xs, w, fb.ACT_SILU, z[at])
    ref.check(gx[at], want[0], off[0])
    assert not bool(gx[8_388_000:8_388_600].any()) and not bool(gx[-1000:-1].any())
    ref.check(gw, want[1], off[1])
    ref.check(gb, want[2], off[2])


@pytest.mark.parametrize("types, gates", [((BF16, BF16, F32), 0), ((BF16, BF16, BF16), ROWS), ((F32, BF16, F32), 2)])
def test_norms_and_their_gradients(types, gates):
    need(90)
    C = 256
    gen = torch.Generator(device="cuda").manual_seed(gates + 1)
    at = torch.tensor(AT, device="cuda")
    x, xs = some(gen, C, types[0])
    y, ys = some(gen, C, types[1])
    gate, shared = None, None
    if gates == ROWS:
        gate, shared = some(gen, C, types[2])
    elif gates:
        gate = torch.randn(gates, C, generator=gen, device="cuda").to(types[2])
        shared = gate[at * gates // ROWS]
    parameters = dict(scale=0.5, after=fb.NORM_RMS, before=fb.NORM_LAYER, eps=1e-5)
    for k in ("after_weight", "after_bias", "before_weight", "before_bias"):
        parameters[k] = (1 + torch.randn(C, generator=gen, device="cuda") * 0.3).to(types[2]) if k != "after_bias" else None
    h, n = fb.block_norm(x, y, gate=gate, **parameters)
    few = dict(x=xs, y=ys, gate=shared, **parameters)
    d = {k: None if few[k] is None else few[k].double().requires_grad_(True) for k in KEYS}
    wh, wn = ref.block_norm(d["x"], d["y"], d["gate"], 0.5, fb.NORM_RMS, d["after_weight"], None, fb.NORM_LAYER, d["before_weight"], d["before_bias"], 1e-5)
    step = 2.0 ** -24
    ref.check(h[at], wh, 64 * step * (wh.abs() + 1))
    ref.check(n[at], wn, 64 * step * (wn.abs() + 1) * 4)
    assert not bool(h[8_388_000:8_388_600].any()) and torch.equal(n[-2], parameters["before_bias"].to(types[1]))
    del h, n
    gh, ghs = some(gen, C, types[0])
    gn, gns = some(gen, C, types[1])
    got = dict(zip(KEYS, fb.block_norm_backward(gh, gn, x, y, gate=gate, **parameters)))
    keys = [k for k in KEYS if d[k] is not None]
    want = dict(zip(keys, torch.autograd.grad([wh, wn], [d[k] for k in keys], [ghs.double(), gns.double()])))
    off = bounds(few, ghs, gns, 64)
    for k in keys:
        t = got[k]
        if k in ("x", "y") or k == "gate" and gates == ROWS:
            ref.check(t[at], want[k], off[k], k)
            assert not bool(t[8_388_000:8_388_600].any()) and not bool(t[-1000:-1].any())
        elif k == "gate":
            for i in range(gates):
                mine = at * gates // ROWS == i
                ref.check(t[i], want[k][mine].sum(0), off[k][mine].sum(0), k)
        else:
            ref.check(t, want[k], off[k], k)


def test_two_host_threads():
    """Each on a stream of its own, as many calls as it can, all of them the same numbers as one after another."""
    gen = torch.Generator(device="cuda").manual_seed(5)

    def draw(*shape, dtype):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def calls(dtype, rows, K, N):
        x, w, b, g, z = draw(rows, K, dtype=dtype), draw(N, K, dtype=dtype), draw(N, dtype=dtype), draw(rows, N, dtype=dtype), draw(rows, N, dtype=dtype)
        y, gate, v = draw(rows, K, dtype=dtype), draw(3, K, dtype=F32), draw(K, dtype=F32)

        def run():
            out = (fb.linear(x, w, b, act=fb.ACT_GELU),) + fb.linear_backward(g, x, w, act=fb.ACT_GELU, preact=z)
            out += fb.block_norm(x, y, gate=gate, before_weight=v) + fb.block_norm_backward(x, y, x, y, gate=gate, before_weight=v)
            return [t for t in out if t is not None]
        return run

    work = [calls(BF16, 3000, 520, 264), calls(F32, 600, 2048, 96)]
    want = [[t.clone() for t in run()] for run in work]
    torch.cuda.synchronize()
    wrong = []

    def go(run, expected):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(60):
                    if not all(torch.equal(s, t) for s, t in zip(run(), expected)):
                        wrong.append("numbers")
        except Exception as e:                                               # (a thread's exception is not the test's)
            wrong.append(repr(e))

    threads = [threading.Thread(target=go, args=a) for a in zip(work, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]
    assert fb.linear_given_up() == 0
