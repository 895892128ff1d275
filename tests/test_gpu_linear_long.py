"""Sums over very many terms, whose results are rounded to bf16 once: what the tensor cores cut off on the way has to stay well below that rounding,
however long the sum is."""
import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32

#: A sum leaves the tensor cores after 32768 terms at the latest, 2048 instructions, each of which cuts off up to two steps, 2 x 2^-23, of what it
#: has so far (its 16 products and the sum are aligned to the largest of them, and each loses what lies below; 1.7 steps were measured): of
#: like-signed terms half of the whole on the average.
MOST_CUT = 2048 * 2 * 2.0 ** -23 / 2


def positive(gen, rows, width, dtype=BF16):
    """|normal| numbers, every column times a number of its own between 1 and 2, so that sums lie anywhere between two powers of two."""
    v = torch.empty(rows, width, dtype=dtype, device="cuda")
    scale = 1 + torch.rand(width, generator=gen, device="cuda")
    for at in range(0, rows, 1 << 17):
        part = v[at:at + (1 << 17)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").abs_() * scale)
    return v


def check(got, want, n_cut=MOST_CUT):
    """Each number within half a step of bf16, 2^-8 of it, beyond what was cut off; and their mean, in which the roundings (of 1.6e-3 each,
    either way) cancel to 1.6e-3 / sqrt(n), six times that."""
    off = (got.double() - want) / want
    assert off.abs().max().item() <= 2.0 ** -8 + n_cut
    assert abs(off.mean().item()) <= n_cut + 6 * 1.6e-3 / off.numel() ** 0.5, off.mean().item()


def test_gradient_of_weights_over_a_million_rows():
    """So many tiles that every sum belongs to one thread block."""
    rows, K, N = (1 << 20) + 70, 2048, 1160
    gen = torch.Generator(device="cuda").manual_seed(1)
    g, x = positive(gen, rows, N), positive(gen, rows, K)
    w = torch.empty(N, K, dtype=BF16, device="cuda")
    _, gw, gb = fb.linear_backward(g, x, w, grad_x=False)
    some = [0, 127, 640, N - 1]
    want = torch.zeros(len(some), K, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 1 << 16):
        want += g[at:at + (1 << 16), some].double().T @ x[at:at + (1 << 16)].double()
    check(gw[some], want)
    bias = sum(g[at:at + (1 << 16)].double().sum(0) for at in range(0, rows, 1 << 16))
    assert ((gb.double() - bias) / bias).abs().max().item() <= 2.0 ** -8 + 1e-5


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows, K, N", [(1300, (1 << 17) + 40, 2000), (1300, (1 << 17) + 40, 1000), (700, (1 << 17) + 40, 700), (20, 1 << 18, 96)])
def test_long_sums_of_a_forward_call(rows, K, N, dtype):
    """Sums of one block each, and sums that blocks share, in shares longer and shorter than a run."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w = positive(gen, rows, K, dtype), positive(gen, N, K, dtype)
    out = fb.linear(x, w, out_dtype=fb.BF16)
    some = sorted({0, min(127, rows - 1), rows // 2, rows - 1})
    want = torch.zeros(len(some), N, dtype=torch.float64, device="cuda")
    for at in range(0, K, 1 << 14):
        want += x[some, at:at + (1 << 14)].double() @ w[:, at:at + (1 << 14)].double().T
    check(out[some], want)
