"""Activations of bf16 results in calls of few rows and of shared sums, which nothing but their rounding may distinguish from the formula."""
import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402

BF16 = torch.bfloat16


@pytest.mark.parametrize("act", [fb.ACT_RELU, fb.ACT_GELU, fb.ACT_SILU])
@pytest.mark.parametrize("rows, K, N, launches", [(1, 1, 20000, 1), (3, 7, 9000, 1), (8, 1, 4096, 1), (8, 1024, 4096, 1), (40, 8192, 520, 2)])
def test_few_rows_and_shared_sums_are_rounded_once(rows, K, N, launches, act):
    """Sums of one product, which is exact: what is left is the activation's formula, a few steps of float32 and, of the two exponentials at
    -z^2 / 2 and z, their arguments' rounding, together below (z^2 + 8) 2^-23 of the result; and half a step of bf16."""
    gen = torch.Generator(device="cuda").manual_seed(rows + N)
    x = torch.zeros(rows, K, dtype=BF16, device="cuda")
    x[:, 0] = 1 + torch.rand(rows, generator=gen, device="cuda")
    w = torch.zeros(N, K, dtype=BF16, device="cuda")
    w[:, 0] = 4 * torch.rand(N, generator=gen, device="cuda") - 2.5
    out = fb.linear(x, w, act=act)
    assert fb.flashbev_last_launch_count() == launches
    z = x[:, :1].double() * w[:, 0].double()
    want = ref.activation(z, act)
    step = 2.0 ** (torch.floor(torch.log2(want.abs().clamp_min(1e-30))) - 7)
    over = (out.double() - want).abs() - 0.5 * step - (z * z + 8) * 2.0 ** -23 * want.abs()
    assert over.max().item() <= 0, (int((over > 0).sum()), over.numel())


EXTREMES = [0.0, -0.0, 1e-30, -1e-30, 0.7, -0.7, -0.75, 5.9, -5.9, 6.1, -6.1, 13.9, -13.9, 14.1, -14.1, 60.0, -60.0, 90.0, -90.0, 1e19, -1e19, 2e19, -2e19, 3e38, -3e38]


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("act", [fb.ACT_RELU, fb.ACT_GELU, fb.ACT_SILU])
def test_slopes_at_extreme_values(act, dtype):
    """z^2 beyond what float32 holds, exponentials of 0 and infinity.  The slopes' formulas are 3.1e-5 off for bf16 numbers, eight roundings of
    terms up to 1.3 for float32 ones; the bf16 gradient is rounded twice, the three pieces of a float32 one hold it."""
    z = torch.tensor(EXTREMES, device="cuda").to(dtype).reshape(-1, 1)
    one = torch.ones(1, 1, dtype=dtype, device="cuda")
    gx, _, gb = fb.linear_backward(torch.ones_like(z), z, one, act=act, preact=z)
    want = ref.activation_slope(z.double(), act)
    off = 3.1e-5 if dtype is BF16 else 1.3 * 8 * 2.0 ** -24
    half = ref.HALF_STEP[dtype]
    assert ((gx.double() - want).abs() - off - 2 * half * want.abs()).max().item() <= 0
    assert abs(gb.item() - want.sum().item()) <= len(EXTREMES) * off + (half + 2.0 ** -20) * want.abs().sum().item()


@pytest.mark.parametrize("rows", [1, 8, 300])
def test_infinite_sums(rows):
    """GELU and ReLU of minus infinity are 0, their limit, whichever kernel forms them."""
    x = torch.full((rows, 1), float("-inf"), dtype=BF16, device="cuda")
    w = torch.ones(3, 1, dtype=BF16, device="cuda")
    for act in (fb.ACT_RELU, fb.ACT_GELU):
        for out_dtype in (fb.BF16, fb.F32):
            assert bool((fb.linear(x, w, act=act, out_dtype=out_dtype) == 0).all()), (act, out_dtype)
            assert bool((fb.linear(-x, w, act=act, out_dtype=out_dtype) == float("inf")).all())
    assert bool((fb.linear(x, w) == float("-inf")).all())
