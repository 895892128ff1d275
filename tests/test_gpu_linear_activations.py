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
