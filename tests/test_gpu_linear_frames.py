"""Matrices that are part of wider ones, whose rows start on 16-byte boundaries and end anywhere: what lies behind a row's end is neither
read nor written."""
import ctypes

import pytest

from paper_2607_10071_b200 import binding as fb

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests import layer_reference as ref  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Frame:
    """rows x width in the first columns of a wider matrix of `fill`, one row of which follows"""

    def __init__(self, rows, width, dtype, fill, data=None):
        self.all = torch.full((rows + 1, (width + 7) // 8 * 8 + 8), fill, dtype=dtype, device="cuda")
        self.part = self.all[:rows, :width]
        self.fill = fill
        if data is not None:
            self.part.copy_(data)
        assert self.part.data_ptr() % 16 == 0 and self.part.stride(0) * self.part.element_size() % 16 == 0

    def untouched(self):
        return bool((self.all[-1] == self.fill).all()) and bool((self.all[:, self.part.shape[1]:] == self.fill).all())


def inputs(rows, K, N, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + 31 * K + N)

    def draw(*shape, dtype=dtype, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    return draw, Frame(rows, K, dtype, float("nan"), draw(rows, K)), Frame(N, K, dtype, float("nan"), draw(N, K, scale=K ** -0.5))


SHAPES = [(20, 207, 51), (300, 82, 130), (61, 29, 483), (1677, 208, 11), (20000, 33, 65), (400, 3000, 97), (130, 64, 7), (40000, 90, 250), (5, 83, 41)]


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, types):
    rows, K, N = shape
    dtype, out_dtype = types
    draw, x, w = inputs(rows, K, N, dtype)
    for act, keep, residual in ((fb.ACT_NONE, False, False), (fb.ACT_RELU, True, True), (fb.ACT_SILU, False, True), (fb.ACT_NONE, True, False)):
        out, z = Frame(rows, N, out_dtype, 7.0), Frame(rows, N, dtype, 7.0) if keep else None
        r = Frame(rows, N, out_dtype, float("nan"), draw(rows, N, dtype=out_dtype)) if residual else None
        fb.linear(x.part, w.part, act=act, residual=r.part if r else None, out=out.part, preact=z.part if z else None)
        want, wz, off, off_z = ref.linear(x.part, w.part, None, act, r.part if r else None)
        ref.check(out.part, want, off, (shape, act))
        assert out.untouched(), (shape, act)
        if z:
            ref.check(z.part, wz, off_z, (shape, act, "z"))
            assert z.untouched(), (shape, act)


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, types):
    rows, K, N = shape
    dtype, grad_dtype = types
    draw, x, w = inputs(rows, K, N, dtype)
    g = Frame(rows, N, grad_dtype, float("nan"), draw(rows, N, dtype=grad_dtype))
    for act in (fb.ACT_NONE, fb.ACT_SILU):
        z = Frame(rows, N, dtype, float("nan"), draw(rows, N)) if act else None
        gx, gw, gb = Frame(rows, K, dtype, 7.0), Frame(N, K, dtype, 7.0), Frame(1, N, dtype, 7.0)
        p = fb.LinearBackwardParams()
        p.struct_size = ctypes.sizeof(p)
        p.grad_out, p.x, p.weight, p.preact = (m.part.data_ptr() if m else None for m in (g, x, w, z))
        p.grad_x, p.grad_weight, p.grad_bias = (m.part.data_ptr() for m in (gx, gw, gb))
        p.ld_grad_out, p.ld_x, p.ld_weight, p.ld_preact, p.ld_grad_x, p.ld_grad_weight = (m.all.shape[1] if m else 0 for m in (g, x, w, z, gx, gw))
        p.rows, p.in_features, p.out_features, p.act = rows, K, N, act
        p.dtype, p.grad_dtype = (fb.F32 if t is F32 else fb.BF16 for t in types)
        scratch = torch.full((fb.flashbev_linear_backward_workspace_bytes(p),), 255, dtype=torch.uint8, device="cuda")
        p.workspace, p.workspace_bytes = (scratch.data_ptr(), scratch.numel()) if scratch.numel() else (None, 0)
        fb.flashbev_linear_backward(p, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        wants, bounds = ref.linear_backward(g.part, x.part, w.part, act, z.part if z else None)
        for m, want, off, what in zip((gx, gw, gb), wants, bounds, ("x", "weight", "bias")):
            ref.check(m.part[0] if what == "bias" else m.part, want, off, (shape, act, what))
            assert m.untouched(), (shape, act, what)
