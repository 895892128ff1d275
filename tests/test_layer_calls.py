"""The calls of a transformer layer (``linear``, ``block_norm`` and their gradients): what they refuse, before any CUDA call."""
import ctypes

import pytest

from paper_2607_10071_b200 import binding as fb


def linear_params(**over):
    p = fb.LinearParams()
    p.struct_size = ctypes.sizeof(p)
    p.x, p.weight, p.bias, p.residual, p.out, p.preact_out = 4096, 8192, 12288, 16384, 20480, 24576
    p.rows, p.in_features, p.out_features = 100, 64, 96
    p.dtype, p.out_dtype, p.act = fb.BF16, fb.BF16, fb.ACT_GELU
    for k, v in over.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("over,status", [
    (dict(struct_size=8), fb.INVALID_ARG), (dict(x=None), fb.INVALID_ARG), (dict(weight=None), fb.INVALID_ARG), (dict(out=None), fb.INVALID_ARG),
    (dict(rows=-1), fb.INVALID_ARG), (dict(in_features=0), fb.INVALID_ARG), (dict(out_features=-3), fb.INVALID_ARG),
    (dict(dtype=2), fb.INVALID_ARG), (dict(out_dtype=-1), fb.INVALID_ARG), (dict(act=4), fb.INVALID_ARG), (dict(reserved=1), fb.INVALID_ARG),
    (dict(ld_x=63), fb.INVALID_ARG), (dict(ld_out=95), fb.INVALID_ARG), (dict(ld_weight=-64), fb.INVALID_ARG), (dict(ld_residual=1), fb.INVALID_ARG),
    (dict(ld_preact=95), fb.INVALID_ARG),
    (dict(rows=1 << 31), fb.UNSUPPORTED), (dict(in_features=(1 << 24) + 1), fb.UNSUPPORTED), (dict(ld_x=1 << 61), fb.UNSUPPORTED),
    (dict(rows=(1 << 31) - 200, out_features=1 << 23), fb.UNSUPPORTED),
    (dict(x=4097), fb.MISALIGNED), (dict(out_dtype=fb.F32, out=20482), fb.MISALIGNED), (dict(workspace=8200), fb.MISALIGNED),
    (dict(error_word=4098), fb.MISALIGNED),
])
def test_linear_refuses(over, status):
    assert fb.flashbev_linear(linear_params(**over), None, check=False) == status
    assert fb.flashbev_linear_workspace_bytes(linear_params(**over)) == 0


def test_linear_without_rows_enqueues_nothing():
    p = linear_params(rows=0, x=None, out=None)
    assert fb.flashbev_linear(p, None, check=False) == fb.OK and fb.flashbev_last_launch_count() == 0
    assert fb.lib().flashbev_linear(None, None) == fb.INVALID_ARG
    with pytest.raises(fb.FlashBevError):
        fb.flashbev_linear(linear_params(act=9), None)


def test_linear_asks_for_scratch_where_a_long_sum_has_few_tiles():
    assert fb.flashbev_linear_workspace_bytes(linear_params(rows=100000)) == 0
    few = linear_params(rows=100, in_features=8192)
    need = fb.flashbev_linear_workspace_bytes(few)
    assert need > 0 and need % (100 * 96 * 4) == 0                       # whole sums of 100 x 96
    assert fb.flashbev_linear_workspace_bytes(linear_params(rows=1, in_features=8192)) == 0


def backward_params(**over):
    p = fb.LinearBackwardParams()
    p.struct_size = ctypes.sizeof(p)
    p.grad_out, p.x, p.weight, p.preact, p.grad_x, p.grad_weight, p.grad_bias = (4096 * i for i in range(1, 8))
    p.rows, p.in_features, p.out_features = 100, 64, 96
    p.dtype, p.grad_dtype, p.act = fb.BF16, fb.BF16, fb.ACT_GELU
    p.workspace, p.workspace_bytes = 1 << 20, 1 << 30
    for k, v in over.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("over,status", [
    (dict(struct_size=16), fb.INVALID_ARG), (dict(grad_out=None), fb.INVALID_ARG), (dict(preact=None), fb.INVALID_ARG),
    (dict(x=None), fb.INVALID_ARG), (dict(weight=None), fb.INVALID_ARG), (dict(rows=-5), fb.INVALID_ARG), (dict(act=-1), fb.INVALID_ARG),
    (dict(ld_grad_x=63), fb.INVALID_ARG), (dict(ld_grad_weight=5), fb.INVALID_ARG), (dict(grad_dtype=3), fb.INVALID_ARG),
    (dict(dtype=fb.F32), fb.UNSUPPORTED),                                # a bf16 gradient beside float32 operands
    (dict(out_features=(1 << 24) + 8), fb.UNSUPPORTED),
    (dict(grad_weight=4097), fb.MISALIGNED), (dict(workspace=24), fb.MISALIGNED),
    (dict(workspace=None), fb.TOO_SMALL), (dict(workspace_bytes=100), fb.TOO_SMALL),
])
def test_linear_backward_refuses(over, status):
    assert fb.flashbev_linear_backward(backward_params(**over), None, check=False) == status


def test_linear_backward_scratch():
    # the rounded gradient before the activation, and sums for the bias
    assert fb.flashbev_linear_backward_workspace_bytes(backward_params()) >= 100 * 96 * 2 + 96 * 4
    assert fb.flashbev_linear_backward_workspace_bytes(backward_params(act=fb.ACT_NONE, rows=1 << 16, grad_bias=None, grad_weight=None)) == 0
    assert fb.lib().flashbev_linear_backward(None, None) == fb.INVALID_ARG


def norm_params(**over):
    p = fb.BlockNormParams()
    p.struct_size = ctypes.sizeof(p)
    p.x, p.y, p.gate, p.after_weight, p.after_bias, p.before_weight, p.before_bias, p.h, p.n = (4096 * i for i in range(1, 10))
    p.rows, p.gate_groups, p.C = 12, 3, 64
    p.after, p.before = fb.NORM_RMS, fb.NORM_LAYER
    p.dtype, p.branch_dtype, p.param_dtype = fb.F32, fb.BF16, fb.F32
    p.scale, p.eps = 1.0, 1e-5
    for k, v in over.items():
        setattr(p, k, v)
    return p


NORM_REFUSALS = [
    (dict(struct_size=8), fb.INVALID_ARG), (dict(x=None), fb.INVALID_ARG), (dict(rows=-1), fb.INVALID_ARG), (dict(C=0), fb.INVALID_ARG),
    (dict(after=3), fb.INVALID_ARG), (dict(before=-1), fb.INVALID_ARG), (dict(gate_groups=5), fb.INVALID_ARG), (dict(gate_groups=0), fb.INVALID_ARG),
    (dict(scale=float("nan")), fb.INVALID_ARG), (dict(eps=-1.0), fb.INVALID_ARG), (dict(eps=float("inf")), fb.INVALID_ARG),
    (dict(ld_x=63), fb.INVALID_ARG), (dict(ld_y=1), fb.INVALID_ARG), (dict(dtype=7), fb.INVALID_ARG),
    (dict(y=None), fb.INVALID_ARG),                                      # a gate and a norm behind a block that is not there
    (dict(after=fb.NORM_NONE), fb.INVALID_ARG),                          # parameters of a norm that is not there
    (dict(before=fb.NORM_NONE), fb.INVALID_ARG),
    (dict(dtype=fb.BF16, branch_dtype=fb.F32), fb.UNSUPPORTED), (dict(branch_dtype=fb.F32, param_dtype=fb.BF16), fb.UNSUPPORTED),
    (dict(C=fb.NORM_MAX_CHANNELS + 1), fb.UNSUPPORTED), (dict(rows=3 << 30), fb.UNSUPPORTED), (dict(ld_x=1 << 60), fb.UNSUPPORTED),
    (dict(x=4098), fb.MISALIGNED), (dict(before_weight=4098), fb.MISALIGNED), (dict(y=4097), fb.MISALIGNED),
]


@pytest.mark.parametrize("over,status", NORM_REFUSALS + [(dict(n=None), fb.INVALID_ARG), (dict(h=4097), fb.MISALIGNED), (dict(ld_n=63), fb.INVALID_ARG)])
def test_block_norm_refuses(over, status):
    assert fb.flashbev_block_norm(norm_params(**over), None, check=False) == status


def norm_backward_params(**over):
    p = fb.BlockNormBackwardParams()
    p.struct_size = ctypes.sizeof(p)
    for i, k in enumerate(("grad_h", "grad_n", "x", "y", "gate", "after_weight", "after_bias", "before_weight", "grad_x", "grad_y", "grad_gate",
                           "grad_after_weight", "grad_after_bias", "grad_before_weight", "grad_before_bias")):
        setattr(p, k, 4096 * (i + 1))
    p.rows, p.gate_groups, p.C = 1200, 3, 64
    p.after, p.before = fb.NORM_RMS, fb.NORM_LAYER
    p.dtype, p.branch_dtype, p.param_dtype = fb.F32, fb.BF16, fb.F32
    p.scale, p.eps = 1.0, 1e-5
    p.workspace, p.workspace_bytes = 1 << 20, 1 << 30
    for k, v in over.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("over,status", NORM_REFUSALS + [
    (dict(gate_groups=7), fb.INVALID_ARG), (dict(grad_n=None), fb.INVALID_ARG), (dict(gate=None), fb.INVALID_ARG),
    (dict(grad_y=4097), fb.MISALIGNED), (dict(workspace=None), fb.TOO_SMALL), (dict(workspace_bytes=64), fb.TOO_SMALL)])
def test_block_norm_backward_refuses(over, status):
    over = {k: v for k, v in over.items() if not (k == "gate_groups" and v == 5)} or dict(gate_groups=7)
    assert fb.flashbev_block_norm_backward(norm_backward_params(**over), None, check=False) == status


def test_block_norm_without_rows_enqueues_nothing():
    assert fb.flashbev_block_norm(norm_params(rows=0, x=None, y=4096, h=None, n=None), None, check=False) == fb.OK
    assert fb.flashbev_last_launch_count() == 0
    assert fb.lib().flashbev_block_norm(None, None) == fb.INVALID_ARG
    assert fb.lib().flashbev_block_norm_backward(None, None) == fb.INVALID_ARG
    assert fb.flashbev_block_norm_backward_workspace_bytes(norm_backward_params(rows=0)) == 0


@pytest.mark.parametrize("cname,mirror", [("flashbev_linear_params", "LinearParams"), ("flashbev_linear_backward_params", "LinearBackwardParams"),
                                          ("flashbev_block_norm_params", "BlockNormParams"),
                                          ("flashbev_block_norm_backward_params", "BlockNormBackwardParams")])
def test_ctypes_struct_matches_the_c_struct(tmp_path, cname, mirror):
    from tests.test_abi import test_ctypes_struct_matches_the_c_struct as check
    check(tmp_path, cname, mirror)


# ---- torch tensors: refused by the extension module (tensors without memory, which exist on machines without a GPU too)

def _fake(*shape, dtype="bfloat16", device="cuda"):
    torch = pytest.importorskip("torch")
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(shape, device=device, dtype=getattr(torch, dtype))


def test_linear_refuses_tensors():
    x, w = _fake(4, 6, 32), _fake(48, 32)
    calls = [
        (TypeError, lambda: fb.linear([1], w)),
        (ValueError, lambda: fb.linear(_fake(4, 32, device="cpu"), w)),
        (ValueError, lambda: fb.linear(_fake(4, 32, dtype="float16"), w)),
        (ValueError, lambda: fb.linear(x, _fake(48, 32, dtype="float32"))),
        (ValueError, lambda: fb.linear(x, _fake(48, 31))),
        (ValueError, lambda: fb.linear(x, _fake(48, 2, 16))),
        (ValueError, lambda: fb.linear(x, w, _fake(32))),
        (ValueError, lambda: fb.linear(x, w, _fake(48, 2)[:, 0])),
        (ValueError, lambda: fb.linear(x, w, residual=_fake(4, 6, 32))),
        (ValueError, lambda: fb.linear(x, w, residual=_fake(24, 48, dtype="float32"))),
        (ValueError, lambda: fb.linear(x, w, out=_fake(24, 47))),
        (ValueError, lambda: fb.linear(x, w, preact=_fake(24, 48, dtype="float32"))),
        (ValueError, lambda: fb.linear(x, w, out_dtype=7)),
        (ValueError, lambda: fb.linear(x.transpose(1, 2), _fake(48, 6))),
        (ValueError, lambda: fb.linear(_fake(1, 32).expand(5, 32), w)),                 # rows on top of one another
        (ValueError, lambda: fb.linear(_fake(4, 9, 32)[:, :6], w)),                     # rows at two distances
        (ValueError, lambda: fb.linear(_fake(), w)),
        (ValueError, lambda: fb.linear(x, _fake(48, 32, device="cuda:1"))),
        (ValueError, lambda: fb.linear_backward(_fake(24, 47), x, w)),
        (ValueError, lambda: fb.linear_backward(_fake(24, 48), x, w, preact=_fake(24, 48, dtype="float32"))),
        
    ]
    for error, call in calls:
        with pytest.raises(error):
            call()


def test_block_norm_refuses_tensors():
    x, y, v = _fake(4, 6, 32), _fake(4, 6, 32), _fake(32, dtype="float32")
    calls = [
        (ValueError, lambda: fb.block_norm(_fake(4, 32, device="cpu"))),
        (ValueError, lambda: fb.block_norm(x, _fake(4, 6, 31))),
        (ValueError, lambda: fb.block_norm(x, y, before_weight=v, before_bias=_fake(32))),  # parameters of two types
        (ValueError, lambda: fb.block_norm(x, y, before_weight=_fake(31, dtype="float32"))),
        (ValueError, lambda: fb.block_norm(x, y, gate=_fake(4, 31, dtype="float32"))),
        (ValueError, lambda: fb.block_norm(x, y, h=_fake(24, 32, dtype="float32"))),
        (ValueError, lambda: fb.block_norm(x, y, n=_fake(24, 31))),
        (ValueError, lambda: fb.block_norm_backward(None, _fake(24, 31), x, y)),
        (ValueError, lambda: fb.block_norm_backward(_fake(4, 6, 32, dtype="float32"), y, x, y)),
    ]
    for error, call in calls:
        with pytest.raises(error):
            call()


def test_linear_refuses_error_words():
    x, w, g = _fake(4, 6, 32), _fake(48, 32), _fake(24, 48)
    assert fb.lib().flashbev_linear_given_up(None) == fb.INVALID_ARG
    for word in (_fake(1, dtype="int32", device="cpu"), _fake(1, dtype="float32"), _fake(2, dtype="int32"), _fake(0, dtype="int32")):
        with pytest.raises(ValueError, match="error_word"):
            fb.linear(x, w, error_word=word)
        with pytest.raises(ValueError, match="error_word"):
            fb.linear_backward(g, x, w, error_word=word)
    with pytest.raises(TypeError):
        fb.linear(x, w, error_word=4096)


@pytest.mark.parametrize("C, gates, per, blocks", [(64, 0, 50000, 296), (4096, 0, 5000, 148), (2050, 0, 5000, 148), (2048, 0, 5000, 296),
                                                   (32, 18000, 5, 282), (256, 600, 5, 75), (256, 100, 50, 200), (32, 1000, 64, 1000), (4096, 40, 100, 120)])
def test_block_norm_backward_scratch_is_that_of_the_blocks_that_run_at_once(C, gates, per, blocks):
    """Partial sums of the norms' parameters, and of the gates where no team has one to itself: a row for each thread block.  Blocks of 512
    threads (more than 2048 channels) are one to an SM; many gates with few rows each are for teams, not blocks."""
    if fb.flashbev_block_norm_backward_workspace_bytes(norm_backward_params(C=2048, rows=1 << 20, gate=None, grad_gate=None)) != 4 * 296 * 2048 * 4:
        pytest.skip("not 148 SMs")
    rows = (gates or 1) * per
    over = dict(C=C, rows=rows, gate_groups=gates) if gates else dict(C=C, rows=rows, gate=None, grad_gate=None)
    need = fb.flashbev_block_norm_backward_workspace_bytes(norm_backward_params(**over))
    assert need in (4 * blocks * C * 4, 5 * blocks * C * 4), need / (4 * C * 4)
    assert (need == 4 * blocks * C * 4) == (gates == 0 or (C, gates) in ((32, 18000), (256, 600)))
