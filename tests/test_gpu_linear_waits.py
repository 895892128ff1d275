"""Matrix products whose waits run out: in the checked build (-DFLASHBEV_DEBUG_BOUNDS) the limits of the waits come from the
environment, one for each of the three roles of a thread block (loads, products, results).  With short ones an ordinary product
gives up somewhere on its way, with loads and products of its own still going on; it has to see them done, give its memory back,
count itself, and leave everything around it as it was."""
import ctypes

import pytest

from paper_2607_10071_b200 import binding as fb
from paper_2607_10071_b200 import build as fbuild

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
LONG = 4_000_000_000
ROLES = ("loads", "products", "results")
LIMITS = (0, 100, 300, 600, 1000, 1500, 2200, 3500, 6000, 12000, 40000)

# rows, K, N, operands, result, activation, z kept, residual
CALLS = dict(one_block=(100, 64, 64, BF16, BF16, fb.ACT_NONE, False, False),      # the loads have all been issued when the first wait begins
             a_ring=(700, 4096, 520, BF16, BF16, fb.ACT_GELU, True, True),        # shared sums, more blocks than stages
             kept_weights=(40000, 128, 256, BF16, BF16, fb.ACT_NONE, False, False),
             several_tiles=(40000, 200, 264, BF16, F32, fb.ACT_SILU, False, True),
             running_sums=(20000, 1000, 256, BF16, F32, fb.ACT_NONE, False, False),
             one_accumulator=(1300, 40000, 2000, BF16, BF16, fb.ACT_NONE, False, False),
             pieces=(20000, 130, 200, F32, F32, fb.ACT_RELU, True, False),
             pieces_running_sums=(20000, 520, 128, F32, F32, fb.ACT_NONE, False, False))


@pytest.fixture(scope="module")
def checked():
    return fb.load_library(fbuild.build(debug_bounds=True))


class Call:
    def __init__(self, library, rows, K, N, dtype, out_dtype, act, keep, residual):
        gen = torch.Generator(device="cuda").manual_seed(rows + K + N)

        def draw(*shape, dtype=dtype, scale=1.0):
            return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

        self.library = library
        self.x, self.w, self.b = draw(rows, K), draw(N, K, scale=K ** -0.5), draw(N)
        self.r = draw(rows, N, dtype=out_dtype) if residual else None
        # rows of 7 behind the last ones
        self.out = torch.full((rows + 40, N), 7.0, dtype=out_dtype, device="cuda")
        self.z = torch.full((rows + 40, N), 7.0, dtype=dtype, device="cuda") if keep else None
        self.word = torch.zeros(1, dtype=torch.int32, device="cuda")
        p = self.p = fb.LinearParams()
        p.struct_size = ctypes.sizeof(p)
        p.x, p.weight, p.bias, p.out, p.error_word = (t.data_ptr() for t in (self.x, self.w, self.b, self.out, self.word))
        p.residual = self.r.data_ptr() if residual else None
        p.preact_out = self.z.data_ptr() if keep else None
        p.rows, p.in_features, p.out_features, p.act = rows, K, N, act
        p.dtype, p.out_dtype = (fb.F32 if t is F32 else fb.BF16 for t in (dtype, out_dtype))
        need = library.flashbev_linear_workspace_bytes(ctypes.byref(p))
        self.scratch = torch.zeros(max(1, need), dtype=torch.uint8, device="cuda")
        p.workspace, p.workspace_bytes = (self.scratch.data_ptr(), need) if need else (None, 0)

    def run(self):
        """How many thread blocks gave up"""
        self.word.zero_()
        assert self.library.flashbev_linear(ctypes.byref(self.p), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == fb.OK
        torch.cuda.synchronize()
        rows = self.p.rows
        assert bool((self.out[rows:] == 7).all()) and (self.z is None or bool((self.z[rows:] == 7).all()))
        return int(self.word)

    def results(self):
        return [t[:self.p.rows].clone() for t in (self.out, self.z) if t is not None]


@pytest.mark.parametrize("name", CALLS)
def test_waits_that_run_out(checked, monkeypatch, name):
    call = Call(checked, *CALLS[name])
    assert call.run() == 0
    want = call.results()
    assert all(bool(t.isfinite().all()) for t in want)
    gave_up = {}
    for role in range(3):
        for limit in LIMITS:
            limits = [LONG] * 3
            limits[role] = limit
            monkeypatch.setenv("FLASHBEV_WAIT_CYCLES", ",".join(map(str, limits)))
            gave_up[ROLES[role], limit] = n = call.run()
            if not n:            # every wait ended in time: the numbers of any other call
                assert all(torch.equal(a, b) for a, b in zip(call.results(), want)), (ROLES[role], limit)
            monkeypatch.delenv("FLASHBEV_WAIT_CYCLES")
            assert call.run() == 0 and all(torch.equal(a, b) for a, b in zip(call.results(), want)), (ROLES[role], limit)
    # Nothing has arrived a cycle after the first wait for it began.  (The epilogue brings its bias before it waits, and a tile of 64 of K may have
    # been loaded and multiplied by then; sums of 1000 and more have not.)
    assert gave_up["products", 0] > 0, gave_up
    assert gave_up["results", 0] > 0 or CALLS[name][1] < 1000, gave_up
    monkeypatch.setenv("FLASHBEV_WAIT_CYCLES", "0,0,0")
    assert call.run() > 0


def test_gradients_whose_waits_run_out(checked, monkeypatch):
    """Both products of a backward call, and the same call again in time."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    rows, K, N = 6000, 264, 520
    g, x, w = (torch.randn(*s, generator=gen, device="cuda").to(BF16) for s in ((rows, N), (rows, K), (N, K)))
    grads = [torch.empty(s, dtype=BF16, device="cuda") for s in ((rows, K), (N, K), (N,))]
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    p = fb.LinearBackwardParams()
    p.struct_size = ctypes.sizeof(p)
    p.grad_out, p.x, p.weight, p.error_word = (t.data_ptr() for t in (g, x, w, word))
    p.grad_x, p.grad_weight, p.grad_bias = (t.data_ptr() for t in grads)
    p.rows, p.in_features, p.out_features, p.dtype, p.grad_dtype = rows, K, N, fb.BF16, fb.BF16
    need = checked.flashbev_linear_backward_workspace_bytes(ctypes.byref(p))
    scratch = torch.zeros(need, dtype=torch.uint8, device="cuda")
    p.workspace, p.workspace_bytes = scratch.data_ptr(), need

    def run():
        word.zero_()
        assert checked.flashbev_linear_backward(ctypes.byref(p), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == fb.OK
        torch.cuda.synchronize()
        return int(word)

    assert run() == 0
    want = [t.clone() for t in grads]
    for limits in ("0,0,0", f"{LONG},{LONG},700", f"{LONG},700,{LONG}", f"700,{LONG},{LONG}", "3000,3000,3000"):
        monkeypatch.setenv("FLASHBEV_WAIT_CYCLES", limits)
        n = run()
        assert n > 0 or limits != "0,0,0"
        if not n:
            assert all(torch.equal(a, b) for a, b in zip(grads, want))
        monkeypatch.delenv("FLASHBEV_WAIT_CYCLES")
        assert run() == 0 and all(torch.equal(a, b) for a, b in zip(grads, want)), limits


SCRIPT = """
import os, sys
import torch
sys.path.insert(0, sys.argv[1])
from paper_2607_10071_b200 import binding as fb
assert fb.LIB_PATH.startswith(sys.argv[1])
x, w, g = (torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in ((600, 1024), (96, 1024), (600, 96)))
words = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(4)]
good = fb.linear(x, w, error_word=words[0])
fb.linear_backward(g, x, w, error_word=words[1])
assert bool((good == 1024).all()) and fb.linear_given_up() == 0
os.environ["FLASHBEV_WAIT_CYCLES"] = "0,0,0"
fb.linear(x, w, error_word=words[2])
fb.linear_backward(g, x, w, error_word=words[3])
fb.linear(x, w)
torch.cuda.synchronize()
counts = [int(v) for v in words]
assert counts[:2] == [0, 0] and counts[2] > 0 and counts[3] > 0, counts
assert fb.linear_given_up() > sum(counts) and fb.linear_given_up(0) == fb.linear_given_up(x.device)
print("counted")
"""


def test_callers_with_tensors_learn_of_it(checked, tmp_path):
    """The package over the checked build instead of the ordinary one, in a process of its own."""
    import os
    import shutil
    import subprocess
    import sys
    package = os.path.dirname(os.path.abspath(fb.__file__))
    copy = tmp_path / os.path.basename(package)
    shutil.copytree(package, copy, ignore=shutil.ignore_patterns("csrc", "__pycache__", "libflashbev*.so"))
    shutil.copy(fbuild.LIB_DEBUG_BOUNDS, copy / "libflashbev.so")
    env = {k: v for k, v in os.environ.items() if k not in ("FLASHBEV_WAIT_CYCLES", "PYTHONPATH")}
    done = subprocess.run([sys.executable, "-c", SCRIPT, str(tmp_path)], env=env, cwd=tmp_path, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "counted" in done.stdout, done.stderr


def test_nothing_has_given_up():
    x, w = torch.ones(600, 96, dtype=BF16, device="cuda"), torch.ones(40, 96, dtype=BF16, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    fb.linear(x, w, error_word=word)
    fb.linear_backward(torch.ones(600, 40, dtype=BF16, device="cuda"), x, w, error_word=word)
    assert int(word) == 0 and fb.linear_given_up() == 0
