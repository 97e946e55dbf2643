"""The CUDA-core head kernel at hidden sizes whose masked rows come close to 48 KB of shared memory, where a launch
needs a raised limit: 8 rows of d fp32 or bf16 elements next to the kernel's own arrays.  The calls run in a process
of their own, smallest size first, because a limit that an earlier call raised stays raised."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

CALLS = """
import torch
import paper_2603_03333_b200 as pk
from paper_2603_03333_b200 import binding

def grid(shape, std, unit, dtype, seed):      # every fp32 sum of products is exact
    g = torch.Generator(device="cuda:0"); g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda:0").mul_(std / unit).round_().clamp_(-255, 255) * unit).to(dtype)

for d, dtype in ((1512, torch.float32), (1520, torch.float32), (1536, torch.float32), (1544, torch.float32),
                 (3032, torch.bfloat16), (3040, torch.bfloat16), (3064, torch.bfloat16), (3080, torch.bfloat16)):
    W, H = grid((500, d), d ** -0.5, 2.0 ** -10, dtype, 1), grid((9, d), d ** -0.5, 2.0 ** -10, dtype, 2)
    best = (H.double() @ W.double().T).argmax(1).to(torch.int32).view(3, 3)
    ctx = pk.Context(0)
    ctx.set_head(W, max_rows=18)
    ctx.enable_score(9, 1)
    out = ctx.verify_batched(H.view(3, 3, d), best, 2, 0.0, 5)
    assert ctx.last_impl() == binding.IMPL_SIMT
    assert torch.equal(out["tokens"], best[..., None].expand(3, 3, 2)), d
    assert (out["accept_len"] == 3).all(), d
    assert torch.equal(ctx.score(H, None, n_top=1)["top_ids"][:, 0], best.view(-1)), d
    out = binding.verify_batched_static(W, H.view(3, 3, d), best, 2, 0.0, 5)
    assert torch.equal(out["tokens"], best[..., None].expand(3, 3, 2)), d
    assert ctx.device_error() == 0
    ctx.close()
print("every size ran")
"""


def test_sizes_around_the_default_limit_of_shared_memory():
    done = subprocess.run([sys.executable, "-c", CALLS], cwd=Path(__file__).resolve().parent.parent, capture_output=True,
                          text=True, timeout=300)
    assert done.returncode == 0 and "every size ran" in done.stdout, done.stderr[-2000:]
