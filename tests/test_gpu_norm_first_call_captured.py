"""The first call of a process may be one that is captured: each layer norm and 8-bit checkpoint call, alone in a new process, captured into
a graph before it ever ran, gives what it gives outside."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys, torch
from paper_2609_09821_b200 import binding as B
g = torch.Generator("cuda").manual_seed(1)
rand = lambda *s: torch.randn(*s, device="cuda", generator=g)
M, N, Mo = {M}, 512, {Mo}
x, dy, A = rand(M, N).bfloat16(), rand(M, N).bfloat16(), rand(M, Mo).bfloat16()
gamma, beta, mean, rstd = rand(N), rand(N), rand(M), rand(M).abs() + 0.5
y, dx, dg, db, C = (torch.zeros_like(t) for t in (x, x, gamma, beta, rand(Mo, N)))
ck = B.Act8.empty(M, N)
ck.code.random_(0, 255, generator=g), ck.scale.random_(120, 130, generator=g)
status = torch.zeros(1, dtype=torch.int32, device="cuda")
ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
calls = dict(forward=lambda: B.layer_norm(x, gamma, beta, y, mean, rstd, relu=True), keep=lambda: B.layer_norm(x, gamma, beta, y, mean, rstd, relu=True, ckpt=ck),
             backward=lambda: B.layer_norm_backward(dy, gamma, beta, rstd, dx, dg, db, ws, relu=True, x=x, mean=mean),
             backward_kept=lambda: B.layer_norm_backward(dy, gamma, beta, rstd, dx, dg, db, ws, ckpt=ck), pack=lambda: B.act8_pack(x, ck),
             unpack=lambda: B.act8_unpack(ck, y, gamma, beta, True), product=lambda: B.gemm_act8_tn(A, ck, C, ws, status, gamma, beta, True))
outs = (y, dx, dg, db, C, ck.code, ck.scale)
call = calls["{call}"]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
graph.replay()
torch.cuda.synchronize()
first = [t.clone() for t in outs]
if "{call}" not in ("keep", "pack"):
    assert any(bool((t != 0).any()) for t in first[:5])
for t in (y, dx, dg, db, C):
    t.zero_()
call()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, outs)) and int(status) == 0
print("same")
"""


@pytest.mark.parametrize("call,M,Mo", [("forward", 700, 64), ("keep", 700, 64), ("backward", 8, 64), ("backward", 3000, 64), ("backward_kept", 700, 64), ("pack", 700, 64),
                                       ("unpack", 700, 64), ("product", 3000, 64), ("product", 3000, 128), ("product", 3000, 512)])
def test_first_call_is_captured(call, M, Mo):
    done = subprocess.run([sys.executable, "-c", PROGRAM.format(call=call, M=M, Mo=Mo)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]
