"""The operators of a transformer block, each captured into a graph by its very first call in a process."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import sys
sys.path[:0] = [%r, %r]
import torch
from paper_2609_10018_gb300 import binding
which = sys.argv[1]
st = torch.zeros(1, dtype=torch.int32, device="cuda")
if which.startswith("prefix"):
    from test_gpu_prefix_attention import Case
    n = 1 if which == "prefix_token" else 30
    c = Case([(300, 2)], [n] * 2, [n + 40, n]).device()
    args = c.args()
    run = lambda h: binding.elasto_op_prefix_attention(h, args, st.data_ptr())
    check = lambda: c.check(c.out.cpu())
elif which == "rope":
    from test_gpu_qk_norm_rope_axes import Case, AXIS, runs
    c = Case(40, 4, 4, 64, runs(8, 16, 8), AXIS)
    d = c.device()
    run = lambda h: binding.elasto_op_qk_norm_rope_axes(h, c.args(d), st.data_ptr())
    check = lambda: c.near(d["q_out"], c.want()[0])
else:
    from test_gpu_residual_norm import Case
    c = Case(40, 777 if which == "any" else 776, y_scale=True)
    d = c.device()
    run = lambda h: binding.elasto_op_residual_norm(h, c.args(d), st.data_ptr())
    check = lambda: c.check(d)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run(torch.cuda.current_stream().cuda_stream)
graph.replay()
torch.cuda.synchronize()
check()
assert int(st.item()) == 0
""" % (HERE, os.path.dirname(HERE))


@pytest.mark.parametrize("which", ["prefix_token", "prefix_prompt", "rope", "norm", "any"])
def test_first_call_is_captured(which):
    r = subprocess.run([sys.executable, "-c", PROGRAM, which], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
