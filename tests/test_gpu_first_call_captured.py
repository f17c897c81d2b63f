"""The calls for long sequences, each captured into a graph by its very first call in a process."""
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
from test_gpu_window_attention import Case
which = sys.argv[1]
st = torch.zeros(1, dtype=torch.int32, device="cuda")
if which == "gemm":
    a = torch.full((300, 128), 0x38, dtype=torch.uint8, device="cuda")  # ones
    s, out = torch.ones((3, 300), device="cuda"), torch.zeros((300, 300), device="cuda")
    run = lambda h: binding.elasto_op_gemm_fp8(h, a.data_ptr(), 128, s.data_ptr(), 300, a.data_ptr(), 128, s.data_ptr(), None,
                                               out.data_ptr(), 300, 300, 300, 128, binding.EPI_BIAS_F32, st.data_ptr())
    check = lambda: bool((out == 128.0).all())
else:
    c = Case([150], [200]) if which == "attention" else Case([1], [200], packed=False)
    c.device()
    run = lambda h: binding.elasto_op_window_attention(h, c.args(), st.data_ptr())
    check = lambda: c.check(c.out.cpu()) is None
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run(torch.cuda.current_stream().cuda_stream)
graph.replay()
torch.cuda.synchronize()
assert check() and int(st.item()) == 0
""" % (HERE, os.path.dirname(HERE))


@pytest.mark.parametrize("which", ["gemm", "attention", "token"])
def test_first_call_is_captured(which):
    r = subprocess.run([sys.executable, "-c", PROGRAM, which], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
