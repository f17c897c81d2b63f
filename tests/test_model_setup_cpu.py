"""What a model's first call sets up. CPU only: reads the source, since the setup itself needs a GPU."""
import os
import re

from paper_2609_10018_gb300 import build


def test_models_set_up_only_their_own_kernels():
    """A kernel of the calls for long sequences that cannot be set up (its register count is checked) must not refuse
    elasto_create: their setup runs when they are first called."""
    with open(os.path.join(build.CSRC, "api.cu")) as f:
        text = f.read()
    body = text[text.index("cudaError_t ensure_kernel_attributes() {"):]
    calls = re.findall(r"(\w+)_init_attributes\(\)", body[:body.index("\n}\n")])
    assert calls == ["gemm", "halo", "attn", "cnn", "head", "pk"]
