"""Rules of the 8-bit projections' sources, read from them."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_24899_b200", "csrc")


def _text(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_no_failed_cuda_call_leaves_its_error_behind():
    """Calls of the C ABI that give up because one of CUDA's has failed say so through `failed`, which takes the pending error away."""
    for name in ("fp8_norm.cu", "fp8_matmul.cu"):
        text = _text(name)
        assert "failed()" in text and "AS_ERR_CUDA" not in text, name
