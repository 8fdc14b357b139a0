"""The Python binding without a GPU: what it needs of torch, and which tensors it refuses."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_import_without_gpu_support_in_torch():
    """A torch built without GPUs has no handles of streams: the module loads, and a call for the stream says what is missing."""
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2404_05019_amd import binding as B
assert B.scmoe_capacity(64, 4, 1, 1.0) == 16
class Stream:
    cuda_stream = 77
torch.cuda.current_stream = lambda: Stream
assert B._stream(None) == 77 and B._stream(Stream) == 77 and B._stream(5) == 5
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
