"""The Python binding without a GPU: what it needs of torch, and which tensors it refuses."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2404_05019_amd import binding as B

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


class OnGpu:
    """A host tensor that says it lies on a GPU: nothing that is called here reads it."""

    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index


class Library:
    """Takes every call and keeps its name."""

    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        return lambda *a: self.called.append(name) or 0


@pytest.fixture
def library(monkeypatch):
    it = Library()
    monkeypatch.setattr(B, "lib", lambda: it)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    return it


T, D, E, K = 6, 64, 4, 2
SHAPES = dict(x=(T, D), dy=(T, D), dx=(T, D), base=(T, D), dbase=(T, D), y_perm=(9, D), dx_perm=(9, D), dy_perm=(9, D), W_g=(D, E), dW_g=(D, E),
              probs=(T, E), expert_idx=(T, K), dst_row=(T, K), gate_w=(T, K), dgate_w=(T, K), coef=(T, 2), dcoef=(T, 2), dbias=(E,), load=(E,),
              mean_prob=(E,), slope=(E,), loss=(1,), gamma=(D,), beta=(D,), mean=(T,), rstd=(T,), y=(T, D), dgamma=(D,), dbeta=(D,),
              residual=(T, D), sum_out=(T, D), dsum=(T, D), mask=(T,), dloss=(1,))
INTS = ("expert_idx", "dst_row", "load")
CALLS = {
    "scmoe_layer_norm": ("x", "gamma", "beta", "y", "residual", "sum_out", "mean", "rstd"),
    "scmoe_layer_norm_backward": ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "dsum"),
    "scmoe_balance_loss": ("probs", "expert_idx", "load", "mean_prob", "slope", "loss", "mask"),
    "scmoe_gate_backward": ("x", "W_g", "probs", "expert_idx", "gate_w", "dgate_w", "dx", "dW_g", "dbias", "slope", "dloss", "mask", "dx_perm", "dst_row"),
    "scmoe_combine_backward": ("dy", "y_perm", "dst_row", "gate_w", "dy_perm", "dgate_w", "base", "coef", "dbase", "dcoef"),
}


def call(name, **other):
    """The call with tensors that fit, but for `other`."""
    args = {n: OnGpu(torch.zeros(SHAPES[n], dtype=torch.int32 if n in INTS else torch.uint8 if n == "mask" else torch.float32)) for n in CALLS[name]}
    args.update(other)
    if name == "scmoe_layer_norm":
        args["eps"] = 1e-5
    if name == "scmoe_balance_loss":
        args["coef"] = 0.1
    if "expert_idx" in args or "dst_row" in args:
        args["k"] = K
    if name not in ("scmoe_layer_norm", "scmoe_combine_backward"):
        args["workspace"] = OnGpu(torch.zeros(64))
    getattr(B, name)(stream=0, **args)


TABLES = [(name, n) for name in CALLS for n in CALLS[name] if n in ("probs", "expert_idx", "dst_row", "gate_w", "dgate_w", "dW_g", "coef", "dcoef")
          and not (name == "scmoe_balance_loss" and n == "probs")]       # (its shape says how many tokens and experts there are)


@pytest.mark.parametrize("name,n", TABLES)
def test_a_transposed_table_is_refused(library, name, n):
    """As many elements in the other order, without gaps: the kernel would read them as other tokens'."""
    t = torch.zeros(SHAPES[n][::-1], dtype=torch.int32 if n in INTS else torch.float32)
    with pytest.raises(TypeError, match="expected"):
        call(name, **{n: OnGpu(t)})
    assert library.called == []
    # flat, or with the tokens in sequences, they lie as they should
    for shape in ((t.numel(),), (2, SHAPES[n][0] // 2, SHAPES[n][1])):
        call(name, **{n: OnGpu(t.reshape(shape))})
    assert library.called == [name] * 2


@pytest.mark.parametrize("name", CALLS)
def test_tensors_that_fit_are_taken(library, name):
    call(name)
    assert library.called == [name]


@pytest.mark.parametrize("name,n", [(name, n) for name in CALLS for n in CALLS[name]])
def test_a_tensor_on_another_gpu_is_refused(library, name, n):
    """The kernel runs on one GPU, and on another one's memory at best by its grace."""
    other = OnGpu(torch.zeros(SHAPES[n], dtype=torch.int32 if n in INTS else torch.uint8 if n == "mask" else torch.float32), 1)
    with pytest.raises(TypeError, match="on the GPU"):
        call(name, **{n: other})
    assert library.called == []


def test_the_gpu_of_a_call_is_its_stream_s(library, monkeypatch):
    """The current one, or the one of the stream that is given."""
    class Stream:
        cuda_stream, device_index = 5, 1
    x0, x1 = (OnGpu(torch.zeros(T, D), i) for i in (0, 1))
    monkeypatch.setattr(B, "_current_stream", lambda device: 0)
    B.scmoe_layer_norm(x0, None, None, 1e-5, x0)
    B.scmoe_layer_norm(x1, None, None, 1e-5, x1, stream=Stream)
    for x, stream in ((x1, None), (x0, Stream)):
        with pytest.raises(TypeError, match="on the GPU"):
            B.scmoe_layer_norm(x, None, None, 1e-5, x, stream=stream)
    assert len(library.called) == 2
