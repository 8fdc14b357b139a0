"""What the compiler gave the kernels, from the metadata of the built library: without a GPU."""
import os
import re
import shutil
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2404_05019_amd", "libscmoe.so")
READELF = shutil.which("llvm-readelf") or os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """Bytes of scratch memory per lane of every kernel."""
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    data = open(LIB, "rb").read()
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    kernels = {}
    for found in re.finditer(re.escape(magic), data):
        start = found.start()
        at = start + len(magic)
        (n,) = struct.unpack_from("<Q", data, at)
        at += 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, at)
            name = data[at + 24:at + 24 + length]
            at += 24 + length
            if b"gfx950" not in name:
                continue
            path = tmp_path_factory.mktemp("object") / "code.o"
            path.write_bytes(data[start + offset:start + offset + size])
            notes = subprocess.check_output([READELF, "--notes", str(path)], text=True)
            names, sizes = re.findall(r"^ +\.symbol: +(\S+)\.kd$", notes, re.M), re.findall(r"\.private_segment_fixed_size: (\d+)", notes)
            assert len(names) == len(sizes)
            kernels.update({k: int(v) for k, v in zip(names, sizes)})
    return kernels


@pytest.mark.parametrize("kernel", ["gate_backward_kernel", "combine_backward_kernel", "balance_loss_kernel", "sum_parts_kernel", "layer_norm_kernel",
                                    "layer_norm_backward_kernel"])
def test_training_kernels_fit_their_registers(scratch, kernel):
    """A register that goes to memory and back waits for the loads that are kept in flight."""
    of = {k: v for k, v in scratch.items() if kernel in k}
    assert of
    assert not {k: v for k, v in of.items() if v}
