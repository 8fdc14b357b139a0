"""Which kernels the sizes of tests/test_gated_ops.py take, without a GPU (tests/hip_recorder.c in place of the HIP runtime): between them every
form is run there; and none of them spills registers."""
import re

import pytest

from test_gated_abi import BF16, EIGHT, F32, FULL, NOTHING, P, record  # noqa: F401 (a fixture)
from test_gated_ops import FORMS
from test_kernel_resources import scratch  # noqa: F401 (a fixture)

GATE, DOWN, DH, DX, DW = range(5)


def kernels(lines):
    """(mode, how it is kept, type, tile) of the block's own kernels, (type, tiles of DX and of DW with their stages) of those that have both
    gradients; the others by name."""
    got = []
    for w in lines:
        m = re.search(r"gated_pair_kernelINS_9GatedPairINS_8GatedCfgILb(\d)ELi(\d+)ELi\d+ELi\dELi\dELi(\d).*?EE(S3_|NS2_ILb\dELi(\d+)ELi\d+ELi\dELi\dELi(\d))", w[2])
        if m:
            x = (int(m[2]), int(m[3]))
            got.append(("f32" if m[1] == "1" else "bf16", x, x if m[4] == "S3_" else (int(m[5]), int(m[6]))))
            continue
        m = re.search(r"gated_kernel.*GatedCfgILb(\d)ELi(\d+)ELi(\d+)E.*?EELi(\d)ELi(\d)ELi\d", w[2])
        got.append((int(m[4]), int(m[5]), "f32" if m[1] == "1" else "bf16", (int(m[2]), int(m[3]))) if m else re.search(r"[a-z_0-9]+_kernel|gemm_bf16_kernel|zero_ints", w[2])[0])
    return got


def calls(rows, E, d, F, dtype):
    kw = dict(rows=rows, E=E, d=d, F=F, dtype=BF16 if dtype == "bf16" else F32)
    for keep in (NOTHING, FULL, EIGHT):
        yield "ffn", dict(kw, keep=keep, pre=P if keep else None)
    for keep in (FULL, EIGHT):
        yield "grad", dict(kw, xk=keep, pk=keep, dx=2 * P)
    yield "grad", dict(kw, dx=None)
    yield "grad", dict(kw, dW1=None, dW2=None)


def test_every_form_is_run(record):  # noqa: F811
    taken = {}
    for form, (counts, d, F, dtype) in FORMS.items():
        asked = list(calls(sum(counts) + 3, len(counts), d, F, dtype))
        for _, (st, lines) in zip(asked, record(asked)):
            assert st == 0
            for k in kernels(lines):
                if isinstance(k, tuple):
                    taken.setdefault(k, set()).add(form)
    T256, T256_128, T128, T64 = (256, 256), (256, 128), (128, 128), (64, 64)
    want = [(DW, NOTHING, "bf16", t) for t in (T256, T128)] + [(DX, NOTHING, "bf16", t) for t in (T256, T256_128, T128, T64)]
    want += [(DOWN, NOTHING, "bf16", t) for t in (T256, T256_128, T128, T64)]
    want += [(GATE, k, "bf16", t) for k in (NOTHING, FULL, EIGHT) for t in (T256, T128, T64)] + [(DH, k, "bf16", t) for k in (FULL, EIGHT) for t in (T256, T128, T64)]
    for t in (T128, T64):
        want += [(m, NOTHING, "f32", t) for m in (DOWN, DX, DW)] + [(GATE, k, "f32", t) for k in (NOTHING, FULL, EIGHT)] + [(DH, k, "f32", t) for k in (FULL, EIGHT)]
    want += [("bf16", t, w) for t, w in (((256, 2), (256, 2)), ((128, 2), (128, 2)), ((64, 3), (128, 2)))] + [("f32", (64, n), (64, 2)) for n in (2, 3)]
    assert not [k for k in want if k not in taken], sorted(map(str, taken.items()))
    assert set(taken) == set(want)


@pytest.mark.parametrize("kernel", ["gated_kernel", "gated_pair_kernel", "gated_few_kernel", "checkpoint_kernel"])
def test_the_kernels_fit_their_registers(scratch, kernel):  # noqa: F811
    """A register that goes to memory and back waits for the copies that are kept in flight."""
    of = {k: v for k, v in scratch.items() if kernel in k}
    assert of
    assert not {k: v for k, v in of.items() if v}
