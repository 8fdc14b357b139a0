"""How many workgroups and launches calls of the training operators take, without a GPU (tests/hip_recorder.c in place of the HIP runtime)."""
import pytest

from test_training_abi import BF16, F32, record  # noqa: F401 (a fixture)


def launches(record, *calls):  # noqa: F811
    """Of each call the workgroups of its launches."""
    got = record([(name, dict(kw, **{n: kw["d"] for n in ("ldx", "lddy", "lddx") if n in FIELDS[name]})) for name, kw in calls])
    assert all(st == 0 for st, _ in got)
    return [[int(w[3]) for w in lines] for _, lines in got]


FIELDS = {"norm_grad": ("ldx", "lddy", "lddx"), "gate_grad": ("ldx", "lddx")}


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_gradient_without_sums_fills_the_device(record, dtype):  # noqa: F811
    """dx alone: one group of rows per workgroup up to the compute units, however few workgroups the sums would be left to."""
    none = dict(dgamma=None, dbeta=None, ws=None, nb=0, dtype=dtype)
    got = launches(record, *[("norm_grad", dict(T=T, d=d, **none)) for T, d in ((256, 1024), (64, 2048), (8, 4096), (4, 16384), (1 << 20, 1024))])
    assert got == [[32], [16], [4], [4], [256]]
