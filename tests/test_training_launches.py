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


def test_norm_gradient_of_few_rows(record):  # noqa: F811
    """Both sides of the rules: rows that one workgroup takes, parts that the last one adds up, and a second launch for them."""
    want = {
        (1, 64): [1], (128, 64): [1], (129, 64): [5], (1024, 64): [32], (1025, 64): [33, 8],      # (32 rows a workgroup in fp32)
        (32, 512): [1], (33, 512): [5], (128, 512): [16], (129, 512): [17, 64],
        (16, 520): [1], (17, 520): [3, 65], (16, 1024): [1], (17, 1024): [3, 128], (256, 1024): [32, 128], (8, 2048): [1], (9, 2048): [3, 256],
        (4, 4096): [1], (5, 4096): [3, 512], (2, 8192): [1], (3, 8192): [3, 1024],
        (1, 8200): [1], (2, 8200): [2, 1025], (1, 16384): [1], (2, 16384): [2, 2048],
    }
    assert dict(zip(want, launches(record, *[("norm_grad", dict(T=T, d=d)) for T, d in want]))) == want


def test_gate_gradient_of_few_tokens(record):  # noqa: F811
    """Both sides of the rule: parts that a column block's last workgroup adds up, and a second launch for them (64 tokens a part)."""
    bf16 = dict(dtype=BF16)
    want = [(dict(T=64, E=16), 1), (dict(T=512, E=8), 1), (dict(T=513, E=4), 2), (dict(T=512, E=9), 2), (dict(T=256, E=16), 1), (dict(T=257, E=16), 2),
            (dict(T=65, E=17), 2), (dict(T=512, E=4, **bf16), 1), (dict(T=513, E=4, **bf16), 2), (dict(T=256, E=8, **bf16), 1),
            (dict(T=257, E=8, **bf16), 2), (dict(T=65, E=9, **bf16), 2), (dict(T=64, E=64, **bf16), 1)]
    got = launches(record, *[("gate_grad", dict(kw, d=256)) for kw, _ in want])
    assert [len(lines) for lines in got] == [n for _, n in want]
