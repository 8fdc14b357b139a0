"""Which kernel the products of the gated experts take for few rows, without a GPU (tests/hip_recorder.c in place of the HIP runtime)."""
import pytest

from test_gated_abi import BF16, F32, P, record  # noqa: F401 (a fixture)

# type, rows, model width, hidden width, experts, and what a forward call takes with the other kernels, with the kernel for few rows in the first product alone, in the
# second alone, and in both (us)
CALLS = [("bf16", 8, 2048, 8192, 16, 147.2, 126.0, 142.5, 120.7), ("bf16", 16, 2048, 8192, 32, 263.0, 237.1, 256.3, 217.9), ("bf16", 40, 2048, 8192, 8, 160.9, 190.8, 198.5, 228.4),
         ("bf16", 5, 512, 2048, 4, 16.9, 16.0, 16.0, 15.5), ("bf16", 40, 512, 2048, 8, 17.2, 30.1, 20.7, 34.3), ("bf16", 64, 256, 1024, 64, 21.1, 35.6, 24.6, 40.0),
         ("bf16", 96, 512, 512, 64, 21.5, 28.0, 37.3, 44.1), ("bf16", 64, 1024, 4096, 64, 169.8, 205.8, 170.4, 207.7), ("bf16", 200, 256, 1024, 200, 45.6, 129.6, 66.9, 150.6),
         ("f32", 5, 1024, 4096, 1, 89.4, 78.5, 30.7, 18.0), ("f32", 16, 1024, 4096, 8, 128.6, 111.4, 89.6, 71.5), ("f32", 40, 1024, 4096, 8, 137.8, 133.3, 114.4, 110.1),
         ("f32", 20, 256, 1024, 4, 30.9, 30.2, 17.4, 16.6), ("f32", 64, 2048, 2048, 32, 322.7, 273.1, 303.5, 252.1), ("f32", 80, 2048, 8192, 16, 732.9, 820.1, 831.1, 924.2),
         ("f32", 320, 256, 1024, 64, 64.1, 100.4, 73.5, 110.4), ("f32", 1000, 1024, 1024, 200, 622.0, 646.2, 851.3, 872.4)]


@pytest.mark.parametrize("dtype,rows,d,F,E,others,first,second,both", CALLS)
def test_the_kernel_for_few_rows_is_taken_where_it_is_faster(record, dtype, rows, d, F, E, others, first, second, both):  # noqa: F811
    """Within a seventh of the fastest."""
    (st, lines), = record([("ffn", dict(rows=rows, d=d, F=F, E=E, dtype=BF16 if dtype == "bf16" else F32, ws=P, nb=1 << 40))])
    assert st == 0
    names = [w[2] for w in lines]
    taken = (others, first, second, both)[("gated_few" in names[0]) + 2 * ("gated_few" in names[-1])]
    assert taken <= 1.15 * min(others, first, second, both), names


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 4])
@pytest.mark.parametrize("d,F,E", [(8, 8, 1), (64, 256, 64), (2048, 8192, 16)])
def test_no_more_rows_than_its_tile_has_take_it(record, dtype, rows, d, F, E):  # noqa: F811
    (st, lines), = record([("ffn", dict(rows=rows, d=d, F=F, E=E, dtype=BF16 if dtype == "bf16" else F32))])
    assert st == 0 and len(lines) == 2 and all("gated_few" in w[2] for w in lines)
