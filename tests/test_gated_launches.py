"""The launch that dx and the weights' gradients of the gated experts share, without a GPU (tests/hip_recorder.c in place of the HIP runtime)."""
import math
import os
import subprocess

import pytest

from test_gated_abi import BF16, P, record  # noqa: F401 (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# tiles and cost of dx, tiles and cost of the weights' gradients, workgroups an XCD
LAUNCHES = {
    "few long tiles beside many small ones": (224, 9.0, 24, 124.0, 64),             # 7001 rows, d = 80, F = 208, E = 4
    "one expert": (97, 7.0, 10, 100.0, 64),
    "more than a workgroup a compute unit": (193, 24.0, 102, 67.4, 64),              # 8183, 320, 680, 2
    "one a compute unit": (128, 67.0, 3000, 4.0, 32),
    "one tile of each": (1, 10.0, 1, 10.0, 32),
    "nothing": (0, 1.0, 0, 1.0, 64),
    "two workgroups": (100, 3.0, 100, 5.0, 2),
}


def rounds(tiles, groups):
    return math.ceil(tiles / (8 * groups))


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("share") / "pair_share")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2404_05019_amd", "csrc"), os.path.join(ROOT, "tests", "pair_share_main.cpp"),
                           "-o", exe])
    args = [str(v) for launch in LAUNCHES.values() for v in (*launch, 256)]
    return dict(zip(LAUNCHES, map(int, subprocess.check_output([exe, *args], text=True).split())))


@pytest.mark.parametrize("name", LAUNCHES)
def test_no_workgroup_is_left_idle_that_would_end_a_product_earlier(shares, name):
    """The slower product ends as early as it can; and no other share does that too, ends the other one earlier and has a compute unit for
    every workgroup."""
    n1, c1, n2, c2, resident = LAUNCHES[name]

    def times(s):
        return rounds(n1, s) * c1, rounds(n2, resident - s) * c2
    s = shares[name]
    assert 1 <= s < resident
    every = {q: times(q) for q in range(1, resident)}
    least = max(times(s))
    assert least == min(max(t) for t in every.values())
    for q, t in every.items():
        if max(t) == least and sum(t) < sum(times(s)):
            assert 8 * q + min(n2, 8 * (resident - q)) > 256, (q, s)


def test_small_tiles_are_spread(shares):
    """A round of 28 workgroups an XCD where one of three would do by the slower product; no more than there are compute units."""
    assert shares["few long tiles beside many small ones"] == 28
    assert shares["one expert"] == 13
    assert 8 * shares["more than a workgroup a compute unit"] + 102 <= 256


# rows, model width, hidden width, experts, and what the gradient takes in two launches and in one (us)
TWO = [(5003, 1000, 2728, 32, 445, 458), (8632, 544, 1592, 24, 228, 258), (18353, 576, 2248, 21, 432, 503), (3925, 1440, 5400, 13, 666, 753),
       (8660, 304, 848, 57, 126, 139), (5028, 1032, 1448, 16, 204, 230), (32768, 2048, 8192, 16, 5227, 5834), (843, 480, 1816, 30, 99, 108), (54, 624, 1736, 22, 88, 98),
       (396, 720, 1384, 20, 77, 83)]
ONE = [(2000, 768, 2048, 64, 314, 270), (8192, 768, 1536, 8, 158, 137), (1000, 1024, 2048, 32, 217, 190), (4096, 1536, 4096, 2, 361, 313),
       (2959, 848, 952, 32, 134, 119), (2008, 1216, 4320, 21, 398, 342), (8192, 384, 1536, 8, 112, 101), (1068, 376, 760, 42, 56, 53),
       (1479, 344, 784, 43, 69, 60), (2205, 576, 2232, 16, 142, 128), (744, 1336, 2408, 9, 169, 153), (7001, 80, 208, 4, 33, 28)]


@pytest.mark.parametrize("rows,d,F,E,two,one", TWO + ONE)
def test_dx_shares_a_launch_with_the_weights_gradients_where_that_is_faster(record, rows, d, F, E, two, one):  # noqa: F811
    (st, lines), = record([("grad", dict(rows=rows, d=d, F=F, E=E, dtype=BF16, dx=2 * P))])
    assert st == 0 and len(lines) == (2 if one < two else 3)
    assert any("gated_pair_kernel" in w[2] for w in lines) == (one < two)
