"""How exact the gated experts and their gradient are as a whole, segment by segment, beside the bounds on every element of
tests/test_gated_ops.py, which let pass whatever is small next to a sum of magnitudes.

Relative error in the 2-norm.  Rounding a value with k bits behind the first is off by a uniform 2^-(k+1) of its power of two, 2^-(k+1) / sqrt 3 in the
mean square; relative to values spread evenly over a power of two's logarithm sqrt((1 - 1/4) / (2 ln 2)) = 0.74 of that: 0.425 times the largest, RMS
below.
  bf16   what goes to the second products is rounded once and their results once; the errors are independent and sums of random signs keep their
         relative size: sqrt 2 RMS 2^-8 = 2.35e-3.  A quarter more for outputs of few elements.
  fp32   in a sum of n random products, taken in any order, every one of n partial sums, which grow as the root of their number, is rounded: RMS 2^-24 sqrt(n / 2)
         in one chain, less in several.  Two sums behind one another of up to 4104: 1.6e-6.  A quarter more."""
import math

import pytest
import torch

from test_gated_abi import BF16, F32, FULL, NOTHING, P, record  # noqa: F401 (a fixture)
from test_gated_ops import ACTS, FORMS, NAN, Block, backward64, check_backward, check_forward, forward64, restored

RMS = 0.425
MOST = {"bf16": 1.25 * math.sqrt(2.0) * RMS * 2.0 ** -8, "f32": 1.25 * math.sqrt(2.0) * RMS * 2.0 ** -24 * math.sqrt(4104 / 2)}


def off(got, want):
    want = want.double()
    return float((got.double() - want).norm() / want.norm())


def exact_enough(got, want, dtype):
    if want.numel() >= 512:
        assert off(got, want) <= MOST[dtype], off(got, want)


def forward_is_exact(b):
    for e, at in b.segments():
        if at.stop > at.start:
            exact_enough(b.y[at], forward64(b.x[at], b.W1[e], b.W2[e], b.act, b.dtype)[0], b.dtype)


def backward_is_exact(b, x, pre):
    for e, at in b.segments():
        if at.stop > at.start:
            want = backward64(b.dy[at], x[at], pre[at], b.W1[e], b.W2[e], b.act, b.dtype)
            for got, w in zip((b.dx[at], b.dW1[e], b.dW2[e]), want):
                exact_enough(got, w, b.dtype)


# ---- what the measure tells apart, without a GPU --------------------------------------------------------


def planted(dtype, fault):
    """Gradients of rows computed in 64 bits with the roundings of the type, and one mistake."""
    g = torch.Generator()
    g.manual_seed(1)
    n, d, F = 70, 136, 520
    normal = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    W1, W2 = normal(2 * F, d) * d ** -0.5, normal(d, F) * F ** -0.5
    x, dy, pre = normal(n, d), normal(n, d), normal(n, 2 * F)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W1, W2, x, dy, pre = (t.to(tt).double() for t in (W1, W2, x, dy, pre))
    rounded = lambda t: t.to(tt).double()  # noqa: E731
    u, gate = pre[:, F:], pre[:, :F]
    p = torch.sigmoid(gate)
    slope = p + (0.9 if fault == "slope" else 1.0) * p * gate * (1 - p)
    dh = dy @ W2
    both = rounded(torch.cat([dh * u * slope, dh * gate * p], 1))
    h = rounded(gate * p * u)
    if fault == "8 bits":
        both = both.float().to(torch.float8_e4m3fn).double()
    if fault == "bf16":
        both, h = both.bfloat16().double(), h.bfloat16().double()
    dx = rounded(both @ W1) * (1.03 if fault == "scaled" else 1.0)
    dW1 = both.t() @ x
    if fault == "a row left out":
        dW1 = both[1:].t() @ x[1:]
    want = backward64(dy, x, pre, W1, W2, "silu", dtype)
    return [off(got, w) for got, w in zip((dx, rounded(dW1), rounded(dy.t() @ h)), want)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_roundings_of_the_type_pass(dtype):
    assert max(planted(dtype, "")) <= MOST[dtype]


@pytest.mark.parametrize("dtype,fault", [("bf16", "slope"), ("bf16", "8 bits"), ("bf16", "scaled"), ("bf16", "a row left out"), ("f32", "bf16"), ("f32", "slope")])
def test_a_mistake_does_not(dtype, fault):
    assert max(planted(dtype, fault)) > MOST[dtype]


# ---- every form of the kernels, with every activation ---------------------------------------------------


@pytest.mark.gpu
@pytest.mark.parametrize("keep", ["full", "8bit"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("form", FORMS)
def test_forms_of_the_kernels(form, act, keep):
    from paper_2404_05019_amd import binding as B
    counts, d, F, dtype = FORMS[form]
    b = Block(counts, d, F, dtype, act, seed=30)
    kept, x = (b.pre, b.x) if keep == "full" else (b.pre8, b.x8)
    b.forward(pre=kept)
    check_forward(b, keep)
    forward_is_exact(b)
    if keep == "8bit":
        B.scmoe_checkpoint_pack(b.x, b.x8, n_rows=b.offsets[-1:])
    b.backward(x, kept)
    if keep == "8bit":
        x, kept = restored(x[:b.K], b.K, d), restored(kept[:2 * b.K], 2 * b.K, F).reshape(b.K, 2 * F)
    check_backward(b, x, kept)
    backward_is_exact(b, x, kept)
    b.y.fill_(NAN)
    b.forward()
    forward_is_exact(b)


# ---- few rows: every turn of the loop over k --------------------------------------------------------------

# A turn of the kernel for few rows is 4096 bytes of a row in the first product, 8192 in the second: widths that end with one, just behind one, and
# behind the second
TURNS = {"bf16": [(2048, 4096), (2056, 4104), (4104, 8200)], "f32": [(1024, 2048), (1032, 2056), (2056, 4104)]}
FEW = [[1], [2], [3], [4], [0, 3, 0, 0, 1, 0]]
WIDE = [(dtype, d, F) for dtype, sizes in TURNS.items() for d, F in sizes]


def test_the_kernel_for_few_rows_takes_them(record):  # noqa: F811
    """Both products, and the widths are on either side of one turn and of two."""
    calls = []
    for dtype, d, F in WIDE:
        bytes_ = 2 if dtype == "bf16" else 4
        assert (d * bytes_ - 1) // 4096 == (F * bytes_ - 1) // 8192 == TURNS[dtype].index((d, F))
        for counts in FEW:
            kw = dict(rows=sum(counts), E=len(counts), d=d, F=F, dtype=BF16 if dtype == "bf16" else F32)
            calls += [("ffn", dict(kw, keep=k, pre=P if k else None, ws=P, nb=1 << 40)) for k in (NOTHING, FULL)]
    for call, (st, lines) in zip(calls, record(calls)):
        assert st == 0 and len(lines) == 2 and all("gated_few_kernel" in w[2] for w in lines), (call, lines)


@pytest.mark.gpu
@pytest.mark.parametrize("counts", FEW)
@pytest.mark.parametrize("dtype,d,F", WIDE)
def test_turns_of_the_kernel_for_few_rows(dtype, d, F, counts):
    for act in ACTS:
        b = Block(counts, d, F, dtype, act, spare=0, seed=31)
        b.forward(pre=b.pre)
        check_forward(b)
        forward_is_exact(b)
        b.untouched(b.pre)
        want = b.y.clone()
        b.y.fill_(NAN)
        b.forward()
        b.untouched(b.y)
        assert torch.equal(b.y, want)
