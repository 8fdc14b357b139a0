"""The activations of the gated feed-forward block and their slopes relative to themselves, far below zero too, in every form of the kernels
that has them (one for each activation).

Weights of ones and zeros hand a call's values through exactly: g is a column of x and u is 1, y and dx are what was rounded on store.  So
one rounding to the type is allowed (STORE) beside the error of the formula, which is counted in H = 2^-24 relative to its terms:
  p = 1 / (1 + e^-t)   e^-t of a t that is off by up to 8 H |t| (its products, the factor log2 e), which moves p by p (1 - p) of that; the
                       exponential, the sum, the reciprocal: 8 H of p
  Phi                  fp32: the library's erfc (16 H) of an argument off by 2 H, which moves it by (g^2 + |g|) of that; bf16:
                       tests/normal_cdf_error_main.cpp on the host, and the hardware's exponential and reciprocal: 4 H
  e^(-g^2/2)           8 H, and 4 H g^2 for its argument
Numbers below LEAST = 2^-126 may be lost: p and Phi by as much, so act(g) = g p by |g| times that, and the slope by 1 + |g| times its inner
factor (GELU, tanh, g = -10.06: p = 0.19 LEAST, and 0.19 * 233 LEAST are missing from the slope); beside that the stored values themselves, FLOOR."""
import math
import os
import subprocess

import pytest
import torch

from test_gated_abi import BF16, EIGHT, F32, FULL, NOTHING, P, record  # noqa: F401 (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
H = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STORE = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
LEAST, FLOOR = 2.0 ** -126, 2.0 ** -118
ACTS = {"silu": 2, "gelu": 0, "gelu_tanh": 1}
# the relative error of Phi in bf16 from where on (below -13 it underflows)
CDF = ((-13.0, 7.6e-5), (-2.0, 2.9e-5), (-1.0, 8.4e-6), (0.0, 7.0e-6))


def test_error_of_the_distribution_function(tmp_path):
    exe = str(tmp_path / "normal_cdf_error")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-I", os.path.join(ROOT, "paper_2404_05019_amd", "csrc"),
                           os.path.join(ROOT, "tests", "normal_cdf_error_main.cpp"), "-o", exe])
    lines = [line.split() for line in subprocess.check_output([exe], text=True).splitlines()]
    for lo, hi, off in ((float(w[1]), float(w[2]), float(w[3])) for w in lines if w[0] == "max"):
        assert off <= [e for at, e in CDF if lo >= at][-1], (lo, hi, off)
    # e: its argument is off by 2 roundings of up to g^2 / 2 each
    assert [float(w[1]) for w in lines if w[0] == "e"][0] <= 1.0
    assert ["least", "0"] in lines
    assert lines[-1] == "special 1 0 0 0 0 1 1".split()


# ---- which kernels the sizes take ----------------------------------------------------------------------

# rows and hidden width (the model width is twice that) by type: the kernel for few rows and 64 x 64 tiles, and the larger ones
SIZES = {"bf16": [(3, 64), (200, 64), (2047, 1024), (4095, 1024), (8191, 1024)], "f32": [(3, 64), (200, 64), (8191, 2048)]}
SPARE = 3


def test_every_form_of_every_activation_is_run(record):  # noqa: F811
    """Of the first product, and of the hidden rows' gradient."""
    import re
    want, got = set(), set()
    for act in ACTS.values():
        for f32, tiles in (("0", ("256", "128", "64")), ("1", ("128", "64"))):
            want |= {(f32, t, "0", str(k), str(act)) for t in tiles for k in (NOTHING, FULL, EIGHT)}
            want |= {(f32, t, "2", str(k), str(act)) for t in tiles for k in (FULL, EIGHT)}
            want.add((f32, "few", "0", str(act)))
    calls = []
    for dtype, sizes in SIZES.items():
        for rows, F in sizes:
            for act in ACTS.values():
                kw = dict(rows=rows + SPARE if rows > 4 else rows, E=1, d=2 * F, F=F, dtype=BF16 if dtype == "bf16" else F32, act=act)
                calls += [("ffn", dict(kw, keep=k, pre=P if k else None)) for k in (NOTHING, FULL, EIGHT)]
                calls += [("grad", dict(kw, pk=k, dx=2 * P, dW1=None)) for k in (FULL, EIGHT)]
    for _, (st, lines) in zip(calls, record(calls)):
        assert st == 0
        for w in lines:
            m = re.search(r"gated_kernel.*GatedCfgILb(\d)ELi(\d+)E.*?EELi([02])ELi(\d)ELi(\d)", w[2])
            if m:
                got.add(m.groups())
            m = re.search(r"gated_few_kernelILb(\d)ELb1ELi(\d)", w[2])
            if m:
                got.add((m[1], "few", "0", m[2]))
    assert got == want, (sorted(want - got), sorted(got - want))


# ---- on the GPU ----------------------------------------------------------------------------------------


def act64(g, act, dtype):
    """Activation and slope in 64 bits, and bounds on their errors for an exact argument."""
    x = g.abs()
    if act == "gelu":
        p = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))
        phi = torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        if dtype == "f32":
            off = 16 * H + 2 * H * (g * g + x)
        else:
            off = torch.full_like(g, CDF[0][1])
            for at, e in CDF[1:]:
                off[g >= at] = e
            off = off + 4 * H
        return g * p, p + g * phi, x * (off * p + LEAST), off * p + x * phi * (8 + 4 * g * g) * H + (1 + x) * LEAST
    c, b = (1.0, 0.0) if act == "silu" else (2 * math.sqrt(2 / math.pi), 0.044715)
    t, inner = c * (g + b * g ** 3), c * (1 + 3 * b * g * g)
    p, q = torch.sigmoid(t), torch.sigmoid(-t)
    off = (8 * H + 8 * H * t.abs() * q) * p + LEAST
    return g * p, p + g * p * q * inner, x * off, off * (1 + x * inner) + 8 * H * (p + x * p * q * inner)


def near(got, want, slack, dtype):
    got = got.double()
    most = STORE[dtype] * (want.abs() + slack) + slack + FLOOR
    off = (got - want).abs()
    assert bool((off <= most).all()), "worst %.3g times the bound" % float((off / most).nan_to_num(1e9).max())


class Through:
    """Rows of g over [-14, 9] and what hands them through: d = 2 F."""

    def __init__(self, rows, F, dtype, act):
        from paper_2404_05019_amd import binding as B
        self.B, self.F, self.d, self.dtype, self.act = B, F, 2 * F, dtype, act
        dev, tt = "cuda:0", TYPES[dtype]
        gen = torch.Generator(device=dev)
        gen.manual_seed(rows + F)
        self.n, self.rows = rows, rows + SPARE if rows > 4 else rows
        self.offsets = torch.tensor([0, rows], dtype=torch.int32, device=dev)
        self.new = lambda *s, dtype=tt: torch.zeros(s, dtype=dtype, device=dev)
        self.g = (torch.rand(self.rows, F, generator=gen, device=dev) * 23 - 14).to(tt)
        self.g[0, :8] = torch.tensor([-4.0, -4.25, -4.5, -5.0, -13.0, 0.0, -0.0, 1e-3], device=dev).to(tt)
        self.u = torch.randn(self.rows, F, generator=gen, device=dev).to(tt)
        self.dh = torch.randn(self.rows, F, generator=gen, device=dev).to(tt)
        self.W2 = self.new(1, 2 * F, F)
        self.W2[0, :F] = torch.eye(F, device=dev)

    def forward(self, pre=None):
        x, W1, F = self.new(self.rows, self.d), self.new(1, self.d, self.d), self.F
        x[:, :F], x[:, F] = self.g, 1.0
        W1[0, :F, :F] = torch.eye(F, device=x.device)
        W1[0, F:, F] = 1.0                                       # u = 1
        y = self.new(self.rows, self.d)
        self.B.scmoe_gated_ffn(x, self.offsets, self.rows, W1, self.W2, self.new(self.rows, F), y, ACTS[self.act], pre=pre)
        return y

    def backward(self, pre):
        """(dg, du) and the hidden rows of the first F rows."""
        F = self.F
        W1, dy, dx, dW2 = self.new(1, self.d, self.d), self.new(self.rows, self.d), self.new(self.rows, self.d), self.new(1, self.d, F)
        W1[0] = torch.eye(self.d, device=dy.device)
        dy[:, :F] = self.dh
        few = min(self.n, F)
        dy[torch.arange(few), F + torch.arange(few)] = 1.0       # (W2 has zeros there) dW2[F + r] = h[r]
        need = self.B.scmoe_gated_ffn_backward_workspace_bytes(self.B.dtype_code(dy), self.rows, 1, self.d, F)
        self.B.scmoe_gated_ffn_backward(dy, None, pre, self.offsets, self.rows, W1, self.W2, ACTS[self.act], dx, None, dW2,
                                        workspace=self.new(need, dtype=torch.uint8))
        return dx[:, :F], dx[:, F:], dW2[0, F:F + few]

    def packed(self, pre):
        q = self.new(2 * self.rows, self.B.scmoe_checkpoint_ld(self.F), dtype=torch.uint8)
        self.B.scmoe_checkpoint_pack(pre.reshape(2 * self.rows, self.F), q)
        return q


CASES = [(dtype, *size) for dtype, sizes in SIZES.items() for size in sizes]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,rows,F", CASES)
def test_activations(dtype, rows, F, act):
    t = Through(rows, F, dtype, act)
    want, _, slack, _ = act64(t.g[:rows].double(), act, dtype)
    full, eight = t.new(t.rows, 2 * F), t.new(2 * t.rows, t.B.scmoe_checkpoint_ld(F), dtype=torch.uint8)
    for pre in (None, full, eight):
        y = t.forward(pre)
        near(y[:rows, :F], want, slack, dtype)
        assert bool((y[:, F:] == 0).all()) and bool((y[rows:] == 0).all())
    ones = torch.cat([t.g + 0.0, torch.ones_like(t.g)], 1)       # (the sum of -0 and the other products, 0, is 0)
    assert torch.equal(full[:rows], ones[:rows]) and bool((full[rows:] == 0).all())
    blocks = F + -(-F // 32)
    assert torch.equal(eight[:2 * rows, :blocks], t.packed(ones)[:2 * rows, :blocks]) and bool((eight[2 * rows:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("keep", ["full", "8bit"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,rows,F", CASES)
def test_slopes(dtype, rows, F, act, keep):
    t = Through(rows, F, dtype, act)
    pre = torch.cat([t.g, t.u], 1)
    g, u = t.g[:rows].double(), t.u[:rows].double()
    if keep == "8bit":
        pre = t.packed(pre)
        back = t.new(2 * t.rows, F, dtype=torch.float32)
        t.B.scmoe_checkpoint_unpack(pre, back)
        g, u = (v[:rows].double() for v in back.reshape(t.rows, 2 * F).split(F, 1))
    dh = t.dh[:rows].double()
    a, s, ea, es = act64(g, act, dtype)
    dg, du, h = t.backward(pre)
    near(du[:rows], dh * a, dh.abs() * (ea + 2 * H * a.abs()), dtype)
    near(dg[:rows], dh * u * s, (dh * u).abs() * (es + 4 * H * s.abs()), dtype)
    few = h.shape[0]
    near(h, (a * u)[:few], (u.abs() * (ea + 2 * H * a.abs()))[:few], dtype)
    assert bool((dg[rows:] == 0).all()) and bool((du[rows:] == 0).all())
