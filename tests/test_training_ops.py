"""Layer norm, balance loss and the gradients of gate, encode and decode against the same formulas in 64 bits.

Tolerances count roundings, element by element: H = 2^-24 for every fp32 operation on the way to a value, times the sum of the
magnitudes that are added up (so a value that cancels is not asked for more than its terms carry), and one rounding
to the stored type (bf16: 2^-8 of the value).  The longest ways: 32 values in a lane, 6 steps across a wave, up to 8 waves,
one or two operations ahead of the sum: under 64.  Sums over tokens: the tokens of a wave's turns, the waves, the parts: under
256 at these sizes.  The tokens' gradient in bf16 is made from matrix operands of two bf16 parts each, which keep
2^-16 of their product twice and leave out their smallest product: 4 * 2^-16 of the terms."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2404_05019_amd import binding as B
    from gpu_util import DEV

H = 2.0 ** -24
NAN = float("nan")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STORE = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, scale=1.0, dtype="f32"):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(TYPES[dtype])


def padded(t, pad=8, fill=NAN):
    """The same values in rows `pad` elements longer, with `fill` between them."""
    store = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    store[:, :t.shape[1]] = t
    return store[:, :t.shape[1]]


def empty(T, d, dtype, pad=0):
    return torch.full((T, d + pad), NAN, dtype=TYPES[dtype], device=DEV)[:, :d]


def close(got, want, slack, dtype="f32"):
    """|got - want| <= one rounding to the type of |want| + slack, everywhere; non-finite values the same."""
    got, want = got.double(), want.double()
    off = (got - want).abs()
    most = STORE[dtype] * want.abs() + slack + 1e-38
    same = (got == want) | (got.isnan() & want.isnan())
    ok = same | (off <= most)
    assert bool(ok.all()), "%d of %d differ; worst %.3g times the bound" % (int((~ok).sum()), ok.numel(), float((off / most)[~ok].nan_to_num(1e9).max()))


def workspace(n):
    """Workspace full of NaN with a guard behind it."""
    w = torch.full((n // 4 + 64,), NAN, dtype=torch.float32, device=DEV)
    return w[:max(n // 4, 4)], w


# ---- layer norm -----------------------------------------------------------------------------------


def norm_ref(h, gamma, beta, eps):
    """y, mean, rstd and the slack of y in 64 bits."""
    h = h.double()
    mean = h.mean(1, keepdim=True)
    c = h - mean
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    g = torch.ones(h.shape[1], dtype=torch.float64, device=DEV) if gamma is None else gamma.double()
    b = torch.zeros(h.shape[1], dtype=torch.float64, device=DEV) if beta is None else beta.double()
    y = c * rstd * g + b
    slack = 64 * H * ((c * rstd * g).abs() + b.abs() + h.abs().mean(1, keepdim=True) * rstd * g.abs())
    return y, mean[:, 0], rstd[:, 0], slack


NORM_SHAPES = [(1, 8), (1, 2048), (2, 72), (3, 16384), (5, 136), (64, 2048), (37, 512), (33, 520), (130, 1000), (129, 2056), (66, 4104),
               (19, 8200), (4099, 64), (2500, 384)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", NORM_SHAPES)
def test_layer_norm(T, d, dtype):
    g = gen(T + d)
    x, r = padded(normal(g, T, d, dtype=dtype) + 3), padded(normal(g, T, d, dtype=dtype), 16)
    gamma, beta = normal(g, d), normal(g, d)
    y, s = empty(T, d, dtype, 24), empty(T, d, dtype, 8)
    mean, rstd = normal(g, T), normal(g, T)
    B.scmoe_layer_norm(x, gamma, beta, 1e-5, y, residual=r, sum_out=s, mean=mean, rstd=rstd)
    assert torch.equal(s, (x.float() + r.float()).to(TYPES[dtype]))
    wy, wm, wr, slack = norm_ref(s, gamma, beta, 1e-5)
    close(y, wy, slack, dtype)
    close(mean, wm, 64 * H * s.double().abs().mean(1))
    close(rstd, wr, 64 * H * wr)
    # without the residual, the affine part and the statistics
    y2 = empty(T, d, dtype)
    B.scmoe_layer_norm(x, None, None, 0.1, y2)
    wy, _, _, slack = norm_ref(x, None, None, 0.1)
    close(y2, wy, slack, dtype)
    # a row's bits do not depend on the others; every write stays in its rows
    y1 = empty(1, d, dtype)
    B.scmoe_layer_norm(x[T - 1:], None, None, 0.1, y1)
    assert torch.equal(y1[0], y2[T - 1])
    for v in (y, s):
        assert bool(v.as_strided((T, v.stride(0) - d), (v.stride(0), 1), d)[:T - 1].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm_of_extreme_rows(dtype):
    """A mean far above the deviation, a constant row, the largest values, a NaN and an infinity: each stays in its row."""
    g = gen(0)
    x = normal(g, 8, 256, dtype=dtype)
    x[1] = (normal(g, 256) + 4096.0).to(x.dtype)
    x[2] = 5.0
    x[3] *= 1e-30
    x[4, 17] = NAN
    x[5, 255] = float("inf")
    x[6, 3] = 1e15
    y = empty(8, 256, dtype)
    mean, rstd = torch.zeros(8, device=DEV), torch.zeros(8, device=DEV)
    B.scmoe_layer_norm(x, None, None, 1e-5, y, mean=mean, rstd=rstd)
    wy, wm, wr, slack = norm_ref(x, None, None, 1e-5)
    fine = [0, 1, 2, 3, 6, 7]
    close(y[fine], wy[fine], slack[fine], dtype)
    assert bool(y[4].isnan().all()) and bool(y[5].isnan().all()) and bool(mean[4].isnan()) and float(mean[5]) == float("inf")
    assert bool((y[2] == 0).all())


@pytest.mark.parametrize("T,d", [(1, 64), (130, 1000), (70, 4104), (9, 16384)])
def test_layer_norm_in_place(T, d):
    g = gen(5)
    for dtype in TYPES:
        x, r, gamma = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype), normal(g, d)
        y, s = empty(T, d, dtype), empty(T, d, dtype)
        B.scmoe_layer_norm(x, gamma, None, 1e-5, y, residual=r, sum_out=s)
        a, b = x.clone(), r.clone()
        B.scmoe_layer_norm(a, gamma, None, 1e-5, b, residual=b, sum_out=a)
        assert torch.equal(a, s) and torch.equal(b, y)
        # the backward pass over its own inputs
        mean, rstd = torch.zeros(T, device=DEV), torch.ones(T, device=DEV)
        dx = empty(T, d, dtype)
        B.scmoe_layer_norm_backward(y, x, gamma, mean, rstd, dx, dsum=r)
        for which in range(3):
            bufs = [y.clone(), x.clone(), r.clone()]
            B.scmoe_layer_norm_backward(bufs[0], bufs[1], gamma, mean, rstd, bufs[which], dsum=bufs[2])
            assert torch.equal(bufs[which], dx), which


def norm_grad_ref(dy, x, gamma, mean, rstd, dsum):
    """dx, dgamma, dbeta and their slacks."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    g = torch.ones(x.shape[1], dtype=torch.float64, device=DEV) if gamma is None else gamma.double()
    xh = (x - mean) * rstd
    gy = dy * g
    dx = rstd * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
    slack = 64 * H * rstd * (gy.abs() + gy.abs().mean(1, keepdim=True) + xh.abs() * (gy * xh).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx = dx + dsum.double()
        slack = slack + H * dsum.double().abs()
    return dx, slack, (dy * xh).sum(0), 256 * H * (dy * xh).abs().sum(0), dy.sum(0), 256 * H * dy.abs().sum(0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", NORM_SHAPES)
def test_layer_norm_backward(T, d, dtype):
    g = gen(T * 7 + d)
    x, dy, dsum = (padded(normal(g, T, d, dtype=dtype), p) for p in (8, 16, 24))
    gamma = normal(g, d)
    mean, rstd = 0.1 * normal(g, T), 0.5 + torch.rand(T, generator=g, device=DEV)
    need = B.scmoe_layer_norm_backward_workspace_bytes(T, d)
    ws, whole = workspace(need)
    for with_sum in (True, False):
        dx, dgamma, dbeta = empty(T, d, dtype, 8), torch.full((d,), NAN, device=DEV), torch.full((d,), NAN, device=DEV)
        s, ga = (dsum, gamma) if with_sum else (None, None)
        B.scmoe_layer_norm_backward(dy, x, ga, mean, rstd, dx, dgamma, dbeta, ws, dsum=s)
        wx, sx, wg, sg, wb, sb = norm_grad_ref(dy, x, ga, mean, rstd, s)
        close(dx, wx, sx, dtype)
        close(dgamma, wg, sg)
        close(dbeta, wb, sb)
        assert bool(whole[need // 4:].isnan().all()) and bool(dx.as_strided((T, 8), (d + 8, 1), d)[:T - 1].isnan().all())
        # the same bits again, and each result without the others
        dx2, dgamma2, dbeta2 = empty(T, d, dtype), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
        B.scmoe_layer_norm_backward(dy, x, ga, mean, rstd, dx2, dgamma2, None, ws, dsum=s)
        B.scmoe_layer_norm_backward(dy, x, ga, mean, rstd, dx2, None, dbeta2, ws, dsum=s)
        assert torch.equal(dx, dx2) and torch.equal(dgamma, dgamma2) and torch.equal(dbeta, dbeta2)
        B.scmoe_layer_norm_backward(dy, x, ga, mean, rstd, dx2, dsum=s)
        assert torch.equal(dx, dx2)


def test_layer_norm_of_no_rows():
    e = torch.zeros((0, 64), device=DEV)
    v, dgamma, dbeta = torch.zeros(0, device=DEV), torch.full((64,), NAN, device=DEV), torch.full((64,), NAN, device=DEV)
    B.scmoe_layer_norm(e, None, None, 1e-5, e)
    B.scmoe_layer_norm_backward(e, e, None, v, v, e, dgamma, dbeta)
    assert bool((dgamma == 0).all()) and bool((dbeta == 0).all())


# ---- balance loss and gate ------------------------------------------------------------------------


def routing(g, T, E, k, normalize):
    p = torch.softmax(2 * normal(g, T, E), 1)
    w, at = p.topk(k, 1)
    return p, at.to(torch.int32).contiguous(), (w / w.sum(1, keepdim=True) if normalize else w).contiguous()


def spoil(mask, *tensors):
    """NaN, infinities and the lowest value in what belongs to tokens that the mask leaves out."""
    out = (mask == 0).nonzero().flatten()
    for t in tensors:
        for i, v in enumerate((NAN, float("inf"), -float("inf"), torch.finfo(t.dtype).min)):
            t[out[i::4]] = v


@pytest.mark.parametrize("kind", ["all", "some", "one", "none"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 4), (7, 3, 2), (300, 8, 1), (1000, 17, 3), (4097, 33, 2), (20001, 64, 4), (30000, 2, 1),
                                   (5000, 48, 1)])
def test_balance_loss(T, E, k, kind):
    g = gen(T + E + k)
    p, idx, _ = routing(g, T, E, k, 0)
    idx[torch.rand((T, k), generator=g, device=DEV) < 0.03] = -1
    idx[torch.rand((T, k), generator=g, device=DEV) < 0.03] = E
    mask = None
    if kind != "all":
        mask = torch.rand(T, generator=g, device=DEV) < 0.6 if kind == "some" else torch.zeros(T, dtype=torch.bool, device=DEV)
        if kind == "one":
            mask[T // 2] = True
    use = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask
    n = int(use.sum())
    load = torch.stack([((idx == e) & use[:, None]).sum() for e in range(E)])
    mean = (p[use].double().sum(0) / n) if n else torch.zeros(E, dtype=torch.float64, device=DEV)
    share = load.double() / (k * n) if n else torch.zeros(E, dtype=torch.float64, device=DEV)
    if mask is not None:
        spoil(mask, p)
        idx[~mask] = 0
    out = [torch.full((E,), -7, dtype=torch.int32, device=DEV)] + [torch.full((m,), NAN, device=DEV) for m in (E, E, 1)]
    ws, whole = workspace(B.scmoe_balance_loss_workspace_bytes(T, E))
    B.scmoe_balance_loss(p, idx, k, 0.25, *out, ws, mask=mask)
    assert torch.equal(out[0].long(), load)
    close(out[1], mean, 256 * H * mean)
    slope = 0.25 * E * share / max(n, 1)
    close(out[2], slope, 16 * H * slope)
    close(out[3], (0.25 * E * (share * mean).sum()).reshape(1), 320 * H * 0.25 * E * (share * mean).sum())
    assert bool(whole[ws.numel():].isnan().all())
    again = [o.clone() for o in out]
    B.scmoe_balance_loss(p, idx, k, 0.25, *out, ws, mask=None if mask is None else mask.to(torch.uint8) * 3)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


def gate_grad_ref(x, Wg, p, idx, w, dw, normalize, slope, dloss, mask, dxp, dst):
    """dx, dW_g, dbias in 64 bits with the sums of magnitudes behind each."""
    T, E = p.shape
    p64, W = p.double(), Wg.double()
    on = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask.bool()
    p64 = torch.where(on[:, None], p64, 0.0)
    g = torch.zeros_like(p64)
    if slope is not None:
        g += slope.double() * (1.0 if dloss is None else dloss.double())
    own, own_size = torch.zeros_like(p64), torch.zeros_like(p64)
    if dw is not None:
        keep = (idx >= 0) & (idx < E)
        at = idx.long().clamp(0, E - 1)
        d64 = torch.where(keep, dw.double(), 0.0)
        if normalize:
            w64 = torch.where(keep, w.double(), 0.0)
            own.scatter_add_(1, at, w64 * (d64 - (w64 * d64).sum(1, keepdim=True)))
            own_size.scatter_add_(1, at, w64 * (d64.abs() + (w64 * d64).abs().sum(1, keepdim=True)))
        else:
            g.scatter_add_(1, at, d64)
    dl = torch.where(on[:, None], p64 * (g - (p64 * g).sum(1, keepdim=True)) + own, 0.0)
    size = torch.where(on[:, None], p64 * (g.abs() + (p64 * g).abs().sum(1, keepdim=True)) + own_size, 0.0)
    dx, sx = dl @ W.t(), size @ W.abs().t()
    more = torch.zeros_like(dx)
    if dst is not None:
        rows = dst.long().reshape(T, -1)
        add = torch.where((rows >= 0)[:, :, None], dxp[rows.clamp(min=0)].double(), 0.0)
        dx, more = dx + add.sum(1), add.abs().sum(1)
    x64 = torch.where(on[:, None], x.double(), 0.0)
    return dx, sx, more, x64.t() @ dl, x64.abs().t() @ size, dl.sum(0), size.sum(0)


def packed(g, T, E, k, idx, d, dtype, keep=0.7):
    """dst_row of a dispatch that kept some items, and a gradient for its rows (stride d + 8)."""
    kept = (torch.rand((T, k), generator=g, device=DEV) < keep) & (idx >= 0) & (idx < E)
    order = torch.randperm(T * k, generator=g, device=DEV).reshape(T, k)
    rank = torch.where(kept, order, T * k).reshape(-1).argsort().argsort().reshape(T, k)
    dst = torch.where(kept, rank, -1).to(torch.int32)
    return dst, padded(normal(g, max(1, int(kept.sum())), d, dtype=dtype))


def check_gate(T, d, E, k, dtype, normalize, seed, masked=True, loss=True, weights=True, encode=True, bias=True):
    g = gen(seed)
    x = padded(normal(g, T, d, dtype=dtype))
    Wg = normal(g, d, E, scale=0.2)
    p, idx, w = routing(g, T, E, k, normalize)
    idx[torch.rand((T, k), generator=g, device=DEV) < 0.03] = -1
    dw = normal(g, T, k) if weights else None
    slope = torch.rand(E, generator=g, device=DEV) if loss else None
    dloss = torch.full((1,), 0.7, device=DEV) if loss and seed % 2 else None
    mask = torch.rand(T, generator=g, device=DEV) < 0.7 if masked else None
    dst, dxp = packed(g, T, E, k, idx, d, dtype) if encode else (None, None)
    if masked:
        spoil(mask, x, p)
        if dw is not None:
            spoil(mask, dw, w)
    dx, dW, db = empty(T, d, dtype, 16), torch.full((d, E), NAN, device=DEV), torch.full((E,), NAN, device=DEV) if bias else None
    need = B.scmoe_gate_backward_workspace_bytes(T, d, E)
    ws, whole = workspace(need)
    call = lambda *o: B.scmoe_gate_backward(x, Wg, p, idx, w, dw, *o, ws, k=k, normalize=normalize, slope=slope, dloss=dloss,  # noqa: E731
                                            mask=mask, dx_perm=dxp, dst_row=dst)
    call(dx, dW, db)
    wx, sx, more, wW, sW, wb, sb = gate_grad_ref(x, Wg, p, idx, w, dw, normalize, slope, dloss, mask, dxp, dst)
    close(dx, wx, (128 * H + (4 * 2.0 ** -16 if dtype == "bf16" else 0.0)) * sx + 8 * H * more, dtype)
    close(dW, wW, 256 * H * sW)
    if bias:
        close(db, wb, 256 * H * sb)
    assert bool(whole[max(need // 4, 4):].isnan().all()) and bool(dx.as_strided((T, 16), (d + 16, 1), d)[:T - 1].isnan().all())
    dx2, dW2 = empty(T, d, dtype), torch.zeros(d, E, device=DEV)
    call(dx2, dW2, None)
    assert torch.equal(dx, dx2) and torch.equal(dW, dW2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,E,k", [(1, 8, 1, 1), (1, 2048, 16, 1), (15, 64, 2, 2), (17, 72, 3, 1), (63, 136, 16, 4), (65, 128, 17, 2),
                                     (256, 64, 4, 1), (333, 1000, 33, 3), (129, 2056, 64, 2), (2000, 264, 32, 2), (5000, 120, 8, 1),
                                     (31, 16, 48, 4), (700, 4096, 64, 1)])
def test_gate_backward(T, d, E, k, dtype):
    check_gate(T, d, E, k, dtype, 0, T + d)
    if k > 1:
        check_gate(T, d, E, k, dtype, 1, T + d + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E", [5, 24, 64])
def test_gate_backward_parts(E, dtype):
    """Each of its inputs left out."""
    check_gate(200, 192, E, 2, dtype, 0, 1, masked=False, weights=False, encode=False)
    check_gate(200, 192, E, 2, dtype, 1, 2, masked=False, loss=False)
    check_gate(200, 192, E, 2, dtype, 1, 3, weights=False, bias=False)
    check_gate(200, 192, E, 1, dtype, 0, 4, loss=False, encode=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gate_backward_with_nothing_counted(dtype):
    """Every token masked, every item dropped: zeros, whatever the inputs hold."""
    T, d, E = 70, 96, 6
    nan = torch.full((T, d), NAN, dtype=TYPES[dtype], device=DEV)
    p = torch.full((T, E), NAN, device=DEV)
    idx, dst = torch.full((T, 1), -1, dtype=torch.int32, device=DEV), torch.full((T, 1), -1, dtype=torch.int32, device=DEV)
    mask = torch.zeros(T, dtype=torch.uint8, device=DEV)
    dx, dW, db = empty(T, d, dtype), torch.full((d, E), NAN, device=DEV), torch.full((E,), NAN, device=DEV)
    ws, _ = workspace(B.scmoe_gate_backward_workspace_bytes(T, d, E))
    B.scmoe_gate_backward(nan, torch.ones(d, E, device=DEV), p, idx, p[:, :1].contiguous(), p[:, :1].contiguous(), dx, dW, db, ws, mask=mask,
                          slope=torch.ones(E, device=DEV), dx_perm=nan, dst_row=dst)
    for t in (dx, dW, db):
        assert bool((t == 0).all())
    # no token at all
    dW.fill_(NAN)
    db.fill_(NAN)
    B.scmoe_gate_backward(nan[:0], torch.ones(d, E, device=DEV), p[:0], idx[:0], p[:0, :1].contiguous(), p[:0, :1].contiguous(), dx[:0], dW, db, None)
    assert bool((dW == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gate_backward_keeps_non_finite_rows_apart(dtype):
    """A NaN in a token's row reaches its columns' sums and no other token's gradient."""
    T, d, E = 100, 256, 8
    g = gen(2)
    x, Wg = normal(g, T, d, dtype=dtype), normal(g, d, E)
    p, idx, w = routing(g, T, E, 1, 0)
    dw = normal(g, T, 1)
    ws, _ = workspace(B.scmoe_gate_backward_workspace_bytes(T, d, E))
    out = [(empty(T, d, dtype), torch.zeros(d, E, device=DEV), torch.zeros(E, device=DEV)) for _ in range(2)]
    B.scmoe_gate_backward(x, Wg, p, idx, w, dw, *out[0], ws)
    bad = x.clone()
    bad[41, 7] = NAN
    B.scmoe_gate_backward(bad, Wg, p, idx, w, dw, *out[1], ws)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][2], out[1][2])
    assert bool(out[1][1][7].isnan().all())
    rest = [i for i in range(d) if i != 7]
    assert torch.equal(out[0][1][rest], out[1][1][rest])
    p2 = p.clone()
    p2[13] = NAN
    B.scmoe_gate_backward(x, Wg, p2, idx, w, dw, *out[1], ws)
    keep = [t for t in range(T) if t != 13]
    assert bool(out[1][0][13].isnan().all()) and torch.equal(out[0][0][keep], out[1][0][keep])


# ---- decode ---------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cg", [False, True])
@pytest.mark.parametrize("T,d,k", [(1, 8, 1), (1, 2048, 4), (3, 72, 2), (64, 1000, 3), (2047, 520, 1), (2100, 136, 4), (5000, 64, 2), (40, 4104, 2),
                                   (2500, 2056, 1)])
def test_combine_backward(T, d, k, cg, dtype):
    g = gen(T + d + k)
    idx = torch.zeros((T, k), dtype=torch.int32, device=DEV)
    dst, yp = packed(g, T, 1, k, idx, d, dtype)
    dy = padded(normal(g, T, d, dtype=dtype), 16)
    w = torch.rand((T, k), generator=g, device=DEV)
    w[dst < 0] = NAN                                             # a dropped item's weight is not read into anything
    base = padded(normal(g, T, d, dtype=dtype)) if cg else None
    coef = torch.rand((T, 2), generator=g, device=DEV) if cg else None
    rows = yp.shape[0]
    dyp = empty(rows + 3, d, dtype, 8)
    dw = torch.full((T, k), NAN, device=DEV)
    dbase, dcoef = (empty(T, d, dtype, 8), torch.full((T, 2), NAN, device=DEV)) if cg else (None, None)
    B.scmoe_combine_backward(dy, yp, dst, w, k, dy_perm=dyp, dgate_w=dw, base=base, coef=coef, dbase=dbase, dcoef=dcoef)
    kept = dst >= 0
    r = dst.long().clamp(min=0)
    d64, w64 = dy.double(), torch.where(kept, w.double(), 0.0)
    c0, c1 = (coef[:, :1].double(), coef[:, 1:].double()) if cg else (1.0, torch.ones((T, 1), dtype=torch.float64, device=DEV))
    terms = torch.where(kept[:, :, None], yp[r].double(), 0.0) * d64[:, None, :]
    dots, size = terms.sum(2), terms.abs().sum(2)
    close(dw, c1 * dots, 128 * H * c1 * size)
    want = torch.full((rows + 3, d), NAN, dtype=torch.float64, device=DEV)
    want[dst[kept].long()] = ((c1 * w64)[:, :, None] * d64[:, None, :])[kept]
    close(dyp, want, 2 * H * want.abs().nan_to_num(0.0), dtype)
    if cg:
        close(dbase, c0 * d64, 0.0, dtype)
        dc0, dc1 = d64 * base.double(), w64 * dots
        close(dcoef, torch.stack([dc0.sum(1), dc1.sum(1)], 1), 140 * H * torch.stack([dc0.abs().sum(1), (w64 * size).sum(1)], 1))
    # each result alone, and in place
    dyp2, dw2 = empty(rows + 3, d, dtype), torch.zeros((T, k), device=DEV)
    B.scmoe_combine_backward(dy, None, dst, w, k, dy_perm=dyp2, coef=coef)
    B.scmoe_combine_backward(dy, yp, dst, w, k, dgate_w=dw2, coef=coef)
    assert torch.equal(dyp2.nan_to_num(9.0), dyp.nan_to_num(9.0)) and torch.equal(dw2, dw)
    over, over_base = yp.clone(), None if base is None else base.clone()
    B.scmoe_combine_backward(dy, over, dst, w, k, dy_perm=over, dgate_w=dw2, base=over_base, coef=coef, dbase=over_base, dcoef=dcoef)
    named = dst[kept].long()
    assert torch.equal(over[named], dyp[named]) and torch.equal(dw2, dw)
    if cg:
        assert torch.equal(over_base, dbase)


def test_combine_backward_with_nothing_kept():
    T, d = 50, 64
    dy, dst = torch.randn(T, d, device=DEV), torch.full((T, 2), -1, dtype=torch.int32, device=DEV)
    yp, dyp, dw = torch.full((1, d), NAN, device=DEV), torch.full((1, d), 7.0, device=DEV), torch.full((T, 2), NAN, device=DEV)
    B.scmoe_combine_backward(dy, yp, dst, torch.ones(T, 2, device=DEV), 2, dy_perm=dyp, dgate_w=dw)
    assert bool((dw == 0).all()) and bool((dyp == 7).all())
    B.scmoe_combine_backward(dy[:0], yp, dst[:0], torch.ones(0, 2, device=DEV), 2, dy_perm=dyp, dgate_w=dw[:0])


# ---- how a program uses them ------------------------------------------------------------------------


def test_gradients_against_differences():
    """fp32: a scalar of norm -> gate weights and loss -> decode in 64 bits, differentiated numerically, against the
    operators' gradients.  Central differences of step 1e-5 in 64 bits are off by about 1e-9 of the scale; the operators by some
    hundred roundings of 6e-8: 1e-4 of the largest gradient is asked."""
    T, d, E, k, coef = 9, 16, 5, 2, 0.3
    g = gen(11)
    x, Wg, gamma, beta = normal(g, T, d), normal(g, d, E, scale=0.5), 1 + 0.1 * normal(g, d), 0.1 * normal(g, d)
    experts = normal(g, E, d, d, scale=0.3).double()
    up = normal(g, T, d)
    y, mean, rstd = empty(T, d, "f32"), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    B.scmoe_layer_norm(x, gamma, beta, 1e-5, y, mean=mean, rstd=rstd)
    idx, w, p = torch.zeros((T, k), dtype=torch.int32, device=DEV), torch.zeros((T, k), device=DEV), torch.zeros((T, E), device=DEV)
    B.scmoe_gate_topk(y, Wg, None, k, idx, w, p, normalize=1)
    at = idx.long()

    def value(x_, Wg_, gamma_, beta_):
        m = x_.mean(1, keepdim=True)
        h = (x_ - m) / torch.sqrt(((x_ - m) ** 2).mean(1, keepdim=True) + 1e-5) * gamma_ + beta_
        logits = h @ Wg_
        probs = torch.softmax(logits, 1)
        weight = torch.softmax(logits.gather(1, at), 1)
        out = sum(weight[:, j:j + 1] * (experts[at[:, j]] @ h[:, :, None])[:, :, 0] for j in range(k))
        share = torch.bincount(at.reshape(-1), minlength=E).double() / (k * T)
        return (out * up.double()).sum() + 0.7 * coef * E * (share * probs.mean(0)).sum()

    leaves = [t.double() for t in (x, Wg, gamma, beta)]
    numeric = []
    for i, leaf in enumerate(leaves):
        n = torch.zeros_like(leaf)
        for j in range(leaf.numel()):
            side = []
            for step in (1e-5, -1e-5):
                moved = [v.clone() for v in leaves]
                moved[i].view(-1)[j] += step
                side.append(value(*moved))
            n.view(-1)[j] = (side[0] - side[1]) / 2e-5
        numeric.append(n)
    # the operators, backwards; an expert is a matrix here
    dst = torch.arange(T * k, dtype=torch.int32, device=DEV).reshape(T, k)
    yp = torch.stack([(experts[at[:, j]] @ y.double()[:, :, None])[:, :, 0] for j in range(k)], 1).reshape(T * k, d).float()
    dyp, dw = empty(T * k, d, "f32"), torch.zeros((T, k), device=DEV)
    B.scmoe_combine_backward(up, yp, dst, w, k, dy_perm=dyp, dgate_w=dw)
    dxp = torch.stack([(experts[at[:, j]].transpose(1, 2).contiguous() @ dyp.double().reshape(T, k, d)[:, j][:, :, None])[:, :, 0]
                       for j in range(k)], 1).reshape(T * k, d).float()
    load, mp, slope, loss = torch.zeros(E, dtype=torch.int32, device=DEV), torch.zeros(E, device=DEV), torch.zeros(E, device=DEV), torch.zeros(1, device=DEV)
    ws, _ = workspace(1 << 20)
    B.scmoe_balance_loss(p, idx, k, coef, load, mp, slope, loss, ws)
    dh, dWg, db = empty(T, d, "f32"), torch.zeros((d, E), device=DEV), torch.zeros(E, device=DEV)
    B.scmoe_gate_backward(y, Wg, p, idx, w, dw, dh, dWg, db, ws, k=k, normalize=1, slope=slope, dloss=torch.full((1,), 0.7, device=DEV),
                          dx_perm=dxp, dst_row=dst)
    dx, dgamma, dbeta = empty(T, d, "f32"), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    B.scmoe_layer_norm_backward(dh, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    for got, want in zip((dx, dWg, dgamma, dbeta), numeric):
        assert float((got.double() - want).abs().max() / want.abs().max()) < 1e-4


def _step(T, d, E, k, dtype, g):
    """Inputs, outputs and a function that runs all operators once on the current stream."""
    x, dy = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype)
    gamma, Wg = normal(g, d), normal(g, d, E)
    p, idx, w = routing(g, T, E, k, 1)
    dst, yp = packed(g, T, E, k, idx, d, dtype)
    mean, rstd = torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    y, dyp, dh, dx = empty(T, d, dtype), torch.zeros_like(yp), empty(T, d, dtype), empty(T, d, dtype)
    dw, dW, db = torch.zeros((T, k), device=DEV), torch.zeros((d, E), device=DEV), torch.zeros(E, device=DEV)
    dgamma, dbeta = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    load, mp, slope, loss = torch.zeros(E, dtype=torch.int32, device=DEV), torch.zeros(E, device=DEV), torch.zeros(E, device=DEV), torch.zeros(1, device=DEV)
    ws = torch.zeros(32 << 18, device=DEV)

    def run():
        B.scmoe_layer_norm(x, gamma, None, 1e-5, y, mean=mean, rstd=rstd)
        B.scmoe_balance_loss(p, idx, k, 0.01, load, mp, slope, loss, ws)
        B.scmoe_combine_backward(dy, yp, dst, w, k, dy_perm=dyp, dgate_w=dw)
        B.scmoe_gate_backward(y, Wg, p, idx, w, dw, dh, dW, db, ws, k=k, normalize=1, slope=slope, dx_perm=dyp, dst_row=dst)
        B.scmoe_layer_norm_backward(dh, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    return (x, dy, yp, w), (y, dyp, dh, dx, dw, dW, db, dgamma, dbeta, load, mp, slope, loss), run


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replays_give_the_eager_results(dtype):
    """One workspace for all of them on one stream, captured; inputs change between replays."""
    g = gen(1)
    ins, outs, run = _step(1500, 320, 12, 2, dtype, g)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        for t in ins:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV).abs() * (i + 1))
        for o in outs:
            o.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(-1)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_another_stream():
    g = gen(4)
    ins, outs, run = _step(900, 256, 8, 2, "bf16", g)
    run()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for o in outs:
        o.fill_(-1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Rows so far apart that their element offsets pass 2^32."""
    T, d, E, ld = 40, 64, 4, 1 << 27
    g = gen(6)
    store = torch.empty(T * ld, dtype=TYPES[dtype], device=DEV)
    far = lambda at: store.as_strided((T, d), (ld, 1), at)  # noqa: E731
    x, dy, xs, dys = far(0), far(1024), normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype)
    x.copy_(xs)
    dy.copy_(dys)
    gamma, Wg = normal(g, d), normal(g, d, E)
    p, idx, w = routing(g, T, E, 1, 0)
    dst = torch.arange(T, dtype=torch.int32, device=DEV).flip(0).reshape(T, 1).contiguous()
    ws = torch.zeros(1 << 20, device=DEV)

    def both(x, dy, place):
        y, dx, dyp, dh = (place(at) for at in (2048, 4096, 8192, 16384))
        mean, rstd, dw = torch.zeros(T, device=DEV), torch.zeros(T, device=DEV), torch.zeros((T, 1), device=DEV)
        dgamma, dbeta, dW, db = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV), torch.zeros((d, E), device=DEV), torch.zeros(E, device=DEV)
        B.scmoe_layer_norm(x, gamma, None, 1e-5, y, mean=mean, rstd=rstd)
        B.scmoe_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, dsum=y)
        B.scmoe_combine_backward(dy, x, dst, w, 1, dy_perm=dyp, dgate_w=dw)
        B.scmoe_gate_backward(x, Wg, p, idx, w, dw, dh, dW, db, ws, dx_perm=dyp, dst_row=dst)
        return [t.clone() for t in (y, dx, dyp, dh, mean, rstd, dw, dgamma, dbeta, dW, db)]
    near = both(xs, dys, lambda at: empty(T, d, dtype))
    assert all(torch.equal(a, b) for a, b in zip(near, both(x, dy, far)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_calls_in_graphs(dtype):
    """Calls whose sums over the tokens are finished by the last workgroup of their one launch, replayed over a workspace that other
    work has written to in between."""
    g = gen(9)
    T, d, E = 250, 136, 4
    x, dy, gamma, Wg = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype), normal(g, d), normal(g, d, E)
    p, idx, w = routing(g, T, E, 1, 0)
    mean, rstd, dw = normal(g, T), torch.rand(T, generator=g, device=DEV), normal(g, T, 1)
    big_p, big_idx, _ = routing(g, 9000, 24, 2, 0)
    dx, dh = empty(T, d, dtype), empty(T, d, dtype)
    sums = [torch.zeros(n, device=DEV) for n in (d, d, d * E, E, 24, 24, 1)]
    load = torch.zeros(24, dtype=torch.int32, device=DEV)
    ws = torch.full((1 << 18,), NAN, device=DEV)

    def run():
        B.scmoe_layer_norm_backward(dy, x, gamma, mean, rstd, dx, sums[0], sums[1], ws)
        B.scmoe_gate_backward(x, Wg, p, idx, w, dw, dh, sums[2].view(d, E), sums[3], ws)
        B.scmoe_balance_loss(big_p, big_idx, 2, 0.1, load, sums[4], sums[5], sums[6], ws)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in (dx, dh, load, *sums)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(5):
        for t in (dx, dh, load, *sums):
            t.fill_(-1)
        if i % 2:
            ws.copy_(torch.randn(ws.shape, generator=g, device=DEV))
        graph.replay()
        if i > 2:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (dx, dh, load, *sums)))
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (dx, dh, load, *sums)))


@pytest.mark.parametrize("T,d", [(1, 64), (8, 1024), (9, 1024), (32 * 8, 1024), (32 * 8 + 1, 1024), (64 * 8, 1024), (64 * 8 + 1, 1024), (255 * 8, 64),
                                 (2600, 64), (128 * 32, 64), (128 * 32 + 1, 64), (16, 4096), (17, 4096), (4, 16384), (5, 16384)])
def test_norm_gradient_sums_on_both_sides_of_their_rules(T, d):
    """One workgroup, one launch, one launch with more turns, two launches: dgamma and dbeta."""
    g = gen(T)
    x, dy, gamma, mean, rstd = normal(g, T, d), normal(g, T, d), normal(g, d), 0.1 * normal(g, T), 0.5 + torch.rand(T, generator=g, device=DEV)
    ws, whole = workspace(B.scmoe_layer_norm_backward_workspace_bytes(T, d))
    dx, dgamma, dbeta = empty(T, d, "f32"), torch.full((d + 1,), NAN, device=DEV)[1:], torch.full((d + 1,), NAN, device=DEV)[1:]
    B.scmoe_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    wx, sx, wg, sg, wb, sb = norm_grad_ref(dy, x, gamma, mean, rstd, None)
    close(dx, wx, sx)
    close(dgamma, wg, sg)
    close(dbeta, wb, sb)
    assert bool(whole[ws.numel():].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E", [(64, 4), (65, 4), (500, 8), (1100, 16), (300, 64), (4000, 32)])
def test_unaligned_probabilities_and_gate_matrix(T, E, dtype):
    """Rows that 16-byte loads could take but for where the tensors begin: the same bits as from aligned ones."""
    g = gen(T + E)
    d = 136
    x, Wg = normal(g, T, d, dtype=dtype), normal(g, d, E)
    p, idx, w = routing(g, T, E, 2, 1)
    dw, slope = normal(g, T, 2), normal(g, E)

    def shifted(t):
        store = torch.full((t.numel() + 1,), NAN, device=DEV)
        store[1:] = t.reshape(-1)
        return store[1:].view(t.shape)
    ws, _ = workspace(B.scmoe_gate_backward_workspace_bytes(T, d, E))
    out = []
    for f in (lambda t: t, shifted):
        dx, dW, db = empty(T, d, dtype), torch.full((d, E), NAN, device=DEV), torch.full((E,), NAN, device=DEV)
        B.scmoe_gate_backward(x, f(Wg), f(p), idx, f(w), f(dw), dx, f(dW), f(db), ws, k=2, normalize=1, slope=f(slope))
        dW, db = f(dW), f(db)
        B.scmoe_gate_backward(x, f(Wg), f(p), idx, f(w), f(dw), dx, dW, db, ws, k=2, normalize=1, slope=f(slope))
        load, m, s, loss = torch.zeros(E, dtype=torch.int32, device=DEV), f(torch.zeros(E, device=DEV)), f(torch.zeros(E, device=DEV)), f(torch.zeros(1, device=DEV))
        wl, _ = workspace(B.scmoe_balance_loss_workspace_bytes(T, E))
        B.scmoe_balance_loss(f(p), idx, 2, 0.5, load, m, s, loss, wl)
        out.append((dx, dW.clone(), db.clone(), load, s.clone(), m.clone(), loss.clone()))
    assert all(torch.equal(a, b) for a, b in zip(out[0][:5], out[1][:5]))
    close(out[1][5], out[0][5].double(), 256 * H * out[0][5].double())     # (summed in another order)
    close(out[1][6], out[0][6].double(), 320 * H * out[0][6].double())


def test_nothing_dispatched():
    """Packed rows of which there are none: what stays is the gate's own gradient, and zeros for the weights."""
    T, d, E = 40, 64, 4
    g = gen(3)
    x, Wg = normal(g, T, d), normal(g, d, E)
    p, idx, w = routing(g, T, E, 1, 0)
    dw, dst, none = normal(g, T, 1), torch.full((T, 1), -1, dtype=torch.int32, device=DEV), torch.zeros((0, d), device=DEV)
    out = []
    for kw in (dict(), dict(dx_perm=none, dst_row=dst)):
        dx, dW = empty(T, d, "f32"), torch.zeros(d, E, device=DEV)
        B.scmoe_gate_backward(x, Wg, p, idx, w, dw, dx, dW, None, None, **kw)
        out.append((dx, dW))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    B.scmoe_combine_backward(x, none, dst, w, 1, dy_perm=none, dgate_w=dw)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_past_the_caches(dtype):
    """More than 256 MB: loads and stores go past the caches.  Rows have the same bits as in calls of a part of them, which do not."""
    d, E = 1024, 8
    T = 50000 if dtype == "bf16" else 25000
    g = gen(12)
    x, r, gamma, beta = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype), normal(g, d), normal(g, d)
    half = [slice(0, T // 2), slice(T // 2, T)]
    y, s, mean, rstd = empty(T, d, dtype), empty(T, d, dtype), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    B.scmoe_layer_norm(x, gamma, beta, 1e-5, y, residual=r, sum_out=s, mean=mean, rstd=rstd)
    for at in half:
        y2, s2 = empty(T // 2, d, dtype), empty(T // 2, d, dtype)
        B.scmoe_layer_norm(x[at], gamma, beta, 1e-5, y2, residual=r[at], sum_out=s2)
        assert torch.equal(y[at], y2) and torch.equal(s[at], s2)
    ws = torch.zeros(8 << 20, device=DEV)
    dx, dgamma, dbeta = empty(T, d, dtype), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    B.scmoe_layer_norm_backward(y, s, gamma, mean, rstd, dx, dgamma, dbeta, ws, dsum=r)
    for at in half:
        dx2 = empty(T // 2, d, dtype)
        B.scmoe_layer_norm_backward(y[at], s[at], gamma, mean[at], rstd[at], dx2, dsum=r[at])
        assert torch.equal(dx[at], dx2)
    xh = (s.double() - mean.double()[:, None]) * rstd.double()[:, None] * y.double()
    close(dgamma, xh.sum(0), 256 * H * xh.abs().sum(0))
    del xh
    close(dbeta, y.double().sum(0), 256 * H * y.double().abs().sum(0))
    p, idx, w = routing(g, T, E, 2, 1)
    dst, yp = packed(g, T, E, 2, idx, d, dtype)
    dyp, dw = empty(yp.shape[0], d, dtype), torch.zeros((T, 2), device=DEV)
    B.scmoe_combine_backward(x, yp, dst, w, 2, dy_perm=dyp, dgate_w=dw)
    dyp2, dw2 = empty(yp.shape[0], d, dtype), torch.zeros((T, 2), device=DEV)
    for at in half:
        B.scmoe_combine_backward(x[at], yp, dst[at], w[at], 2, dy_perm=dyp2, dgate_w=dw2[at])
    assert torch.equal(dyp, dyp2) and torch.equal(dw, dw2)
    Wg, dW, db = normal(g, d, E), torch.zeros(d, E, device=DEV), torch.zeros(E, device=DEV)
    B.scmoe_gate_backward(y, Wg, p, idx, w, dw, dx, dW, db, ws, k=2, normalize=1, dx_perm=dyp, dst_row=dst)
    dW2, db2 = torch.zeros(d, E, dtype=torch.float64, device=DEV), torch.zeros(E, dtype=torch.float64, device=DEV)
    for at in half:
        dx2, dWh, dbh = empty(T // 2, d, dtype), torch.zeros(d, E, device=DEV), torch.zeros(E, device=DEV)
        B.scmoe_gate_backward(y[at], Wg, p[at], idx[at], w[at], dw[at], dx2, dWh, dbh, ws, k=2, normalize=1, dx_perm=dyp, dst_row=dst[at])
        assert torch.equal(dx[at], dx2)
        dW2 += dWh.double()
        db2 += dbh.double()
    _, _, _, wW, sW, wb, sb = gate_grad_ref(y, Wg, p, idx, w, dw, 1, None, None, None, None, None)
    close(dW, wW, 256 * H * sW)
    close(db, wb, 256 * H * sb)
    close(dW2, wW, 256 * H * sW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_router_learns(dtype):
    """The example: forty steps find most of the hidden router's choices (by chance 2 of 8 experts agree at a quarter)."""
    from paper_2404_05019_amd.train_routing import train
    errors, first, last = train(steps=40, T=1024, d=128, F=256, dtype=TYPES[dtype])
    assert first < 0.4 and last > 0.75 and errors[-1] < errors[0] / 3, (errors[0], errors[-1], first, last)


def test_binding_refuses_tensors_that_do_not_fit():
    x, v = torch.zeros((4, 64), device=DEV), torch.zeros(64, device=DEV)
    with pytest.raises(TypeError):
        B.scmoe_layer_norm(x, v, None, 1e-5, x.bfloat16())
    with pytest.raises(TypeError):
        B.scmoe_layer_norm(x, v[:32], None, 1e-5, x)
    with pytest.raises(TypeError):
        B.scmoe_layer_norm(x, v.double(), None, 1e-5, x)
    with pytest.raises(B.ScmoeError) as e:
        B.scmoe_layer_norm_backward(x, x, v, v[:4], v[:4], x, v, None, v[:16])
    assert e.value.status == 4
    i = torch.zeros((4, 1), dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError):
        B.scmoe_balance_loss(x, i.long(), 1, 0.1, i, v, v, v[:1], v)
    with pytest.raises(TypeError):
        B.scmoe_balance_loss(x, i, 1, 0.1, torch.zeros(64, dtype=torch.int32, device=DEV), v, v, v[:1], v, mask=v[:4])
    with pytest.raises(TypeError):
        B.scmoe_combine_backward(x, x[:, :32], i, v[:4], 1, dgate_w=v[:4])
