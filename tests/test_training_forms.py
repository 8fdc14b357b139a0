"""Forms of the training kernels that calls of many bytes and many turns take, against the same formulas in 64 bits.  The bounds are
those of tests/test_training_ops.py; the longest sums here are over five turns of 16 tokens, four waves and 16 parts, or eight values in
each of 21 turns of a row."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2404_05019_amd import binding as B
    from gpu_util import DEV
    from test_training_ops import H, NAN, check_gate, close, empty, gen, norm_grad_ref, norm_ref, normal, packed, routing, workspace

CACHES = 256 << 20          # calls that move more bytes load and store past the caches


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,k,normalize", [(E, k, n) for E in (12, 32, 64) for k in (1, 2, 3, 4) for n in (0, 1) if k > 1 or n == 0])
def test_gate_backward_of_several_turns(E, k, normalize, dtype):
    """Five turns of every wave: what a turn loads ahead is the next one's, for each number of choices."""
    check_gate(4999, 4096, E, k, dtype, normalize, 10 * E + k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,k", [(12, 1), (32, 1), (64, 1), (12, 3), (32, 2), (64, 4)])
def test_gate_backward_past_the_caches(E, k, dtype):
    T, d = CACHES // ((2 + k) * 4096 * (2 if dtype == "bf16" else 4)) + 17, 4096
    check_gate(T, d, E, k, dtype, int(k > 1), E + k)


def norm_rows(d, dtype, rows):
    """Rows for more bytes than the caches hold where a call moves `rows` of them for each."""
    return CACHES // (rows * d * (2 if dtype == "bf16" else 4)) + 5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [264, 520, 2048, 4104, 8200, 16384])
def test_layer_norm_past_the_caches(d, dtype):
    T = norm_rows(d, dtype, 4)
    g = gen(d)
    x, r, gamma, beta = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype), normal(g, d), normal(g, d)
    y, s, mean, rstd = empty(T, d, dtype), empty(T, d, dtype), torch.zeros(T, device=DEV), torch.zeros(T, device=DEV)
    B.scmoe_layer_norm(x, gamma, beta, 1e-5, y, residual=r, sum_out=s, mean=mean, rstd=rstd)
    assert torch.equal(s, (x.float() + r.float()).to(x.dtype))
    wy, wm, wr, slack = norm_ref(s, gamma, beta, 1e-5)
    close(y, wy, slack, dtype)
    close(mean, wm, 64 * H * s.double().abs().mean(1))
    close(rstd, wr, 64 * H * wr)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_sum", [True, False])
@pytest.mark.parametrize("d", [2048, 4104, 8200, 16384])
def test_layer_norm_backward_past_the_caches(d, with_sum, dtype):
    T = norm_rows(d, dtype, 4 if with_sum else 3)
    g = gen(d + 1)
    x, dy, gamma = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype), normal(g, d)
    dsum = normal(g, T, d, dtype=dtype) if with_sum else None
    mean, rstd = 0.1 * normal(g, T), 0.5 + torch.rand(T, generator=g, device=DEV)
    ws, whole = workspace(B.scmoe_layer_norm_backward_workspace_bytes(T, d))
    dx, dgamma, dbeta = empty(T, d, dtype), torch.full((d,), NAN, device=DEV), torch.full((d,), NAN, device=DEV)
    B.scmoe_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, dsum=dsum)
    wx, sx, wg, sg, wb, sb = norm_grad_ref(dy, x, gamma, mean, rstd, dsum)
    close(dx, wx, sx, dtype)
    close(dgamma, wg, sg)
    close(dbeta, wb, sb)
    assert bool(whole[ws.numel():].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1032, 2056])
@pytest.mark.parametrize("k,cg", [(1, False), (1, True), (2, False), (3, True), (4, False)])
def test_combine_backward_past_the_caches(k, cg, d, dtype):
    """Rows of more than 2 KB: the whole call goes past the caches, its halves do not.  The same bits, and those of the formula."""
    rows = 1 + 2 * k + (2 if cg else 0)
    T = 2 * (norm_rows(d, dtype, rows) // 2 + 1)
    g = gen(d + k)
    dst, yp = packed(g, T, 1, k, torch.zeros((T, k), dtype=torch.int32, device=DEV), d, dtype)
    dy, w = normal(g, T, d, dtype=dtype), torch.rand((T, k), generator=g, device=DEV)
    base, coef = (normal(g, T, d, dtype=dtype), torch.rand((T, 2), generator=g, device=DEV)) if cg else (None, None)
    whole = {}
    for parts in (1, 2):
        dyp, dw = empty(yp.shape[0], d, dtype), torch.full((T, k), NAN, device=DEV)
        dbase, dcoef = (empty(T, d, dtype), torch.full((T, 2), NAN, device=DEV)) if cg else (None, None)
        for i in range(parts):
            at = slice(i * (T // parts), (i + 1) * (T // parts))
            cut = lambda t: None if t is None else t[at]  # noqa: B023, E731
            B.scmoe_combine_backward(dy[at], yp, dst[at], w[at], k, dy_perm=dyp, dgate_w=dw[at], base=cut(base), coef=cut(coef),
                                     dbase=cut(dbase), dcoef=cut(dcoef))
        whole[parts] = [t for t in (dyp, dw, dbase, dcoef) if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(whole[1], whole[2]))
    dyp, dw = whole[1][:2]
    kept, d64 = dst >= 0, dy.double()
    c0, c1 = (coef[:, :1].double(), coef[:, 1:].double()) if cg else (1.0, torch.ones((T, 1), dtype=torch.float64, device=DEV))
    dc1, size_c1 = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(T, dtype=torch.float64, device=DEV)
    for j in range(k):
        on = kept[:, j].nonzero().flatten()
        at = dst[on, j].long()
        terms = yp[at].double() * d64[on]
        dot, size = terms.sum(1), terms.abs().sum(1)
        del terms
        c, wj = c1[on, 0], w[on, j].double()
        close(dw[on, j], c * dot, 128 * H * c * size)
        assert bool((dw[~kept[:, j], j] == 0).all())
        want = (c * wj)[:, None] * d64[on]
        close(dyp[at], want, 2 * H * want.abs(), dtype)
        dc1[on] += wj * dot
        size_c1[on] += wj * size
    if cg:
        dbase, dcoef = whole[1][2:]
        close(dbase, c0 * d64, 0.0, dtype)
        dc0 = d64 * base.double()
        close(dcoef, torch.stack([dc0.sum(1), dc1], 1), 140 * H * torch.stack([dc0.abs().sum(1), size_c1], 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gate_backward_keeps_infinities_apart(dtype):
    """An infinity in a token's x reaches its columns of dW_g, one in W_g its column of dx: non-finite there (in bf16 perhaps NaN, where the
    formula has an infinity), the same bits as without it everywhere else."""
    T, d, E = 150, 264, 8
    g = gen(5)
    x, Wg = normal(g, T, d, dtype=dtype), normal(g, d, E)
    p, idx, w = routing(g, T, E, 2, 1)
    dw = normal(g, T, 2)
    ws, _ = workspace(B.scmoe_gate_backward_workspace_bytes(T, d, E))
    bad_x, bad_W = x.clone(), Wg.clone()
    bad_x[77, 9] = float("inf")
    bad_W[11, 3] = -float("inf")
    out = [(empty(T, d, dtype), torch.zeros(d, E, device=DEV), torch.zeros(E, device=DEV)) for _ in range(3)]
    for (a, b), o in zip(((x, Wg), (bad_x, Wg), (x, bad_W)), out):
        B.scmoe_gate_backward(a, b, p, idx, w, dw, *o, ws, k=2, normalize=1)
    (dx, dW, db), (dx1, dW1, db1), (dx2, dW2, db2) = out
    rows, cols = torch.arange(d, device=DEV) != 9, torch.arange(d, device=DEV) != 11
    assert torch.equal(dx, dx1) and torch.equal(db, db1) and torch.equal(dW[rows], dW1[rows]) and not bool(dW1[9].isfinite().any())
    assert torch.equal(dW, dW2) and torch.equal(db, db2) and torch.equal(dx[:, cols], dx2[:, cols]) and not bool(dx2[:, 11].isfinite().any())
