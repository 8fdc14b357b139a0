"""The training operators without a GPU: what they refuse on the host, the workspaces they ask for, and what they would launch
(tests/hip_recorder.c in place of the HIP runtime)."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1
P = 0x100000                # an aligned address that is never dereferenced
BIG = 1 << 40


def norm(lib, x=P, ldx=64, dtype=F32, res=None, ldres=64, gamma=P, beta=P, eps=1e-5, T=10, d=64, s=None, lds=64, y=P, ldy=64, mean=None,
         rstd=None):
    return lib.scmoe_layer_norm(x, ldx, dtype, res, ldres, gamma, beta, C.c_float(eps), T, d, s, lds, y, ldy, mean, rstd, None)


def norm_grad(lib, dy=P, lddy=64, x=P, ldx=64, dtype=F32, gamma=P, mean=P, rstd=P, dsum=None, ldds=64, T=10, d=64, dx=P, lddx=64, dgamma=P,
              dbeta=P, ws=P, nb=BIG):
    return lib.scmoe_layer_norm_backward(dy, lddy, x, ldx, dtype, gamma, mean, rstd, dsum, ldds, T, d, dx, lddx, dgamma, dbeta, ws, nb, None)


def loss(lib, probs=P, idx=P, mask=None, T=10, E=4, k=1, load=P, mean=P, slope=P, out=P, ws=P, nb=BIG):
    return lib.scmoe_balance_loss(probs, idx, mask, T, E, k, C.c_float(0.01), load, mean, slope, out, ws, nb, None)


def gate_grad(lib, x=P, ldx=64, dtype=F32, Wg=P, probs=P, idx=P, w=P, dw=P, slope=None, dloss=None, mask=None, T=1000, d=64, E=4, k=1,
              normalize=0, dxp=None, ldp=64, dst=None, dx=P, lddx=64, dW=P, db=None, ws=P, nb=BIG):
    return lib.scmoe_gate_backward(x, ldx, dtype, Wg, probs, idx, w, dw, slope, dloss, mask, T, d, E, k, normalize, dxp, ldp, dst, dx, lddx,
                                   dW, db, ws, nb, None)


def combine_grad(lib, dy=P, lddy=64, dtype=F32, yp=P, ldyp=64, dst=P, w=P, T=10, d=64, k=1, base=None, ldb=64, coef=None, dyp=P, lddyp=64,
                 dw=P, dbase=None, lddb=64, dcoef=None):
    return lib.scmoe_combine_backward(dy, lddy, dtype, yp, ldyp, dst, w, T, d, k, base, ldb, coef, dyp, lddyp, dw, dbase, lddb, dcoef, None)


@pytest.fixture(scope="module")
def lib():
    from paper_2404_05019_amd import binding
    return binding.lib()


NULL, SHAPE, DTYPE, WORKSPACE, ARG = 1, 2, 3, 4, 6


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(res=P)), (NULL, dict(s=P)),
    (SHAPE, dict(T=-1)), (SHAPE, dict(d=0)), (SHAPE, dict(d=60)), (SHAPE, dict(d=16392, ldx=16392, ldy=16392)), (SHAPE, dict(ldx=56)),
    (SHAPE, dict(ldx=66)), (SHAPE, dict(x=P + 4)), (SHAPE, dict(ldy=0)), (SHAPE, dict(gamma=P + 4)), (SHAPE, dict(beta=P + 8)),
    (SHAPE, dict(dtype=BF16, ldx=68)), (SHAPE, dict(res=P, s=P, ldres=8)), (SHAPE, dict(res=P, s=P + 8)),
    (DTYPE, dict(dtype=2)), (ARG, dict(eps=0.0)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(eps=float("inf"))),
])
def test_layer_norm_refuses(lib, want, bad):
    assert norm(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(dy=None)), (NULL, dict(x=None)), (NULL, dict(mean=None)), (NULL, dict(rstd=None)), (NULL, dict(dx=None)), (NULL, dict(ws=None)),
    (NULL, dict(ws=None, dbeta=None)), (SHAPE, dict(T=-1)), (SHAPE, dict(d=12)), (SHAPE, dict(d=16392)), (SHAPE, dict(lddy=0)),
    (SHAPE, dict(lddx=60)), (SHAPE, dict(dsum=P, ldds=32)), (SHAPE, dict(ws=P + 8)), (SHAPE, dict(gamma=P + 4)), (DTYPE, dict(dtype=9)),
    (WORKSPACE, dict(nb=0)), (WORKSPACE, dict(nb=64 * 8 + 7)),
])
def test_layer_norm_backward_refuses(lib, want, bad):
    assert norm_grad(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(probs=None)), (NULL, dict(idx=None)), (NULL, dict(load=None)), (NULL, dict(mean=None)), (NULL, dict(slope=None)),
    (NULL, dict(out=None)), (NULL, dict(ws=None)), (SHAPE, dict(T=-1)), (SHAPE, dict(E=0)), (SHAPE, dict(E=65)), (SHAPE, dict(E=2, k=3)),
    (SHAPE, dict(T=1 << 30, k=4)), (SHAPE, dict(ws=P + 4)), (ARG, dict(k=0)), (ARG, dict(E=8, k=5)), (WORKSPACE, dict(nb=0)),
])
def test_balance_loss_refuses(lib, want, bad):
    assert loss(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(x=None)), (NULL, dict(Wg=None)), (NULL, dict(probs=None)), (NULL, dict(idx=None)), (NULL, dict(dw=None)), (NULL, dict(dx=None)),
    (NULL, dict(dW=None)), (NULL, dict(w=None, normalize=1)), (NULL, dict(dxp=P)), (NULL, dict(dst=P)), (NULL, dict(ws=None)),
    (SHAPE, dict(T=-1)), (SHAPE, dict(d=4)), (SHAPE, dict(E=0)), (SHAPE, dict(E=65)), (SHAPE, dict(E=1, k=2)), (SHAPE, dict(ldx=8)),
    (SHAPE, dict(lddx=65)), (SHAPE, dict(dxp=P, dst=P, ldp=8)), (SHAPE, dict(ws=P + 8)), (DTYPE, dict(dtype=-1)), (ARG, dict(k=0)),
    (ARG, dict(E=8, k=5)), (ARG, dict(normalize=2)), (WORKSPACE, dict(nb=64)),
])
def test_gate_backward_refuses(lib, want, bad):
    assert gate_grad(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(dy=None)), (NULL, dict(dst=None)), (NULL, dict(w=None)), (NULL, dict(yp=None)), (NULL, dict(yp=None, dw=None, dcoef=P, base=P)),
    (NULL, dict(dcoef=P)), (SHAPE, dict(T=-1)), (SHAPE, dict(d=10)), (SHAPE, dict(lddy=8)), (SHAPE, dict(ldyp=66)), (SHAPE, dict(lddyp=0)),
    (SHAPE, dict(base=P, ldb=8)), (SHAPE, dict(dbase=P, lddb=62)), (DTYPE, dict(dtype=7)), (ARG, dict(k=0)), (ARG, dict(k=5)),
])
def test_combine_backward_refuses(lib, want, bad):
    assert combine_grad(lib, **bad) == want


def test_calls_without_tokens(lib):
    """No launch is needed where nothing is written."""
    assert norm(lib, T=0, x=None, y=None) == 0
    assert norm_grad(lib, T=0, dy=None, x=None, dx=None, dgamma=None, dbeta=None, ws=None, nb=0) == 0
    assert combine_grad(lib, T=0, dy=None, yp=None, dst=None, w=None) == 0


def test_workspace_sizes(lib):
    from paper_2404_05019_amd import binding as B
    assert B.scmoe_layer_norm_backward_workspace_bytes(0, 64) == 0
    for T in (1, 100, 32768, 1 << 30):
        for d in (8, 64, 2048, 16384):
            assert d * 8 <= B.scmoe_layer_norm_backward_workspace_bytes(T, d) <= 4096 * d
            assert B.scmoe_gate_backward_workspace_bytes(T, d, 64) <= 4 * (1024 * 128 + d) * 65
        assert 0 < B.scmoe_balance_loss_workspace_bytes(T, 64) <= 1 << 18
    for call in (lambda: B.scmoe_layer_norm_backward_workspace_bytes(-1, 64), lambda: B.scmoe_layer_norm_backward_workspace_bytes(1, 12),
                 lambda: B.scmoe_balance_loss_workspace_bytes(1, 65), lambda: B.scmoe_gate_backward_workspace_bytes(1, 64, 0)):
        with pytest.raises(B.ScmoeError):
            call()
    assert lib.scmoe_gate_backward_workspace_bytes(1, 64, 4, None) == 1


def test_binding_refuses_tensors_in_host_memory():
    """An address that the GPU cannot read never reaches a kernel."""
    import torch
    from paper_2404_05019_amd import binding as B
    x, v, i, s = torch.zeros(4, 64), torch.zeros(64), torch.zeros((4, 1), dtype=torch.int32), torch.zeros(4)
    for call in (lambda: B.scmoe_layer_norm(x, v, v, 1e-5, x), lambda: B.scmoe_layer_norm_backward(x, x, v, s, s, x),
                 lambda: B.scmoe_balance_loss(x, i, 1, 0.1, i, v, v, v[:1], v),
                 lambda: B.scmoe_gate_backward(x, x.t().contiguous(), x, i, s, s, x, x, None, v),
                 lambda: B.scmoe_combine_backward(x, x, i, s, 1, dgate_w=s)):
        with pytest.raises(TypeError, match="on the GPU"):
            call()


CALLS = {"norm": norm, "norm_grad": norm_grad, "loss": loss, "gate_grad": gate_grad, "combine_grad": combine_grad}


def _child(recorder, library, calls):
    rec = C.CDLL(recorder, mode=C.RTLD_GLOBAL)
    lib = C.CDLL(library)
    i32, i64, vp, sz, f32 = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t, C.c_float
    lib.scmoe_layer_norm.argtypes = [vp, i64, i32, vp, i64, vp, vp, f32, i32, i32, vp, i64, vp, i64, vp, vp, vp]
    lib.scmoe_layer_norm_backward.argtypes = [vp, i64, vp, i64, i32, vp, vp, vp, vp, i64, i32, i32, vp, i64, vp, vp, vp, sz, vp]
    lib.scmoe_balance_loss.argtypes = [vp, vp, vp, i32, i32, i32, f32, vp, vp, vp, vp, vp, sz, vp]
    lib.scmoe_gate_backward.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, i64, vp, vp, i64, vp, vp,
                                        vp, sz, vp]
    lib.scmoe_combine_backward.argtypes = [vp, i64, i32, vp, i64, vp, vp, i32, i32, i32, vp, i64, vp, vp, i64, vp, vp, i64, vp, vp]
    rec.recorder_text.restype = C.c_char_p
    out = []
    for name, kw in calls:
        rec.recorder_reset()
        st = CALLS[name](lib, **kw)
        out.append([st, rec.recorder_text().decode()])
    print(json.dumps(out))


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("recorder") / "hip_recorder.so")
    subprocess.check_call(["gcc", "-std=c11", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "hip_recorder.c"), "-o", so])
    library = os.path.join(ROOT, "paper_2404_05019_amd", "libscmoe.so")

    def run(calls):
        r = subprocess.run([sys.executable, os.path.abspath(__file__), so, library, json.dumps(calls)], stdout=subprocess.PIPE,
                           stderr=subprocess.PIPE, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return [(st, [line.split(" ") for line in text.splitlines()]) for st, text in json.loads(r.stdout)]
    return run


def _wide(d):
    return {n: d for n in ("ldx", "ldy", "lddy", "lddx", "ldyp", "lddyp")}


def test_launches_stay_within_the_runtime_s_limits(record):
    """Any number of tokens: under 2^32 threads and 2^31 workgroups, at most 1024 threads each, no copies and no memsets."""
    calls = []
    for T in (1, 63, 4096, 32768, 1 << 24, (1 << 31) - 1):
        for d in (8, 512, 2048, 4096, 16384):
            w = _wide(d)
            calls.append(("norm", dict(T=T, d=d, ldx=d, ldy=d)))
            calls.append(("norm_grad", dict(T=T, d=d, ldx=d, lddy=d, lddx=d)))
            calls.append(("gate_grad", dict(T=T, d=d, E=64, ldx=d, lddx=d)))
            calls.append(("combine_grad", dict(T=T, d=d, **{n: w[n] for n in ("lddy", "ldyp", "lddyp")})))
        calls.append(("loss", dict(T=T, E=64)))
    for (name, kw), (st, lines) in zip(calls, record(calls)):
        assert st == 0, (name, kw)
        assert 1 <= len(lines) <= 2 and all(w[0] == "kernel" for w in lines), (name, kw, lines)
        for w in lines:
            gx, gy, gz, bx, by, bz = (int(v) for v in w[3:9])
            assert 1 <= gx < 1 << 31 and gy == gz == by == bz == 1 and 1 <= bx <= 1024 and gx * bx < 1 << 32, (name, kw, w)
            assert int(w[9]) <= 64 << 10


def test_sums_over_no_tokens_are_written(record):
    got = record([("norm_grad", dict(T=0, ws=None, nb=0)), ("loss", dict(T=0, probs=None, idx=None, ws=None, nb=0)),
                  ("gate_grad", dict(T=0, x=None, probs=None, dx=None, ws=None, nb=0))])
    assert all(st == 0 and len(lines) == 1 for st, lines in got)


if __name__ == "__main__":
    _child(sys.argv[1], sys.argv[2], json.loads(sys.argv[3]))
