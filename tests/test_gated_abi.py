"""The gated feed-forward block, its gradient and the activation checkpoints without a GPU: what they refuse on the host, the workspaces they
ask for, what they would launch (tests/hip_recorder.c in place of the HIP runtime), and which tensors the binding refuses."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1
NOTHING, FULL, EIGHT = 0, 1, 2
P = 0x100000                # an aligned address that is never dereferenced
BIG = 1 << 50
NULL, SHAPE, DTYPE, WORKSPACE, ARG = 1, 2, 3, 4, 6


def pack(lib, x=P, ldx=64, dtype=F32, n=None, rows=10, w=64, q=P, ldq=80):
    return lib.scmoe_checkpoint_pack(x, ldx, dtype, n, rows, w, q, ldq, None)


def unpack(lib, x=P, ldx=64, dtype=F32, n=None, rows=10, w=64, q=P, ldq=80):
    return lib.scmoe_checkpoint_unpack(q, ldq, n, rows, w, x, ldx, dtype, None)


def ffn(lib, x=P, ldx=None, dtype=F32, offs=P, rows=10, E=2, d=64, F=96, W1=P, ldw1=None, W2=P, ldw2=None, act=2, hid=P, ldh=None, pre=None, ldpre=None,
        keep=NOTHING, y=P, ldy=None, ws=None, nb=0):
    ldpre = (2 * F if keep == FULL else 16 * F) if ldpre is None else ldpre
    return lib.scmoe_gated_ffn(x, ldx or d, dtype, offs, rows, E, d, F, W1, ldw1 or d, W2, ldw2 or F, act, hid, ldh or F, pre, ldpre, keep, y, ldy or d, ws, nb,
                               None)


def grad(lib, dy=P, lddy=None, dtype=F32, x=P, ldx=None, xk=FULL, pre=P, ldpre=None, pk=FULL, offs=P, rows=10, E=2, d=64, F=96, W1=P, ldw1=None, W2=P,
         ldw2=None, act=2, dx=P, lddx=None, dW1=P, dW2=P, ws=P, nb=BIG):
    ldpre = (2 * F if pk == FULL else 16 * F) if ldpre is None else ldpre
    ldx = (d if xk == FULL else 16 * d) if ldx is None else ldx
    return lib.scmoe_gated_ffn_backward(dy, lddy or d, dtype, x, ldx, xk, pre, ldpre, pk, offs, rows, E, d, F, W1, ldw1 or d, W2, ldw2 or F, act, dx, lddx or d,
                                        dW1, dW2, ws, nb, None)


CALLS = {"pack": pack, "unpack": unpack, "ffn": ffn, "grad": grad}


def declare(lib):
    i32, i64, vp, sz = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
    lib.scmoe_checkpoint_pack.argtypes = [vp, i64, i32, vp, i32, i32, vp, i64, vp]
    lib.scmoe_checkpoint_unpack.argtypes = [vp, i64, vp, i32, i32, vp, i64, i32, vp]
    lib.scmoe_gated_ffn.argtypes = [vp, i64, i32, vp, i32, i32, i32, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, i32, vp, i64, vp, sz, vp]
    lib.scmoe_gated_ffn_backward.argtypes = [vp, i64, i32, vp, i64, i32, vp, i64, i32, vp, i32, i32, i32, i32, vp, i64, vp, i64, i32, vp, i64, vp, vp, vp, sz, vp]
    return lib


@pytest.fixture(scope="module")
def lib():
    from paper_2404_05019_amd import binding
    return binding.lib()


@pytest.mark.parametrize("call", [pack, unpack])
@pytest.mark.parametrize("want,bad", [
    (NULL, dict(x=None)), (NULL, dict(q=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(w=0)), (SHAPE, dict(w=60)), (SHAPE, dict(x=P + 4)),
    (SHAPE, dict(q=P + 8)), (SHAPE, dict(ldx=56)), (SHAPE, dict(ldx=66)), (SHAPE, dict(ldq=64)), (SHAPE, dict(ldq=72)), (SHAPE, dict(dtype=BF16, ldx=68)),
    (SHAPE, dict(w=104, ldx=104, ldq=104)), (DTYPE, dict(dtype=2)), (DTYPE, dict(dtype=-1)),
    (SHAPE, dict(w=(1 << 28) + 8, ldx=1 << 30, ldq=1 << 30)), (SHAPE, dict(w=(1 << 31) - 8, ldx=1 << 31, ldq=1 << 33, dtype=BF16)),
])
def test_checkpoints_refuse(lib, call, want, bad):
    assert call(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(x=None)), (NULL, dict(offs=None)), (NULL, dict(W1=None)), (NULL, dict(W2=None)), (NULL, dict(hid=None)), (NULL, dict(y=None)),
    (NULL, dict(keep=FULL)), (NULL, dict(keep=EIGHT)), (SHAPE, dict(rows=-1)), (SHAPE, dict(E=0)), (SHAPE, dict(d=0)), (SHAPE, dict(d=60)), (SHAPE, dict(F=100)),
    (SHAPE, dict(F=-8)), (SHAPE, dict(d=(1 << 17) + 8)), (SHAPE, dict(F=(1 << 17) + 8)), (SHAPE, dict(ldx=56)), (SHAPE, dict(ldx=66)),
    (SHAPE, dict(dtype=BF16, ldx=68)), (SHAPE, dict(ldw1=62)), (SHAPE, dict(ldw2=64)), (SHAPE, dict(ldh=8)), (SHAPE, dict(ldy=8)), (SHAPE, dict(x=P + 8)),
    (SHAPE, dict(W1=P + 4)), (SHAPE, dict(W2=P + 2)), (SHAPE, dict(hid=P + 1)), (SHAPE, dict(y=P + 8)), (SHAPE, dict(ldx=(1 << 18) + 8)),
    (SHAPE, dict(F=1 << 15, ldw1=1 << 15)), (SHAPE, dict(d=1 << 15, ldw2=1 << 16)), (SHAPE, dict(keep=FULL, pre=P, ldpre=96)),
    (SHAPE, dict(keep=EIGHT, pre=P, ldpre=96)), (SHAPE, dict(keep=EIGHT, pre=P, ldpre=104)), (SHAPE, dict(keep=EIGHT, pre=P + 8)), (SHAPE, dict(ws=P + 8, nb=64)),
    (SHAPE, dict(rows=(1 << 30) + 1)), (SHAPE, dict(rows=1 << 30, F=8192)), (SHAPE, dict(E=1 << 30)), (SHAPE, dict(E=1 << 20, d=2048, F=8192)),
    (DTYPE, dict(dtype=2)), (ARG, dict(act=3)), (ARG, dict(act=-1)), (ARG, dict(keep=3, pre=P)), (ARG, dict(keep=-1, pre=P)),
])
def test_forward_refuses(lib, want, bad):
    assert ffn(lib, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (NULL, dict(dy=None)), (NULL, dict(x=None)), (NULL, dict(pre=None)), (NULL, dict(offs=None)), (NULL, dict(W1=None)), (NULL, dict(W2=None)),
    (NULL, dict(ws=None)), (NULL, dict(dx=None, dW1=None, dW2=None)), (NULL, dict(rows=0, offs=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(E=0)),
    (SHAPE, dict(d=4)), (SHAPE, dict(F=4)), (SHAPE, dict(lddy=56)), (SHAPE, dict(ldx=56)), (SHAPE, dict(ldpre=96)), (SHAPE, dict(pk=EIGHT, ldpre=96)),
    (SHAPE, dict(xk=EIGHT, ldx=64)), (SHAPE, dict(lddx=8)), (SHAPE, dict(ldw1=8)), (SHAPE, dict(ldw2=8)), (SHAPE, dict(dy=P + 8)), (SHAPE, dict(dx=P + 8)),
    (SHAPE, dict(dW1=P + 8)), (SHAPE, dict(dW2=P + 4)), (SHAPE, dict(ws=P + 8)), (SHAPE, dict(lddy=(1 << 18) + 8)), (SHAPE, dict(F=1 << 15, ldw1=1 << 15)),
    (DTYPE, dict(dtype=5)), (ARG, dict(act=9)), (ARG, dict(pk=NOTHING)), (ARG, dict(xk=NOTHING)), (ARG, dict(pk=3)), (WORKSPACE, dict(nb=0)),
    (WORKSPACE, dict(nb=4 * 10 * (192 + 96 + 64) - 1)),
])
def test_backward_refuses(lib, want, bad):
    assert grad(lib, **bad) == want


def test_sizes(lib):
    from paper_2404_05019_amd import binding as B
    assert [B.scmoe_checkpoint_ld(w) for w in (8, 32, 40, 480, 1000, 8192)] == [16, 48, 48, 496, 1040, 8448]
    assert B.scmoe_checkpoint_ld(1 << 28) == (1 << 28) + (1 << 23)
    for w in (0, -8, 12, (1 << 28) + 8, (1 << 31) - 8):
        with pytest.raises(B.ScmoeError):
            B.scmoe_checkpoint_ld(w)
    assert lib.scmoe_checkpoint_ld(8, None) == NULL
    out = C.c_size_t(77)
    assert lib.scmoe_gated_ffn_workspace_bytes(BF16, 64, 64, None) == NULL and lib.scmoe_gated_ffn_backward_workspace_bytes(BF16, 1, 1, 64, 64, None) == NULL
    for bad in ((2, 64, 64), (BF16, 60, 64), (BF16, 64, 0)):
        assert lib.scmoe_gated_ffn_workspace_bytes(*bad, C.byref(out)) in (SHAPE, DTYPE)
        assert lib.scmoe_gated_ffn_backward_workspace_bytes(bad[0], 10, 1, *bad[1:], C.byref(out)) in (SHAPE, DTYPE)
    assert out.value == 77
    for rows in (0, 1, 777, 32768, 1 << 24):
        for d, F in ((8, 8), (1000, 1360), (2048, 8192)):
            for dtype, b in ((BF16, 2), (F32, 4)):
                n = B.scmoe_gated_ffn_backward_workspace_bytes(dtype, rows, 16, d, F)
                assert rows * (d + 3 * F) * b <= n <= rows * ((d + 3 * F) * b + 256) + (1 << 28)


def test_calls_without_rows(lib):
    """No launch is needed where nothing is written."""
    assert pack(lib, rows=0, x=None, q=None) == 0 and unpack(lib, rows=0, x=None, q=None) == 0
    assert ffn(lib, rows=0, x=None, y=None, hid=None, W1=None, W2=None, offs=None) == 0
    assert grad(lib, rows=0, dy=None, x=None, pre=None, dW1=None, dW2=None, offs=None, ws=None, nb=0) == 0


def _child(recorder, library, calls):
    rec = C.CDLL(recorder, mode=C.RTLD_GLOBAL)
    lib = declare(C.CDLL(library))
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


def test_launches_stay_within_the_runtime_s_limits(record):
    """Any number of rows: under 2^32 threads and 2^31 workgroups, at most 160 KiB of LDS, no copies and no memsets (which a graph may not
    hold here)."""
    calls = []
    for rows in (1, 16, 300, 5000, 32768, 1 << 24):
        for d, F, E in ((8, 8, 1), (1000, 2728, 32), (2048, 8192, 16), (4096, 14336, 64)):
            for dtype in (F32, BF16):
                calls.append(("ffn", dict(rows=rows, d=d, F=F, E=E, dtype=dtype, ws=P, nb=BIG)))
                for keep in (FULL, EIGHT):
                    calls.append(("ffn", dict(rows=rows, d=d, F=F, E=E, dtype=dtype, keep=keep, pre=P)))
                    calls.append(("grad", dict(rows=rows, d=d, F=F, E=E, dtype=dtype, xk=keep, pk=keep)))
        for w in (8, 1000, 8192):
            calls += [(n, dict(rows=rows, w=w, ldx=w, ldq=16 * w, dtype=dtype)) for n in ("pack", "unpack") for dtype in (F32, BF16)]
    for (name, kw), (st, lines) in zip(calls, record(calls)):
        assert st == 0, (name, kw)
        assert 1 <= len(lines) <= 6 and all(w[0] == "kernel" for w in lines), (name, kw, lines)
        for w in lines:
            gx, gy, gz, bx, by, bz = (int(v) for v in w[3:9])
            assert 1 <= gx < 1 << 31 and 1 <= gy < 65536 and gz == by == bz == 1 and 1 <= bx <= 1024 and gx * bx < 1 << 32, (name, kw, w)
            assert int(w[9]) <= 160 << 10


def test_what_is_not_asked_for_is_not_needed(record):
    for kw, launches in ((dict(dx=None, W1=None), 2), (dict(dx=None, W1=None, dW1=None, x=None, xk=NOTHING), 2), (dict(dW1=None, dW2=None, x=None, xk=NOTHING), 2),
                         (dict(dW1=None, x=None, xk=NOTHING), 3), (dict(), 3), (dict(xk=EIGHT), 4)):
        (st, lines), = record([("grad", kw)])
        assert st == 0 and len(lines) == launches, kw


@pytest.mark.parametrize("keep", [NOTHING, FULL, EIGHT])
def test_the_counters_of_a_cut_product_are_cleared(record, keep):
    """By the first product's launch, or by one of their own where that is the kernel for few rows, which clears nothing."""
    kw = dict(E=600, rows=1100, d=64, F=2048, dtype=BF16, ws=P, nb=BIG, keep=keep, pre=P if keep else None)
    (st, lines), = record([("ffn", kw)])
    names = [w[2] for w in lines]
    assert st == 0 and "gemm_bf16_kernel" in names[-1]
    assert ("zero_ints" in names[1]) == ("gated_few_kernel" in names[0]), names
    assert ("gated_few_kernel" in names[0]) == (keep != EIGHT)


def test_dx_that_takes_the_place_of_an_input_is_made_last(record):
    """Else its launch may have the weights' gradients beside it."""
    for kw, launches in ((dict(dx=2 * P), 2), (dict(dx=2 * P, x=2 * P), 3), (dict(dx=2 * P, dy=2 * P), 3), (dict(dx=2 * P, xk=EIGHT), 3)):
        (st, lines), = record([("grad", kw)])
        assert st == 0 and len(lines) == launches, kw


def test_gradients_of_no_rows_are_written(record):
    none = dict(rows=0, dy=None, x=None, pre=None, W1=None, W2=None, ws=None, nb=0)
    for kw in (none, dict(none, dW1=None), dict(none, dW2=None), dict(none, dx=None)):
        (st, lines), = record([("grad", kw)])
        assert st == 0 and len(lines) == 1


# ---- binding ----------------------------------------------------------------------------------------


class OnGpu:
    """A host tensor that says it lies on a GPU: nothing that is called here reads it."""

    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index


R, E, D, HID = 6, 2, 64, 96


def tensors():
    import torch
    f = lambda *s: torch.zeros(s)  # noqa: E731
    return dict(x_perm=f(R, D), dy_perm=f(R, D), x=f(R, D), hidden=f(R, HID), y_perm=f(R, D), dx_perm=f(R, D), pre=f(R, 2 * HID), W1=f(E, 2 * HID, D),
                W2=f(E, D, HID), dW1=f(E, 2 * HID, D), dW2=f(E, D, HID), offsets=torch.zeros(E + 1, dtype=torch.int32), workspace=f(64),
                q=torch.zeros(R, 80, dtype=torch.uint8), n_rows=torch.zeros(1, dtype=torch.int32))


ARGS = {
    "scmoe_gated_ffn": ("x_perm", "offsets", "W1", "W2", "hidden", "y_perm", "pre", "workspace"),
    "scmoe_gated_ffn_backward": ("dy_perm", "x", "pre", "offsets", "W1", "W2", "dx_perm", "dW1", "dW2", "workspace"),
    "scmoe_checkpoint_pack": ("x", "q", "n_rows"),
    "scmoe_checkpoint_unpack": ("q", "x", "n_rows"),
}


@pytest.fixture
def library(monkeypatch):
    from paper_2404_05019_amd import binding as B

    class Library:
        def __init__(self):
            self.called = []

        def __getattr__(self, name):
            return lambda *a: self.called.append((name, a)) or 0
    it = Library()
    monkeypatch.setattr(B, "lib", lambda: it)
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    return it


def call(name, **other):
    from paper_2404_05019_amd import binding as B
    args = {n: OnGpu(t) for n, t in tensors().items() if n in ARGS[name]}
    args.update(other)
    if "gated" in name:
        args["max_rows"] = R
    getattr(B, name)(stream=0, **args)


@pytest.mark.parametrize("name", ARGS)
def test_tensors_that_fit_are_taken(library, name):
    call(name)
    assert [n for n, _ in library.called] == [name]


@pytest.mark.parametrize("name,n", [(name, n) for name in ARGS for n in ARGS[name]])
def test_a_tensor_on_another_gpu_is_refused(library, name, n):
    with pytest.raises(TypeError, match="on the GPU"):
        call(name, **{n: OnGpu(tensors()[n], 1)})
    assert library.called == []


@pytest.mark.parametrize("name,n", [(name, n) for name in ARGS for n in ARGS[name] if n != "workspace"])
def test_a_tensor_of_another_type_is_refused(library, name, n):
    import torch
    with pytest.raises(TypeError):
        call(name, **{n: OnGpu(tensors()[n].to(torch.float16))})
    assert library.called == []


@pytest.mark.parametrize("name,n", [(name, n) for name in ARGS for n in ARGS[name] if n not in ("workspace", "offsets", "n_rows")
                                    and not ("checkpoint" in name and n == "x")])       # (its shape says how many rows there are, how wide)
def test_a_tensor_that_is_too_small_is_refused(library, name, n):
    """A row, an expert or some columns less."""
    t = tensors()[n]
    for cut in (t[1:], t[..., :-32].contiguous()):
        if name == "scmoe_gated_ffn_backward" and n in ("W2", "dy_perm") or n == "W2":
            continue                                                                     # (W2 says how many experts there are, and both widths)
        with pytest.raises(TypeError):
            call(name, **{n: OnGpu(cut)})
    if n == "W2":
        with pytest.raises(TypeError):
            call(name, W2=OnGpu(t[1:]))
    assert library.called == []


def test_kept_activations_say_how_they_are_kept(library):
    import torch
    for t, kind in ((None, NOTHING), (tensors()["pre"], FULL), (torch.zeros(2 * R, 112, dtype=torch.uint8), EIGHT)):
        call("scmoe_gated_ffn", pre=None if t is None else OnGpu(t))
        assert library.called[-1][1][17] == kind
    eight = dict(x=OnGpu(torch.zeros(R, 80, dtype=torch.uint8)), pre=OnGpu(torch.zeros(2 * R, 112, dtype=torch.uint8)))
    call("scmoe_gated_ffn_backward", **eight)
    assert library.called[-1][1][5] == EIGHT and library.called[-1][1][8] == EIGHT
    library.called.clear()
    for n, rows, ld in (("x", R - 1, 80), ("x", R, 64), ("pre", 2 * R - 1, 112), ("pre", 2 * R, 96)):
        with pytest.raises(TypeError):
            call("scmoe_gated_ffn_backward", **dict(eight, **{n: OnGpu(torch.zeros(rows, ld, dtype=torch.uint8))}))
    assert library.called == []


if __name__ == "__main__":
    _child(sys.argv[1], sys.argv[2], json.loads(sys.argv[3]))
