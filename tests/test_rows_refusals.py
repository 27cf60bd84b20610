"""What the operators on node rows refuse, before anything is enqueued; no GPU is needed to be refused."""
import ctypes
import struct

import pytest

torch = pytest.importorskip("torch")

import paper_2301_00391_amd as pipad

INVALID, TOO_LARGE, SCRATCH = -1, -4, -6
P = 4096  # stands for an aligned device address: nothing that is refused looks at it


def pointers(k, at=P):
    return struct.pack(f"{k}P", *[at] * k)


def norm(F=8, post=1, pre=1, eps=1e-5, scale=0, w_post=0, b_post=0, w_pre=0, b_pre=0):
    return struct.pack("iiif5P", F, post, pre, eps, scale, w_post, b_post, w_pre, b_pre)


def forward(c=None, n=4, k=2, R=1, ldr=8, B=1, ldb=8, gate=1, ldg=8, R_out=1, ldro=8, Z=1, ldz=8, **kw):
    a = [pointers(max(1, min(k, 32))) if x == 1 else x for x in (R, B, gate, R_out, Z)]
    return pipad.load_library().pipad_residual_norm(norm(**kw) if c is None else c, n, k, a[0], ldr, a[1], ldb, a[2], ldg, a[3], ldro, a[4], ldz, None)


@pytest.mark.parametrize("status,kw", [
    (INVALID, {"F": 0}), (INVALID, {"F": -3}), (INVALID, {"post": 3}), (INVALID, {"pre": -1}), (INVALID, {"eps": -1.0}), (INVALID, {"eps": float("nan")}),
    (INVALID, {"n": -1}), (INVALID, {"k": 0}), (INVALID, {"k": 33}), (INVALID, {"R": None}), (INVALID, {"R_out": None, "Z": None}),
    (INVALID, {"ldr": 7}), (INVALID, {"ldb": 7}), (INVALID, {"ldg": 7}), (INVALID, {"ldro": 7}), (INVALID, {"ldz": 7}),
    (INVALID, {"B": None}), (INVALID, {"B": None, "gate": None, "R_out": None}), (INVALID, {"B": None, "gate": None, "post": 0}),
    (INVALID, {"B": None, "gate": None, "post": 0, "R_out": None, "scale": P}), (INVALID, {"B": None, "post": 0, "R_out": None}),
    (INVALID, {"post": 0, "w_post": P}), (INVALID, {"post": 0, "b_post": P}), (INVALID, {"pre": 0}), (INVALID, {"pre": 0, "Z": None, "w_pre": P}),
    (INVALID, {"pre": 0, "Z": None, "b_pre": P}), (INVALID, {"R": pointers(2, 0)}), (INVALID, {"Z": struct.pack("2P", P, 0)}),
    (TOO_LARGE, {"F": 4097, "ldr": 8192, "ldb": 8192, "ldg": 8192, "ldro": 8192, "ldz": 8192}), (TOO_LARGE, {"ldz": 1 << 38}), (TOO_LARGE, {"ldr": 1 << 62})])
def test_residual_norm(status, kw):
    assert forward(**kw) == status


def test_residual_norm_of_nothing():
    assert forward(n=0) == 0 and forward(n=0, R=pointers(2, 0)) == 0
    assert pipad.load_library().pipad_residual_norm(None, 0, 1, None, 0, None, 0, None, 0, None, 0, None, 0, None) == INVALID


def backward(n=4, k=2, R=1, ldr=8, B=1, ldb=8, gate=1, ldg=8, dRo=1, lddro=8, dZ=1, lddz=8, dR=1, lddr=8, dB=1, lddb=8, dgate=1, lddg=8, grads=1, ws=P,
             nbytes=1 << 30, **kw):
    a = [pointers(max(1, min(k, 32))) if x == 1 else x for x in (R, B, gate, dRo, dZ, dR, dB, dgate)]
    lds = (ldr, ldb, ldg, lddro, lddz, lddr, lddb, lddg)
    g = struct.pack("5P", *[P] * 5) if grads else None
    return pipad.load_library().pipad_residual_norm_backward(norm(**kw), n, k, *[x for pair in zip(a, lds) for x in pair], g, ws, nbytes, None)


@pytest.mark.parametrize("status,kw", [
    (INVALID, {"R": None}), (INVALID, {"dRo": None, "dZ": None}), (INVALID, {"pre": 0}), (INVALID, {"gate": None}), (INVALID, {"B": None}),
    (INVALID, {"B": None, "gate": None, "post": 0, "dB": None}), (INVALID, {"dR": None, "dB": None, "dgate": None, "grads": 0}),
    (INVALID, {"ws": None}), (INVALID, {"ws": P + 8}), (SCRATCH, {"nbytes": 16}), (INVALID, {"lddz": 3}), (INVALID, {"lddr": 7}), (INVALID, {"lddb": 7}),
    (INVALID, {"lddg": 7}), (INVALID, {"lddro": 7}), (INVALID, {"dR": pointers(2, 0)}), (TOO_LARGE, {"lddb": 1 << 40}), (INVALID, {"k": 33})])
def test_residual_norm_backward(status, kw):
    assert backward(**kw) == status


def block(F=8, hidden=20, Fo=6, act=3, Wg=P, Wu=P, Wd=P, ldwg=20, ldwu=20, ldwd=6, bg=0, bu=0, bd=0):
    return struct.pack("4i3P3q3P", F, hidden, Fo, act, Wg, Wu, Wd, ldwg, ldwu, ldwd, bg, bu, bd)


BAD_BLOCKS = [(INVALID, {"F": 0}), (INVALID, {"hidden": 0}), (INVALID, {"Fo": -1}), (INVALID, {"act": 4}), (INVALID, {"act": -1}), (INVALID, {"Wg": 0}),
              (INVALID, {"Wu": 0}), (INVALID, {"Wd": 0}), (INVALID, {"ldwg": 19}), (INVALID, {"ldwu": 19}), (INVALID, {"ldwd": 5}),
              (TOO_LARGE, {"hidden": 1 << 16, "ldwg": 1 << 16, "ldwu": 1 << 16}), (TOO_LARGE, {"Fo": 1 << 16, "ldwd": 1 << 16}),
              (TOO_LARGE, {"F": 1 << 16}), (TOO_LARGE, {"ldwd": 1 << 40})]


@pytest.mark.parametrize("status,kw", BAD_BLOCKS)
def test_gated_ff_blocks(status, kw):
    lib = pipad.load_library()
    ops = [pointers(2), 1 << 17]
    assert lib.pipad_gated_ff(block(**kw), 4, 2, *ops, *ops, P, 1 << 40, None) == status
    assert lib.pipad_gated_ff_backward(block(**kw), 4, 2, *ops, *ops, *ops, None, P, 1 << 40, None) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, {"n": -1}), (INVALID, {"k": 0}), (INVALID, {"k": 33}), (INVALID, {"X": None}), (INVALID, {"Y": None}), (INVALID, {"ldx": 7}),
    (INVALID, {"ldy": 5}), (INVALID, {"X": pointers(2, 0)}), (INVALID, {"ws": None}), (INVALID, {"ws": P + 4}), (SCRATCH, {"nbytes": 100}),
    (TOO_LARGE, {"ldx": 1 << 39}), (TOO_LARGE, {"ldy": 1 << 41}), (TOO_LARGE, {"n": (1 << 29) + 1})])
def test_gated_ff_operands(status, kw):
    lib = pipad.load_library()
    at = dict(n=4, k=2, X=pointers(2), ldx=8, Y=pointers(2), ldy=6, ws=P, nbytes=1 << 40)
    at.update(kw)
    assert lib.pipad_gated_ff(block(), *(at[q] for q in ("n", "k", "X", "ldx", "Y", "ldy", "ws", "nbytes")), None) == status
    dx = [pointers(2), 8]
    assert lib.pipad_gated_ff_backward(block(), *(at[q] for q in ("n", "k", "X", "ldx", "Y", "ldy")), *dx, None, at["ws"], at["nbytes"], None) == status


def test_gated_ff_of_many_wide_rows():
    lib, got = pipad.load_library(), ctypes.c_size_t()
    for sizes, most in (({}, 1 << 30), ({"F": 257}, 1 << 28), ({"Fo": 257, "ldwd": 257}, 1 << 28)):
        for backward in (0, 1):
            assert lib.pipad_gated_ff_workspace(block(**sizes), most // 32, 32, backward, ctypes.byref(got)) == 0
            assert lib.pipad_gated_ff_workspace(block(**sizes), most // 32 + 1, 32, backward, ctypes.byref(got)) == TOO_LARGE


def test_gated_ff_gradients():
    lib = pipad.load_library()
    x, y = [pointers(2), 8], [pointers(2), 6]
    grads = lambda *v: struct.pack("3P3q3P", *v)  # noqa: E731
    call = lambda dx, g, ws=P, nbytes=1 << 40: lib.pipad_gated_ff_backward(block(), 4, 2, *x, *y, *dx, g, ws, nbytes, None)  # noqa: E731
    assert call([None, 0], None) == INVALID
    assert call([pointers(2), 7], None) == INVALID
    for bad in ((19, 20, 6), (20, 19, 6), (20, 20, 5)):
        assert call([None, 0], grads(P, P, P, *bad, 0, 0, 0)) == INVALID
    assert call([None, 0], grads(P, P, P, 20, 1 << 40, 6, 0, 0, 0)) == TOO_LARGE
    assert call([None, 0], grads(P, P, P, 20, 20, 6, 0, 0, 0), nbytes=64) == SCRATCH
    assert call([None, 0], grads(P, P, P, 20, 20, 6, 0, 0, 0), ws=None) == INVALID


def test_sizes_asked_for():
    lib, got = pipad.load_library(), ctypes.c_size_t()
    assert lib.pipad_gated_ff_workspace(block(), 4, 2, 2, ctypes.byref(got)) == INVALID
    assert lib.pipad_gated_ff_workspace(block(), 4, 2, 0, None) == INVALID
    assert lib.pipad_gated_ff_workspace(None, 4, 2, 0, ctypes.byref(got)) == INVALID
    assert lib.pipad_gated_ff_workspace(block(Wg=0, ldwg=0), 4, 2, 0, ctypes.byref(got)) == 0 and got.value > 0
    assert lib.pipad_residual_norm_workspace(0, 4, 2, ctypes.byref(got)) == INVALID
    assert lib.pipad_residual_norm_workspace(8, 4, 2, None) == INVALID
    assert lib.pipad_residual_norm_workspace(4097, 4, 2, ctypes.byref(got)) == TOO_LARGE
    assert lib.pipad_residual_norm_workspace(8, 0, 2, ctypes.byref(got)) == 0 and got.value == 0


def test_tensors_that_do_not_fit():
    x, w, v = torch.zeros((3, 2, 4)), torch.zeros((4, 4)), torch.zeros(4)
    for call in (lambda: pipad.gated_ff(x, w, w, w), lambda: pipad.gated_ff([x[:, 0]], w, w, w), lambda: pipad.gated_ff([], w, w, w),
                 lambda: pipad.gated_ff(v, w, w, w), lambda: pipad.residual_norm(x), lambda: pipad.residual_norm([v]),
                 lambda: pipad.gated_ff_backward(x, x, w, w, w), lambda: pipad.residual_norm_backward(x, x, x),
                 lambda: pipad.residual_norm([torch.zeros((3, 4))] * 33)):
        with pytest.raises(ValueError):
            call()
