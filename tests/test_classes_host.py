"""Argument checks of the class losses: refused, or host arithmetic, before the GPU is touched."""
import ctypes as C

import pytest

A = 1 << 20     # an address that passes for aligned device memory; nothing dereferences it


@pytest.fixture(scope="module")
def B():
    from paper_2112_08541_amd import binding
    return binding


@pytest.fixture(scope="module")
def L(B):
    return B.load_library()


def loss(B, dtype=0, in_dim=8, classes=5, top=3, temperature=2.0):
    return B.ClassLossStruct(dtype, in_dim, classes, top, temperature)


def forward(L, s, n=4, x=A, xs=8, w=A, b=A, labels=A, tc=A, ts=A, out=A, tout=A, saved=A, ws=A, nbytes=1 << 40):
    return L.bgl_class_loss_forward(C.byref(s) if s else None, n, x, xs, w, b, labels, tc, ts, out, tout, saved, ws, nbytes, None)


def backward(L, s, n=4, x=A, xs=8, w=A, b=A, labels=A, tc=A, ts=A, saved=A, dx=A, dxs=8, dw=A, db=A, ws=A, nbytes=1 << 40):
    return L.bgl_class_loss_backward(C.byref(s) if s else None, n, x, xs, w, b, labels, tc, ts, saved, 1.0, 1.0, dx, dxs, dw, db, ws, nbytes, None)


def room(B, L, s, n):
    f, b = C.c_size_t(), C.c_size_t()
    assert L.bgl_class_loss_workspace_bytes(C.byref(s), n, C.byref(f), C.byref(b)) == B.BGL_OK
    return f.value, b.value


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), "EINVAL"), (dict(dtype=-1), "EINVAL"), (dict(in_dim=0), "EINVAL"), (dict(classes=0), "EINVAL"), (dict(top=-1), "EINVAL"),
    (dict(temperature=0.0), "EINVAL"), (dict(temperature=-1.0), "EINVAL"), (dict(temperature=float("nan")), "EINVAL"), (dict(temperature=2000.0), "EINVAL"),
    (dict(in_dim=16385), "EUNSUPPORTED"), (dict(classes=(1 << 24) + 1), "EUNSUPPORTED"), (dict(top=1025), "EUNSUPPORTED")])
def test_losses_out_of_range_are_refused(B, L, change, code):
    s, want, n = loss(B, **change), getattr(B, "BGL_" + code), C.c_size_t()
    assert L.bgl_class_loss_workspace_bytes(C.byref(s), 10, C.byref(n), None) == want
    assert forward(L, s) == want
    assert backward(L, s) == want
    assert L.bgl_last_error()


def test_arguments_are_checked(B, L):
    s, h, plain = loss(B), loss(B, dtype=1), loss(B, top=0)
    none = dict(tc=None, ts=None)
    bad = [forward(L, None), forward(L, s, n=-1), forward(L, s, n=1 << 31), forward(L, s, x=None), forward(L, s, xs=7), forward(L, s, x=A + 2),
           forward(L, s, w=None), forward(L, s, w=A + 2), forward(L, s, b=A + 1), forward(L, s, labels=A + 2), forward(L, s, tc=A + 1), forward(L, s, ts=A + 2),
           forward(L, s, tc=None), forward(L, s, ts=None), forward(L, plain), forward(L, s, labels=None, out=None, tout=None, **none),
           forward(L, s, labels=None), forward(L, s, **none), forward(L, s, out=A + 2), forward(L, s, tout=A + 1), forward(L, s, saved=A + 2),
           forward(L, s, ws=None), forward(L, s, ws=A + 128), forward(L, h, x=A + 1),
           backward(L, None), backward(L, s, n=-1), backward(L, s, saved=None), backward(L, s, saved=A + 2), backward(L, s, dxs=7), backward(L, s, dx=A + 2),
           backward(L, s, dw=A + 2), backward(L, s, db=A + 2), backward(L, s, dw=None), backward(L, s, dx=None, dw=None, db=None), backward(L, s, ws=None),
           backward(L, s, ws=A + 4), backward(L, s, labels=None, **none), backward(L, plain)]
    assert bad == [B.BGL_EINVAL] * len(bad)
    assert forward(L, s, xs=1 << 31) == B.BGL_EUNSUPPORTED
    assert forward(L, s, nbytes=8) == B.BGL_ECAPACITY and backward(L, s, nbytes=8) == B.BGL_ECAPACITY
    assert forward(L, s, n=0, x=None, w=None) == B.BGL_OK      # nothing to do
    assert L.bgl_class_loss_workspace_bytes(C.byref(s), 1, None, None) == B.BGL_EINVAL


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("in_dim,classes", [(100, 2), (8, 150), (640, 511), (128, 1_001), (512, 1_024), (256, 5_000), (64, 16_384), (500, 16_385), (256, 50_001),
                                            (512, 65_536), (128, 1 << 20), (16_384, 300)])
def test_a_workspace_for_many_rows_is_enough_for_fewer(B, L, dtype, in_dim, classes):
    s = loss(B, dtype, in_dim, classes, top=7)
    sizes = sorted(set([0, 1, 2, 5] + [k + d for k in (16, 64, 100, 128, 500, 512, 640, 1000, 1024, 1500, 2048, 3000, 4096, 5000, 8192, 10_000, 16_384, 20_000, 32_768,
                                                       65_536, 100_000, 204_800, 1_000_000, 1 << 22) for d in (-1, 0, 1)]))
    last = (0, 0)
    for n in sizes:
        have = room(B, L, s, n)
        assert have[0] >= last[0] and have[1] >= last[1], n
        last = have
