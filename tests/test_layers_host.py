"""Argument checks of the layer calls: everything here is refused, or is host arithmetic, before the GPU is touched."""
import ctypes as C

import numpy as np
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2112_08541_amd import binding
    return binding


@pytest.fixture(scope="module")
def L(B):
    return B.load_library()


A = 1 << 20     # an address that passes for aligned device memory; nothing dereferences it


def layer(B, dtype=0, activation=0, residual=0, in_dim=8, out_dim=4, groups=0):
    return B.LinearStruct(dtype, activation, residual, in_dim, out_dim, groups)


def forward(B, L, l, n=4, rows=None, offsets=None, x=A, xs=8, w=A, b=None, r=None, rs=0, y=A, ys=4, s=None, ss=0):
    return L.bgl_linear_forward(C.byref(l) if l else None, n, rows, offsets, x, xs, w, b, r, rs, y, ys, s, ss, None)


def backward(B, L, l, n=4, rows=None, offsets=None, dy=A, ys=4, x=A, xs=8, w=A, s=None, ss=0, dx=A, dxs=8, dw=A, db=None, dr=None,
             drs=0, ws=A, nbytes=1 << 30):
    return L.bgl_linear_backward(C.byref(l), n, rows, offsets, dy, ys, x, xs, w, s, ss, dx, dxs, dw, db, dr, drs, ws, nbytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), "EINVAL"), (dict(dtype=-1), "EINVAL"), (dict(activation=4), "EINVAL"), (dict(activation=-1), "EINVAL"),
    (dict(residual=3), "EINVAL"), (dict(in_dim=0), "EINVAL"), (dict(out_dim=-5), "EINVAL"), (dict(groups=-1), "EINVAL"),
    (dict(in_dim=16385), "EUNSUPPORTED"), (dict(out_dim=1 << 30), "EUNSUPPORTED"), (dict(groups=1025), "EUNSUPPORTED")])
def test_layers_out_of_range_are_refused(B, L, change, code):
    l = layer(B, **change)
    want = getattr(B, "BGL_" + code)
    n = C.c_size_t()
    assert L.bgl_linear_workspace_bytes(C.byref(l), 10, C.byref(n)) == want
    assert forward(B, L, l, offsets=A) == want
    assert backward(B, L, l, offsets=A) == want
    assert L.bgl_last_error()


def test_forward_arguments_are_checked(B, L):
    plain, before, grouped = layer(B), layer(B, residual=1), layer(B, groups=3)
    bad = [forward(B, L, None), forward(B, L, plain, n=-1), forward(B, L, plain, n=1 << 31), forward(B, L, plain, x=None),
           forward(B, L, plain, y=None), forward(B, L, plain, w=None), forward(B, L, plain, xs=7), forward(B, L, plain, ys=3),
           forward(B, L, plain, x=A + 2), forward(B, L, plain, w=A + 1), forward(B, L, plain, b=A + 2), forward(B, L, plain, r=A, rs=4),
           forward(B, L, before), forward(B, L, before, r=A, rs=3), forward(B, L, plain, s=A, ss=3), forward(B, L, plain, offsets=A),
           forward(B, L, plain, rows=A), forward(B, L, grouped), forward(B, L, grouped, offsets=A + 2),
           forward(B, L, layer(B, dtype=1), x=A + 1)]
    assert bad == [B.BGL_EINVAL] * len(bad)
    assert forward(B, L, plain, n=0, x=None, y=None) == B.BGL_OK      # nothing to do


def test_backward_arguments_are_checked(B, L):
    plain, relu, after = layer(B), layer(B, activation=1), layer(B, residual=2)
    bad = [backward(B, L, plain, dy=None), backward(B, L, plain, ys=3), backward(B, L, plain, x=None), backward(B, L, plain, w=None),
           backward(B, L, plain, dxs=7), backward(B, L, plain, dw=None, db=A), backward(B, L, relu), backward(B, L, relu, s=A, ss=3),
           backward(B, L, after, dr=A, drs=4), backward(B, L, plain, dr=A, drs=4), backward(B, L, plain, ws=None),
           backward(B, L, plain, ws=A + 128), backward(B, L, layer(B, residual=1), dr=A, drs=3)]
    assert bad == [B.BGL_EINVAL] * len(bad)
    assert backward(B, L, plain, nbytes=16) == B.BGL_ECAPACITY
    assert b"16 bytes" in L.bgl_last_error()


def test_workspace_sizes_grow_with_the_call_and_stay_bounded(B, L):
    def need(n, **k):
        out = C.c_size_t()
        assert L.bgl_linear_workspace_bytes(C.byref(layer(B, **k)), n, C.byref(out)) == B.BGL_OK
        return out.value
    wide = dict(in_dim=512, out_dim=256)
    assert need(0, **wide) > 0
    # partial sums: at most some 512 tiles of 128 x 128 and one more for each group, however many rows there are
    for n in (1, 1000, 302_709, 2**31 - 1):
        assert need(n, **wide) <= 600 * 128 * 128 * 4 * 2
    # an activation keeps dz too
    assert need(1000, activation=1, **wide) >= need(1000, **wide) + 1000 * 256 * 4
    assert need(2**31 - 1, in_dim=16384, out_dim=16384) > 0
    out = C.c_size_t()
    assert L.bgl_linear_workspace_bytes(C.byref(layer(B)), -1, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_linear_workspace_bytes(C.byref(layer(B)), 1, None) == B.BGL_EINVAL
    assert L.bgl_linear_workspace_bytes(None, 1, C.byref(out)) == B.BGL_EINVAL


def test_grouping_arguments_are_checked(B, L):
    out = C.c_size_t()
    assert L.bgl_group_rows_workspace_bytes(100, 8, C.byref(out)) == B.BGL_OK and out.value >= 200
    assert L.bgl_group_rows_workspace_bytes(100, 0, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_group_rows_workspace_bytes(-1, 8, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_group_rows_workspace_bytes(100, 1025, C.byref(out)) == B.BGL_EUNSUPPORTED
    assert L.bgl_group_rows_workspace_bytes(100, 8, None) == B.BGL_EINVAL

    def call(of=A, nodes=100, ids=None, n=100, groups=8, rows=A, offsets=A, ws=A, nbytes=1 << 20):
        return L.bgl_group_rows(of, nodes, ids, n, groups, rows, offsets, ws, nbytes, None)
    bad = [call(of=None), call(rows=None), call(offsets=None), call(ws=None), call(ws=A + 16), call(nodes=99), call(nodes=-1, ids=A),
           call(n=-1), call(groups=0), call(of=A + 2), call(ids=A + 1), call(rows=A + 2), call(offsets=A + 3)]
    assert bad == [B.BGL_EINVAL] * len(bad)
    assert call(groups=2000) == B.BGL_EUNSUPPORTED
    assert call(nbytes=100) == B.BGL_ECAPACITY


def test_orthogonalising_arguments_are_checked(B, L):
    out = C.c_size_t()
    assert L.bgl_orthogonalize_workspace_bytes(2, 64, 32, 0, C.byref(out)) == B.BGL_OK and out.value > 2 * 64 * 32 * 4
    assert L.bgl_orthogonalize_workspace_bytes(2, 0, 32, 0, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_orthogonalize_workspace_bytes(-2, 4, 32, 0, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_orthogonalize_workspace_bytes(2, 4, 32, 7, C.byref(out)) == B.BGL_EINVAL
    assert L.bgl_orthogonalize_workspace_bytes(2, 4, 16385, 0, C.byref(out)) == B.BGL_EUNSUPPORTED
    assert L.bgl_orthogonalize_workspace_bytes(65536, 4, 4, 0, C.byref(out)) == B.BGL_EUNSUPPORTED

    def call(u=A, um=2048, ur=32, batch=2, rows=64, cols=32, dtype=0, steps=5, co=(3.4445, -4.775, 2.0315), eps=1e-7, o=A, om=2048,
             orow=32, ws=A, nbytes=1 << 30):
        co = None if co is None else np.asarray(co, dtype=np.float32)
        return L.bgl_orthogonalize(u, um, ur, batch, rows, cols, dtype, steps, None if co is None else co.ctypes.data, eps, o, om, orow,
                                   ws, nbytes, None)
    bad = [call(u=None), call(o=None), call(u=A + 2), call(ur=31), call(orow=31), call(um=2047), call(om=100), call(steps=0),
           call(steps=65), call(co=None), call(eps=-1.0), call(eps=float("nan")), call(ws=None), call(ws=A + 8), call(rows=-1)]
    assert bad == [B.BGL_EINVAL] * len(bad)
    assert call(nbytes=1000) == B.BGL_ECAPACITY
    # coefficients whose steps leave the range the split halves are laid out for
    for co in ((10.0, 0.0, 0.0), (3.4445, 4.775, 2.0315), (float("nan"), 0.0, 0.0), (float("inf"), 0.0, 0.0)):
        assert call(co=co) == B.BGL_EUNSUPPORTED, co
    assert call(batch=0, u=None, o=None, ws=None) == B.BGL_OK


def test_the_binding_names_what_the_header_numbers(B):
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bgl.h")).read()
    define = {k: int(v) for k, v in re.findall(r"#define (BGL_\w+) \(?(-?\d+)\)?", text)}
    assert (B.BGL_F32, B.BGL_BF16) == (define["BGL_F32"], define["BGL_BF16"])
    assert (B.BGL_MAX_GROUPS, B.BGL_MAX_DIM) == (define["BGL_MAX_GROUPS"], define["BGL_MAX_DIM"])
    assert B.ACTIVATIONS == {k[8:].lower(): v for k, v in define.items() if k.startswith("BGL_ACT_")}
    assert B.RESIDUALS == {k[13:].lower(): v for k, v in define.items() if k.startswith("BGL_RESIDUAL_")}


@pytest.mark.parametrize("groups", [1, 8, 100, 1024])
def test_a_workspace_for_many_rows_is_enough_for_fewer(B, L, groups):
    """Around every size at which the rows of a grouping tile, or the tiles or shares of a layer's gradients, change."""
    edges = [0, 1, 63, 64, 65, 2047, 2048, 2049, 8191, 8192, 8193]
    edges += [k * 131_072 + d for k in range(1, 24) for d in (-512, -1, 0, 1, 511, 512)] + [2**31 - 1 - 131_072, 2**31 - 1]

    def grows(need):
        sizes = [need(n) for n in sorted(edges)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), [n for n, a, b in zip(sorted(edges), sizes, sizes[1:]) if a > b]

    def grouping(n):
        out = C.c_size_t()
        assert L.bgl_group_rows_workspace_bytes(n, groups, C.byref(out)) == B.BGL_OK
        return out.value
    grows(grouping)
    for dtype in (0, 1):
        for activation in range(4):
            l = layer(B, dtype, activation, 0, 100, 256, groups)

            def gradients(n):
                out = C.c_size_t()
                assert L.bgl_linear_workspace_bytes(C.byref(l), n, C.byref(out)) == B.BGL_OK
                return out.value
            grows(gradients)


def test_training_refuses_a_pipeline_whose_sampling_it_cannot_order():
    from paper_2112_08541_amd import sage
    from paper_2112_08541_amd.pipeline import NativePipeline
    pipe = object.__new__(NativePipeline)
    pipe._tier = object()
    with pytest.raises(ValueError, match="tier"):
        sage.train(pipe, None, None, None, 0, None, None)
