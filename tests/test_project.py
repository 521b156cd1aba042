"""Refusals of the dense projection and of the gradient norm and clipping, on the host.

Every call fails host-side validation, so nothing reaches the GPU; the
pointers are placeholders that are never dereferenced.
"""
import ctypes

import pytest
import torch

from paper_2608_23794_amd import binding as mb
from paper_2608_23794_amd.layer import ProjectLayer, clip_gradients, gradient_norm

FAKE = 0x10000
GIB = 1 << 30


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(mb.LIB_PATH):
        from paper_2608_23794_amd import build
        build.build()
    return mb.load()


def desc(**kw):
    d = dict(B=2, C=64, H=8, W=8, O=48, dtype=mb.MOCE_BF16, layout=mb.MOCE_NHWC, act=mb.MOCE_ACT_RELU)
    d.update(kw)
    return mb.make_project_desc(**d)


def project(d, x=FAKE, weight=FAKE, scale=None, shift=None, residual=None, y=FAKE, z=None, ws=FAKE, n=GIB):
    return mb.raw_status("moce_project", ctypes.byref(d) if d else None, x, weight, scale, shift, residual, y, z, ws,
                         n, None)


def backward(d, x=FAKE, weight=FAKE, scale=None, z=FAKE, dy=FAKE, ws=FAKE, n=GIB, grads=True, **kw):
    g = mb.make_project_grads(**(kw or {"dx": FAKE}))
    return mb.raw_status("moce_project_backward", ctypes.byref(d) if d else None, x, weight, scale, z, dy,
                         ctypes.byref(g) if grads else None, ws, n, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), -2), (dict(C=0), -2), (dict(H=0), -2), (dict(W=-3), -2), (dict(O=0), -2), (dict(act=4), -2),
    (dict(act=-1), -2), (dict(dtype=2), -3), (dict(layout=2), -4), (dict(C=(1 << 20) + 1), -10),
    (dict(O=(1 << 20) + 1), -10), (dict(B=(1 << 29) + 1, H=1, W=1, C=1, O=1), -10), (dict(H=1 << 20, W=1 << 11), -10),
    (dict(C=1 << 16, H=1 << 8, W=1 << 8), -10), (dict(C=1 << 18, O=(1 << 17) + 1, B=1, H=1, W=1), -10), (dict(B=1 << 20, C=1 << 10, H=4, W=4), -10),
])
def test_descriptor(lib, change, code):
    d = desc(**change)
    assert project(d) == code
    assert backward(d) == code
    assert lib.moce_project_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.moce_project_backward_workspace_bytes(ctypes.byref(d)) == 0


def test_project_pointers(lib):
    d = desc(B=1, H=1, W=1, C=4096)
    need = lib.moce_project_workspace_bytes(ctypes.byref(d))
    assert project(None) == -1
    assert project(d, x=None) == -1 and project(d, weight=None) == -1 and project(d, y=None) == -1
    assert project(d, z=FAKE) == -2            # z is y
    for name in ("x", "weight", "y", "residual", "z"):
        assert project(d, **{name: FAKE + 8}) == -8
    assert project(d, scale=FAKE + 2) == -8 and project(d, shift=FAKE + 2) == -8
    if need:
        assert project(d, ws=None) == -7 and project(d, n=need - 256) == -7 and project(d, ws=FAKE + 16) == -8


def test_backward_pointers(lib):
    d = desc()
    need = lib.moce_project_backward_workspace_bytes(ctypes.byref(d))
    assert need > 0
    assert backward(None) == -1 and backward(d, grads=False) == -1
    assert backward(d, x=None) == -1 and backward(d, weight=None) == -1 and backward(d, dy=None) == -1
    assert backward(d, z=None) == -1
    assert backward(d, dscale=FAKE) == -1      # no scale
    for act in (mb.MOCE_ACT_GELU, mb.MOCE_ACT_SILU):
        assert backward(desc(act=act), scale=FAKE, dscale=FAKE) == -10
    for name in ("x", "weight", "z", "dy"):
        assert backward(d, **{name: FAKE + 8}) == -8
    for name in ("dx", "dweight", "dresidual"):
        assert backward(d, **{name: FAKE + 8}) == -8
    assert backward(d, dshift=FAKE + 2) == -8 and backward(d, scale=FAKE, dscale=FAKE + 2) == -8
    assert backward(d, ws=None) == -7 and backward(d, n=need - 1) == -7 and backward(d, ws=FAKE + 16) == -8


def test_overlapping_tensors(lib):
    """No output, and no workspace, over another tensor: the first and the last of its bytes."""
    d = desc(act=mb.MOCE_ACT_NONE, C=60)          # x packed: a workspace
    M = 2 * 64
    size = {"x": M * 60 * 2, "y": M * 48 * 2, "weight": 48 * 60 * 2, "row": 48 * 4}
    size.update(z=size["y"], residual=size["y"], dy=size["y"], dresidual=size["y"], dx=size["x"], dweight=size["weight"])
    need, bneed = (f(ctypes.byref(d)) for f in (lib.moce_project_workspace_bytes, lib.moce_project_backward_workspace_bytes))
    apart = {n: FAKE + (i << 20) for i, n in enumerate(("x", "weight", "scale", "shift", "residual", "y", "z", "dy", "dx",
                                                         "dweight", "dscale", "dshift", "dresidual"))}
    ws = FAKE + (100 << 20)
    fwd = {n: apart[n] for n in ("x", "weight", "scale", "shift", "residual", "y", "z")}
    for out in ("y", "z"):
        for other in fwd:
            if other != out:
                assert need > 0
                last = size.get(other, size["row"]) - 1 & ~15
                if other != "residual":           # residual may be y or z, but only as a whole
                    assert project(d, ws=ws, n=need, **{**fwd, out: fwd[other]}) == -2, (out, other)
                assert project(d, ws=ws, n=need, **{**fwd, out: fwd[other] + last}) == -2, (out, other)
    for other in fwd:
        assert project(d, n=need, **{**fwd, "ws": fwd[other]}) == -2, other
    ins = {n: apart[n] for n in ("x", "weight", "scale", "dy")}
    outs = {n: apart[n] for n in ("dx", "dweight", "dscale", "dshift", "dresidual")}
    for out in outs:
        for other in {**ins, **outs}:
            if other != out:
                last = size.get(other, size["row"]) - 1 & ~15
                place = {**ins, **outs}[other]
                if (out, other) != ("dresidual", "dy"):
                    assert backward(d, ws=ws, n=bneed, **ins, **{**outs, out: place}) == -2, (out, other)
                assert backward(d, ws=ws, n=bneed, **ins, **{**outs, out: place + last}) == -2, (out, other)
    for other, place in {**ins, **outs}.items():
        assert backward(d, ws=place, n=bneed, **ins, **outs) == -2, other
    assert backward(desc(C=60), ws=ws, z=outs["dx"], **ins, **outs) == -2


def test_one_position_an_image_is_the_same_in_both_layouts(lib):
    sizes = {lib.moce_project_backward_workspace_bytes(ctypes.byref(desc(B=300, H=1, W=1, layout=l))) for l in (0, 1)}
    assert len(sizes) == 1


# ---- gradients -------------------------------------------------------------------

def gradients(*items):
    arr = (mb.moce_gradient * max(1, len(items)))()
    for g, it in zip(arr, items):
        g.src, g.dst, g.n, g.dtype = it
    return arr


def norm(arr, n, out=FAKE, ws=FAKE, nb=GIB):
    return mb.raw_status("moce_gradient_norm", ctypes.addressof(arr) if arr is not None else None, n, out, ws, nb, None)


def clip(arr, n, max_norm=1.0, out=FAKE, ws=FAKE, nb=GIB):
    return mb.raw_status("moce_gradient_clip", ctypes.addressof(arr) if arr is not None else None, n, max_norm, out, ws,
                         nb, None)


F32, BF16 = mb.MOCE_F32, mb.MOCE_BF16


@pytest.mark.parametrize("item,code", [
    ((FAKE, FAKE, -1, F32), -2), ((None, FAKE, 4, F32), -1), ((FAKE, FAKE, 4, 5), -3), ((FAKE + 2, FAKE + 2, 4, F32), -8),
    ((FAKE + 1, FAKE + 1, 4, BF16), -8), ((FAKE, FAKE, (1 << 40) + 1, BF16), -10),
])
def test_bad_gradient(lib, item, code):
    arr = gradients((FAKE << 8, FAKE << 8, 16, F32), item)
    assert norm(arr, 2) == code and clip(arr, 2) == code
    assert lib.moce_gradient_workspace_bytes(ctypes.addressof(arr), 2) == 0


def test_gradient_arguments(lib):
    arr = gradients((FAKE, FAKE, 16, F32))
    need = lib.moce_gradient_workspace_bytes(ctypes.addressof(arr), 1)
    assert need > 0 and lib.moce_gradient_workspace_bytes(None, 0) > 0
    assert norm(None, 1) == -1 and clip(None, 1) == -1 and norm(arr, -1) == -2 and clip(arr, -1) == -2
    for f in (norm, clip):
        assert f(arr, 1, out=None) == -1 and f(arr, 1, out=FAKE + 2) == -8
        assert f(arr, 1, ws=None) == -7 and f(arr, 1, nb=16) == -7 and f(arr, 1, ws=FAKE + 8) == -8
    for bad in (-1.0, float("inf"), float("nan")):
        assert clip(arr, 1, max_norm=bad) == -2
    assert clip(gradients((FAKE, None, 4, F32)), 1) == -1
    assert clip(gradients((FAKE, FAKE + 2, 4, F32)), 1) == -8


def test_overlapping_gradients():
    a, b = FAKE, FAKE + 4096
    assert clip(gradients((a, a, 16, F32), (a, a, 16, F32)), 2) == -2            # the same tensor twice
    assert clip(gradients((b, b, 16, F32), (a, a, 1025, F32)), 2) == -2          # the end of one inside another
    assert clip(gradients((a, a, 64, BF16), (a + 64, a + 64, 4, F32)), 2) == -2
    assert clip(gradients((a, a + 32, 16, F32)), 1) == -2                        # its own, partly
    assert clip(gradients((a, b, 16, F32), (b, a, 16, F32)), 2) == -2            # each other's
    assert clip(gradients((a, b, 16, F32), (a + 64, b + 60, 16, F32)), 2) == -2  # destinations
    far = FAKE << 8
    assert clip(gradients((a, b, 16, F32)), 1, out=a + 60, ws=far) == -2         # the norm in a tensor
    assert clip(gradients((a, b, 16, F32)), 1, out=b, ws=far) == -2
    assert clip(gradients((a, b, 16, F32)), 1, out=far, ws=a) == -2
    assert clip(gradients((a, b + 256, 16, F32)), 1, out=far, ws=b) == -2        # the workspace's end


def test_layers_refuse_what_is_not_on_the_gpu():
    with pytest.raises(ValueError):
        ProjectLayer(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        gradient_norm([])
    with pytest.raises(ValueError):
        clip_gradients([torch.zeros(4)], 1.0)


def test_the_norm_over_a_tensor():
    """The workspace is written while the gradients are read, and the norm is no gradient."""
    a, far = FAKE, FAKE << 8
    arr = gradients((a, None, 4096, F32))
    need = 512                                       # the two chunks' sums, rounded up
    assert norm(arr, 1, out=far, ws=a) == -2
    assert norm(arr, 1, out=far, ws=a + 4096 * 4 - 256) == -2
    assert norm(arr, 1, out=far, ws=a - 256, nb=need) == -2
    assert norm(arr, 1, out=a + 4096 * 4 - 4, ws=far) == -2
    assert norm(arr, 1, out=far + 256, ws=far, nb=need) == -2
