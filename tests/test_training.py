"""Refusals of group norm and of the head's losses, on the host.

Every call fails host-side validation, so nothing reaches the GPU; the
pointers are placeholders that are never dereferenced.
"""
import ctypes

import pytest

from paper_2608_23794_amd import binding as mb

GIB = 1 << 30
# every array at a place of its own
PLACE = {n: (1 << 40) + i * 64 * GIB for i, n in enumerate(
    ("x", "y", "dy", "dx", "scale", "shift", "stats", "dscale", "dshift", "weight", "classes", "logits", "loss", "saved",
     "dloss", "dweight", "ws"))}


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(mb.LIB_PATH):
        from paper_2608_23794_amd import build
        build.build()
    return mb.load()


def norm_desc(**kw):
    return mb.make_group_norm_desc(**dict(dict(B=2, C=64, H=8, W=8, G=8, dtype=mb.MOCE_BF16, layout=mb.MOCE_NHWC,
                                               act=mb.MOCE_ACT_RELU, eps=1e-5), **kw))


def norm(d, n=GIB, **at):
    p = dict(PLACE, **at)
    return mb.raw_status("moce_group_norm", ctypes.byref(d) if d else None, p["x"], p["scale"], p["shift"], p["y"],
                         p["stats"], p["ws"], n, None)


def norm_backward(d, n=GIB, grads=True, **at):
    p = dict(PLACE, **at)
    g = mb.make_group_norm_grads(p["dx"], p["dscale"], p["dshift"])
    return mb.raw_status("moce_group_norm_backward", ctypes.byref(d) if d else None, p["x"], p["scale"], p["shift"],
                         p["stats"], p["dy"], ctypes.byref(g) if grads else None, p["ws"], n, None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), -2), (dict(C=0), -2), (dict(H=0), -2), (dict(W=-1), -2), (dict(G=0), -2), (dict(G=7), -2),
    (dict(G=128), -2), (dict(act=4), -2), (dict(act=-1), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2),
    (dict(eps=float("inf")), -2), (dict(dtype=2), -3), (dict(layout=2), -4), (dict(C=1 << 21), -10),
    (dict(H=1 << 20, W=1 << 11), -10), (dict(C=1 << 16, H=1 << 8, W=1 << 8), -10), (dict(B=(1 << 29) + 1, H=1, W=1), -10),
    (dict(B=1 << 20, C=1 << 12, H=32, W=4), -10),
])
def test_norm_descriptor(lib, change, code):
    d = norm_desc(**change)
    assert norm(d) == code and norm_backward(d) == code
    assert lib.moce_group_norm_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.moce_group_norm_backward_workspace_bytes(ctypes.byref(d)) == 0


def test_norm_pointers(lib):
    d = norm_desc()
    need = lib.moce_group_norm_workspace_bytes(ctypes.byref(d))
    back = lib.moce_group_norm_backward_workspace_bytes(ctypes.byref(d))
    assert need > 0 and back > 0
    assert norm(None) == -1 and norm_backward(None) == -1 and norm_backward(d, grads=False) == -1
    assert norm(d, x=None) == -1 and norm(d, y=None) == -1
    for name in ("x", "dy", "stats"):
        assert norm_backward(d, **{name: None}) == -1
    for name, step in (("x", 8), ("y", 8), ("scale", 2), ("shift", 2), ("stats", 2), ("ws", 16)):
        assert norm(d, **{name: PLACE[name] + step}) == -8
    for name, step in (("x", 8), ("dy", 8), ("dx", 8), ("scale", 2), ("shift", 2), ("stats", 2), ("dscale", 2),
                       ("dshift", 2), ("ws", 16)):
        assert norm_backward(d, **{name: PLACE[name] + step}) == -8
    assert norm(d, ws=None) == -7 and norm_backward(d, ws=None) == -7
    assert norm(d, n=0) == -7 and norm_backward(d, n=0) == -7


def test_norm_overlaps():
    d = norm_desc()
    x = 2 * 64 * 64 * 2
    for name in ("x", "scale", "shift"):
        for off in (0, 16 if name == "x" else 0):
            if name == "x" and off == 0:
                continue                      # in place
            assert norm(d, y=PLACE[name] + off) == -2
        assert norm(d, ws=PLACE[name]) == -2 and norm(d, stats=PLACE[name]) == -2
    assert norm(d, y=PLACE["x"] + x - 16) == -2 and norm(d, y=PLACE["x"] - x + 16) == -2
    assert norm(d, stats=PLACE["y"]) == -2 and norm(d, ws=PLACE["y"]) == -2 and norm(d, ws=PLACE["stats"]) == -2
    for out in ("dx", "dscale", "dshift", "ws"):
        for name in ("x", "dy", "scale", "shift", "stats"):
            if out == "dx" and name in ("x", "dy"):
                assert norm_backward(d, dx=PLACE[name] + 16) == -2
            else:
                assert norm_backward(d, **{out: PLACE[name]}) == -2
    assert norm_backward(d, dscale=PLACE["dshift"]) == -2 and norm_backward(d, ws=PLACE["dx"]) == -2
    # x and dy the same memory, and dx over both
    assert norm_backward(d, dx=PLACE["x"], dscale=PLACE["x"] + 64) == -2


def head_desc(**kw):
    return mb.make_head_desc(**dict(dict(P=100, C=64, V=1000, dtype=mb.MOCE_BF16, K=1), **kw))


FORWARD = ("x", "weight", "shift", "classes", "loss", "saved")
BACKWARD = ("x", "weight", "shift", "classes", "saved", "dloss")


def head(d, teacher, n=64 * GIB - 1, **at):
    p = dict(PLACE, **at)
    t = (p["logits"],) if teacher else ()
    return mb.raw_status("moce_head_distill" if teacher else "moce_head_cross_entropy", ctypes.byref(d) if d else None,
                         p["x"], p["weight"], p["shift"], p["classes"], *t, p["loss"], p["saved"], p["ws"], n, None)


def head_backward(d, teacher, n=64 * GIB - 1, grads=True, **at):
    p = dict(PLACE, **at)
    t = (p["logits"],) if teacher else ()
    g = mb.make_head_grads(p["dx"], p["dweight"], p["dshift"])
    return mb.raw_status("moce_head_distill_backward" if teacher else "moce_head_cross_entropy_backward",
                         ctypes.byref(d) if d else None, p["x"], p["weight"], p["shift"], p["classes"], *t, p["saved"],
                         p["dloss"], ctypes.byref(g) if grads else None, p["ws"], n, None)


@pytest.mark.parametrize("change,code", [
    (dict(P=0), -2), (dict(C=0), -2), (dict(V=0), -2), (dict(K=0), -2), (dict(index_bytes=2), -2),
    (dict(reduction=2), -2), (dict(reduction=-1), -2), (dict(dtype=2), -3), (dict(P=(1 << 24) + 1, V=1, C=1), -10),
    (dict(C=(1 << 20) + 1), -10), (dict(V=(1 << 20) + 1), -10), (dict(C=1 << 16, V=1 << 20), -10),
    (dict(P=1 << 16, V=1 << 20), -10), (dict(P=1 << 24, C=1 << 10, V=1), -10),
])
def test_head_descriptor(lib, change, code):
    d = head_desc(**change)
    for teacher in (False, True):
        assert head(d, teacher) == code and head_backward(d, teacher) == code
    for fn in ("moce_head_saved_floats", "moce_head_workspace_bytes", "moce_head_backward_workspace_bytes"):
        assert getattr(lib, fn)(ctypes.byref(d)) == 0


@pytest.mark.parametrize("teacher,change,code", [
    (False, dict(K=2), -2), (False, dict(smoothing=-0.1), -2), (False, dict(smoothing=1.5), -2),
    (False, dict(smoothing=float("nan")), -2), (True, dict(temperature=0.0), -2), (True, dict(temperature=-1.0), -2),
    (True, dict(temperature=float("inf")), -2), (True, dict(temperature=float("nan")), -2),
    (True, dict(teacher_dtype=2), -3), (True, dict(K=1025), -10),
])
def test_head_descriptor_of_one_loss(teacher, change, code):
    d = head_desc(**change)
    assert head(d, teacher) == code and head_backward(d, teacher) == code


def test_head_pointers(lib):
    for teacher in (False, True):
        d = head_desc(K=5 if teacher else 1)
        need = lib.moce_head_workspace_bytes(ctypes.byref(d))
        back = lib.moce_head_backward_workspace_bytes(ctypes.byref(d))
        assert need > 0 and back > 0
        assert lib.moce_head_saved_floats(ctypes.byref(d)) == 100 * ((5 if teacher else 1) + 1) + 2
        assert head(None, teacher) == -1 and head_backward(None, teacher) == -1
        assert head_backward(d, teacher, grads=False) == -1
        for name in ("x", "weight", "classes", "loss") + (("logits",) if teacher else ()):
            assert head(d, teacher, **{name: None}) == -1
        for name in ("x", "weight", "classes", "saved", "dloss") + (("logits",) if teacher else ()):
            assert head_backward(d, teacher, **{name: None}) == -1
        for name in FORWARD + ("ws",):
            step = {"x": 8, "weight": 8, "classes": 4, "ws": 16}.get(name, 2)
            assert head(d, teacher, **{name: PLACE[name] + step}) == -8
        for name in BACKWARD + ("dx", "dweight", "dshift", "ws"):
            step = {"x": 8, "weight": 8, "dx": 8, "dweight": 8, "classes": 4, "ws": 16}.get(name, 2)
            assert head_backward(d, teacher, **{name: PLACE[name] + step}) == -8
        assert head(d, teacher, ws=None) == -7 and head_backward(d, teacher, ws=None) == -7
        assert head(d, teacher, n=need // 2) == -7 and head_backward(d, teacher, n=back // 2) == -7


def test_head_overlaps():
    for teacher in (False, True):
        d = head_desc(K=5 if teacher else 1)
        targets = ("classes", "logits") if teacher else ("classes",)
        for out in ("loss", "saved", "ws"):
            for name in ("x", "weight", "shift") + targets:
                assert head(d, teacher, **{out: PLACE[name]}) == -2
        assert head(d, teacher, loss=PLACE["saved"] + 4) == -2 and head(d, teacher, ws=PLACE["loss"]) == -2
        for out in ("dx", "dweight", "dshift", "ws"):
            for name in ("x", "weight", "shift", "saved", "dloss") + targets:
                assert head_backward(d, teacher, **{out: PLACE[name]}) == -2
        assert head_backward(d, teacher, dx=PLACE["dweight"]) == -2
        assert head_backward(d, teacher, ws=PLACE["dshift"]) == -2


def test_temperatures_at_their_ends(lib):
    """A temperature whose square or inverse is no normal float32 number would lose the loss; those at the ends count."""
    for t in (2.0 ** -63, 2.0 ** 62.01, 1e-38, 1e38):
        d = head_desc(temperature=t, K=5)
        assert head(d, True) == -2 and head_backward(d, True) == -2
        assert lib.moce_head_workspace_bytes(ctypes.byref(d)) == 0
    for t in (2.0 ** -62, 2.0 ** 62):
        d = head_desc(temperature=t, K=5)
        assert lib.moce_head_workspace_bytes(ctypes.byref(d)) > 0 and head(d, True, n=0) == -7
