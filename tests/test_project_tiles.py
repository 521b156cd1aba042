"""Every kernel that the dense projection's products can take, on whole numbers: results equal to the last bit.

A product's kernel goes by its type, its tile and stages in LDS, how its two operands lie in memory, whether lines
pass from image to image, and whether its contraction is split.  SIZES reach each of them; the host's choice is
compared with that of many drawn sizes, so that a change of the choice that leaves a kernel untested shows here.
"""
import random

import pytest
import torch

from paper_2608_23794_amd import binding as mb
from paper_2608_23794_amd.layer import ProjectLayer

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PRODUCTS = (mb.MOCE_PRODUCT_FORWARD, mb.MOCE_PRODUCT_DX, mb.MOCE_PRODUCT_DWEIGHT)

# images, channels in and out, plane, type, layout; the last ones are whole layers: tokens, a long prompt, expansions
SIZES = [
    (1, 32, 32, 10, 1, "f32", "nhwc"), (1, 32, 32, 4, 4, "bf16", "nhwc"), (1, 4448, 224, 5, 1, "f32", "nchw"),
    (5, 4256, 376, 4, 1, "bf16", "nchw"), (3, 304, 4282, 2, 4, "f32", "nchw"), (2, 3277, 1789, 1, 4, "f32", "nchw"),
    (20, 1716, 958, 1, 4, "f32", "nchw"), (2, 1912, 2496, 4, 4, "bf16", "nchw"), (155, 1, 8, 28, 28, "f32", "nhwc"),
    (10, 3399, 1037, 1, 8, "f32", "nchw"), (2, 3276, 3581, 4, 4, "bf16", "nchw"),
    (2, 4616, 752, 8, 8, "bf16", "nchw"), (9, 3618, 4393, 1, 4, "f32", "nchw"), (127, 6, 2, 56, 56, "bf16", "nhwc"),
    (4, 956, 4473, 2, 16, "bf16", "nchw"), (4, 4248, 1440, 6, 4, "bf16", "nchw"),
    (264, 127, 1529, 3, 3, "f32", "nhwc"), (2, 4224, 2976, 8, 8, "bf16", "nchw"),
    (3, 1420, 1546, 16, 16, "f32", "nchw"), (86, 2152, 520, 4, 4, "bf16", "nchw"),
    (120, 1309, 1521, 1, 8, "bf16", "nchw"), (3, 1308, 1247, 21, 21, "bf16", "nhwc"),
    (40, 8, 216, 399, 4, "f32", "nchw"), (17, 4278, 2326, 4, 4, "f32", "nhwc"), (192, 96, 1056, 7, 7, "f32", "nchw"),
    (3, 147, 333, 454, 16, "bf16", "nchw"), (2, 3777, 352, 28, 28, "bf16", "nchw"),
    (68, 25, 68, 56, 56, "f32", "nhwc"), (41, 1256, 152, 16, 16, "bf16", "nchw"),
    (18, 352, 184, 1741, 1, "bf16", "nhwc"), (98, 1488, 128, 131, 1, "bf16", "nhwc"),
    (84, 4320, 32, 5, 16, "f32", "nchw"), (1, 688, 312, 1046, 16, "bf16", "nchw"),
    (1, 2397, 3, 954, 16, "bf16", "nchw"), (11, 4352, 4, 28, 28, "bf16", "nchw"),
    (1, 136, 880, 1823, 16, "bf16", "nchw"), (211, 1, 3647, 8, 8, "bf16", "nchw"),
    (26, 896, 344, 28, 28, "f32", "nhwc"), (1, 512, 928, 1869, 8, "bf16", "nchw"),
    (2, 3, 2051, 922, 16, "bf16", "nchw"), (16, 472, 990, 32, 32, "f32", "nchw"),
    (101, 3772, 1, 14, 14, "bf16", "nchw"), (10, 473, 4149, 566, 1, "bf16", "nhwc"),
    (288, 161, 2202, 75, 1, "bf16", "nchw"), (1, 75, 2067, 2003, 16, "bf16", "nchw"),
    (21, 416, 1728, 28, 28, "bf16", "nchw"), (4, 613, 3377, 56, 56, "f32", "nchw"),
    (52, 412, 1206, 32, 32, "bf16", "nhwc"), (128, 1248, 432, 49, 8, "bf16", "nchw"),
    (1, 640, 2441, 1885, 16, "bf16", "nchw"), (1, 2848, 768, 1880, 16, "f32", "nchw"),
    (256, 768, 768, 197, 1, "bf16", "nhwc"), (8, 4096, 4096, 2048, 1, "bf16", "nhwc"),
    (64, 64, 256, 56, 56, "bf16", "nchw"), (64, 256, 1024, 14, 14, "bf16", "nchw"),
]


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(mb.LIB_PATH):
        from paper_2608_23794_amd import build
        build.build()
    return mb.load()


def kernels(B, C, O, H, W, dtype, layout):
    """The kernels of the three products."""
    d = mb.make_project_desc(B, C, H, W, O, mb.MOCE_BF16 if dtype == "bf16" else mb.MOCE_F32,
                             mb.MOCE_NHWC if layout == "nhwc" else mb.MOCE_NCHW)
    cuts = [mb.moce_project_path(d, p) for p in PRODUCTS]
    return {(dtype, c.rows, c.columns, c.stages, c.a_along, c.b_along, c.images, c.splits > 1) for c in cuts}


def drawn(rng):
    def log(top):
        return int(2 ** rng.uniform(0, top))

    C, O = log(12.2), log(12.2)
    if rng.random() < 0.45:
        C, O = max(8, C // 8 * 8), max(8, O // 8 * 8)
    layout = rng.choice(["nchw", "nhwc"])
    H = W = rng.choice([4, 7, 8, 14, 16, 28, 32, 56, log(6)])
    if rng.random() < 0.5:
        H, W = log(11), 1 if layout == "nhwc" else rng.choice([1, 4, 8, 16])
    return log(9), C, O, H, W, rng.choice(["bf16", "bf16", "f32"]), layout


def test_the_sizes_take_every_kernel(lib):
    covered = set().union(*(kernels(*s) for s in SIZES))
    rng = random.Random(7)
    found = {}
    for _ in range(40000):
        size = drawn(rng)
        try:
            for k in kernels(*size):
                found.setdefault(k, size)
        except mb.MoceError:     # past the limits
            pass
    assert not {k: found[k] for k in set(found) - covered}
    # both types, the tiles of each, and the four ways that operands lie
    assert {k[:4] for k in covered if k[1]} == {(t, *c) for t in TYPES for c in (
        (128, 128, 2), (128, 64, 2), (64, 128, 2), (64, 64, 3), (128, 64, 1), (64, 128, 1))} | {
        ("bf16", *c) for c in ((256, 256, 2), (128, 64, 3), (64, 128, 3))}
    assert {k[4:7] for k in covered} == {(1, 1, 0), (1, 0, 0), (0, 0, 0), (1, 1, 1)}


def test_the_kernel_of_a_product(lib):
    import ctypes
    d = mb.make_project_desc(8, 4096, 2048, 1, 4096, mb.MOCE_BF16, mb.MOCE_NHWC)
    cut = mb.moce_project_cut()
    assert lib.moce_project_path(None, 0, ctypes.byref(cut)) == -1
    assert lib.moce_project_path(ctypes.byref(d), 0, None) == -1
    for p in (-1, 3):
        assert lib.moce_project_path(ctypes.byref(d), p, ctypes.byref(cut)) == -2
    d.act = 9
    assert lib.moce_project_path(ctypes.byref(d), 0, ctypes.byref(cut)) == -2
    few = mb.moce_project_path(mb.make_project_desc(32, 64, 1, 1, 64, mb.MOCE_BF16, mb.MOCE_NHWC), 0)
    assert few.rows == 0 and few.splits == 1


# the last planes whose tiles' offsets have 31 bits, and the first that are turned for that although their lines are whole
SPANS = [(2, 256, 256, 8, 174762, "bf16", "nchw"), (2, 256, 256, 8, 174763, "bf16", "nchw"),
         (3, 8, 8, 8, 493447, "bf16", "nchw"), (3, 8, 8, 8, 493448, "bf16", "nchw"),
         (2, 72, 80, 8, 161319, "f32", "nchw"), (2, 72, 80, 8, 161320, "f32", "nchw")]


def turned(size):
    return {k[4:6] for k in kernels(*size)} == {(1, 1), (0, 0)}


def test_the_planes_that_are_turned_for_their_offsets(lib):
    assert [turned(s) for s in SPANS] == [False, True] * 3


@pytest.mark.gpu
@pytest.mark.parametrize("size", SPANS, ids=str)
def test_planes_at_the_limit_of_a_tiles_offsets(size):
    check_products(size, "relu", True)


@pytest.mark.gpu
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_products_of_whole_numbers(size):
    i = SIZES.index(size)
    check_products(size, ("none", "relu")[i % 2], i % 3 != 0)


def check_products(size, act, affine):
    """Small whole numbers, scales that are powers of two: every sum is exact in float32, so y, z and the gradients are
    the exact ones rounded once, whatever the tile."""
    B, C, O, H, W, dtype, layout = size
    g = torch.Generator(device="cuda").manual_seed(C + O)
    dt = TYPES[dtype]
    xs, ys = ((B, C, H, W), (B, O, H, W)) if layout == "nchw" else ((B, H, W, C), (B, H, W, O))

    def whole(shape, lo, hi, t):
        return torch.empty(shape, device="cuda").random_(lo, hi + 1, generator=g).to(t)

    def rows(t):
        t = t.movedim(1, -1) if layout == "nchw" else t
        return t.reshape(-1, t.shape[-1])

    x, w, dy, res = whole(xs, -1, 2, dt), whole((O, C), -1, 2, dt), whole(ys, -1, 2, dt), whole(ys, -4, 4, dt)
    scale = 2.0 ** whole((O,), -1, 1, torch.float32) if affine else None
    shift = whole((O,), -3, 3, torch.float32) if affine else None
    layer = ProjectLayer(w, scale, shift, act=act, layout=layout)
    z = torch.full(ys, float("nan"), dtype=dt, device="cuda")
    y = layer.forward(x, residual=res, z=z)
    # float64 products in slices of positions, for their memory
    xr, rr, dyr, zr, yr = (rows(t) for t in (x, res, dy, z, y))
    s64 = scale.double() if affine else torch.ones(O, dtype=torch.float64, device="cuda")
    wd, G, dshift = w.double(), torch.zeros(O, C, dtype=torch.float64, device="cuda"), 0.0
    out = layer.backward(x, dy, z=z if act == "relu" else None, residual=True)
    dxr, drr = rows(out["dx"]), rows(out["dresidual"])
    step = max(1, (1 << 27) // max(C, O))
    for i in range(0, xr.shape[0], step):
        p = slice(i, i + step)
        want = (xr[p].double() @ wd.t().contiguous()) * s64 + rr[p].double()
        if affine:
            want = want + shift.double()
        assert torch.equal(zr[p], want.to(dt))
        assert torch.equal(yr[p], (want.clamp(min=0) if act == "relu" else want).to(dt))
        dz = dyr[p].double()
        if act == "relu":
            dz = torch.where(zr[p] > 0, dz, torch.zeros_like(dz))
        assert torch.equal(drr[p], dz.to(dt))
        assert torch.equal(dxr[p], ((dz * s64) @ wd).to(dt))
        G += dz.t().contiguous() @ xr[p].double()
        dshift = dshift + dz.sum(0)
    assert float(G.abs().max()) < 2.0 ** 24
    assert torch.equal(out["dweight"], (s64[:, None] * G).to(dt))
    if affine:
        assert torch.equal(out["dshift"], dshift.float())
        # a sum of whole numbers of which some pass 2^24: half a step each
        want, mag = (wd * G).sum(1), (wd.abs() * G.abs()).sum(1)
        exact = mag < 2.0 ** 24
        assert torch.equal(out["dscale"][exact], want[exact].float())
        assert ((out["dscale"].double() - want).abs() <= C * 2.0 ** -24 * mag)[~exact].all()
