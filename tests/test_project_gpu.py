"""The dense projection and its gradients on the GPU, against plain products in float64.

Tolerances count roundings.  An output of type T is off by half a step of T at
most (bfloat16 2^-8, float32 2^-24 of the value); a float32 sum of n terms by
n 2^-24 of the sum of their magnitudes; an operand rounded to bfloat16 by 2^-8
of the same sum.  The activations' slopes are below 1.13, and their own
evaluation is off by a few 1e-7 of the argument (bfloat16) or steps (float32).
"""
import math

import pytest
import torch

from paper_2608_23794_amd import binding as mb
from paper_2608_23794_amd.layer import ProjectLayer

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
STEP32 = 2.0 ** -24
ACT_ERR = 2e-6
SLOPE = 1.13


def act64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def make(B, C, O, H, W, dtype, layout, act="none", scale=False, shift=False, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[dtype]

    def n(*s):
        return torch.randn(*s, generator=g, device="cuda")

    xs, ys = ((B, C, H, W), (B, O, H, W)) if layout == "nchw" else ((B, H, W, C), (B, H, W, O))
    t = {"x": n(*xs).to(dt), "w": (n(O, C) * C ** -0.5).to(dt), "scale": n(O) if scale else None,
         "shift": n(O) if shift else None, "residual": n(*ys).to(dt), "dy": n(*ys).to(dt), "z": n(*ys).to(dt)}
    t["layer"] = ProjectLayer(t["w"], t["scale"], t["shift"], act=act, layout=layout)
    return t


def rows(t, layout):
    t = t.double()
    return (t.movedim(1, -1) if layout == "nchw" else t).reshape(-1, t.shape[1] if layout == "nchw" else t.shape[-1])


def check(name, got, want, tol):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), name
    over = err - tol
    i = int(over.argmax())
    assert float(over.flatten()[i]) <= 0, (f"{name}: off by {float(err.flatten()[i]):.3e} of "
                                           f"{float(want.flatten()[i]):.3e}, allowed {float(tol.flatten()[i]):.3e}")


def check_forward(t, dtype, layout, act, residual, y, z):
    x, w = rows(t["x"], layout), t["w"].double()
    C = w.shape[1]
    v, mag = x @ w.t(), x.abs() @ w.abs().t()
    if t["scale"] is not None:
        v, mag = v * t["scale"].double(), mag * t["scale"].double().abs()
    if t["shift"] is not None:
        v, mag = v + t["shift"].double(), mag + t["shift"].double().abs()
    if residual is not None:
        r = rows(residual, layout)
        v, mag = v + r, mag + r.abs()
    sums = (C + 4) * STEP32 * mag
    want = act64(v, act)
    check("y", rows(y, layout), want,
          HALF[dtype] * want.abs() * 1.01 + SLOPE * sums + (ACT_ERR * v.abs() if act in ("gelu", "silu") else 0))
    if z is not None:
        check("z", rows(z, layout), v, HALF[dtype] * v.abs() * 1.01 + sums)


def check_backward(t, dtype, layout, act, out):
    x, w, dy, z = rows(t["x"], layout), t["w"].double(), rows(t["dy"], layout), rows(t["z"], layout)
    P, C, O = x.shape[0], x.shape[1], dy.shape[1]
    smooth = act in ("gelu", "silu")
    low = HALF[dtype] if dtype == "bf16" else 0.0
    dz = dy * act_grad64(z, act)
    dz_err = ACT_ERR * dy.abs() * (1 + z.abs()) if smooth else torch.zeros_like(dz)
    s = t["scale"].double() if t["scale"] is not None else torch.ones(O, dtype=torch.float64, device="cuda")
    if "dresidual" in out:
        check("dresidual", rows(out["dresidual"], layout), dz, HALF[dtype] * 1.01 * dz.abs() + dz_err)
    if "dshift" in out:
        check("dshift", out["dshift"], dz.sum(0), (P + 4) * STEP32 * dz.abs().sum(0) + dz_err.sum(0) +
              STEP32 * dz.sum(0).abs())
    # one operand of dx is rounded: dz, or the scaled weight; dz alone for dweight
    dx, mag = (dz * s) @ w, (dz * s).abs() @ w.abs()
    in_x = low if smooth or t["scale"] is not None else 0.0
    check("dx", rows(out["dx"], layout), dx, HALF[dtype] * 1.01 * dx.abs() + ((O + 8) * STEP32 + in_x * 1.02) * mag +
          (dz_err * s.abs()) @ w.abs())
    G, Gm = dz.t() @ x, dz.abs().t() @ x.abs()
    in_w = low if smooth else 0.0
    gerr = ((P + 8) * STEP32 + in_w * 1.02) * Gm + dz_err.t() @ x.abs()
    want = s[:, None] * G
    check("dweight", out["dweight"], want, HALF[dtype] * 1.01 * want.abs() + s.abs()[:, None] * gerr)
    if "dscale" in out:
        check("dscale", out["dscale"], (w * G).sum(1), (w.abs() * (gerr + (C + 4) * STEP32 * G.abs())).sum(1))


# images, channels in and out, plane, layout: single positions and channels, sizes around a tile and its parts, long
# contractions with few outputs, odd planes
SIZES = [
    (1, 1, 1, 1, 1, "nhwc"), (1, 8, 8, 1, 1, "nhwc"), (1, 768, 33, 1, 1, "nhwc"), (3, 100, 1, 1, 1, "nchw"),
    (1, 64, 64, 64, 1, "nhwc"), (2, 65, 63, 33, 1, "nhwc"), (1, 1000, 24, 5, 3, "nhwc"), (4, 128, 256, 16, 9, "nhwc"),
    (1, 7, 300, 130, 1, "nhwc"), (5, 72, 40, 8, 8, "nchw"), (3, 33, 31, 7, 7, "nchw"), (9, 64, 128, 2, 1, "nchw"),
    (2, 130, 66, 14, 14, "nchw"), (70, 16, 8, 3, 5, "nchw"), (1, 2048, 16, 4, 4, "nchw"), (2, 24, 16, 61, 64, "nchw"),
    (2, 16, 24, 97, 101, "nhwc"), (16, 4096, 72, 1, 1, "nhwc"), (17, 513, 1030, 1, 1, "nhwc"),
    (5000, 8, 16, 2, 1, "nchw"), (4200, 8, 72, 4, 2, "nchw"), (33, 264, 40, 1, 1, "nhwc"), (20, 777, 90, 1, 1, "nhwc"),
]
KINDS = [("none", False, False, False), ("relu", True, True, True), ("gelu", False, True, False),
         ("silu", False, True, True), ("none", True, False, True), ("gelu", True, True, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(size, dtype):
    B, C, O, H, W, layout = size
    for i, (act, scale, shift, residual) in enumerate(KINDS):
        t = make(B, C, O, H, W, dtype, layout, act, scale, shift, seed=i)
        res = t["residual"] if residual else None
        z = torch.empty_like(t["residual"]) if i % 2 else None
        y = t["layer"].forward(t["x"], residual=res, z=z)
        check_forward(t, dtype, layout, act, res, y, z)
        out = t["layer"].backward(t["x"], t["dy"], z=t["z"], residual=residual)
        check_backward(t, dtype, layout, act, out)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_against_differences(dtype, layout):
    """The layer's backward against central differences of its own float32 forward."""
    act = "silu"
    t = make(2, 12, 10, 3, 4, "f32", layout, act, scale=True, shift=True)
    dt = TYPES[dtype]
    x, w, dy = t["x"].to(dt).float(), t["w"].to(dt).float(), t["dy"].to(dt).float()

    def loss(x, w, shift):
        y = ProjectLayer(w, t["scale"], shift, act=act, layout=layout).forward(x)
        return float((y.double() * dy.double()).sum())

    z = torch.empty_like(dy)
    ProjectLayer(w, t["scale"], t["shift"], act=act, layout=layout).forward(x, z=z)
    out = ProjectLayer(w.to(dt), t["scale"], t["shift"], act=act, layout=layout).backward(x.to(dt), dy.to(dt), z=z.to(dt))
    h = 2.0 ** -6      # the differences are off by h^2 / 6 of a third derivative of order 1, and by roundings over h
    for name, v, g in (("x", x, out["dx"]), ("w", w, out["dweight"]), ("shift", t["shift"], out["dshift"])):
        scale = float(g.float().abs().max())
        for i in range(0, v.numel(), max(1, v.numel() // 12)):
            a, b = v.clone(), v.clone()
            a.view(-1)[i] += h
            b.view(-1)[i] -= h
            args = {"x": x, "w": w, "shift": t["shift"]}
            d = (loss(**{**args, name: a}) - loss(**{**args, name: b})) / (2 * h)
            assert abs(d - float(g.reshape(-1)[i])) <= (2e-2 if dtype == "bf16" else 2e-3) * max(1.0, scale), (name, i)


def test_one_gradient_at_a_time():
    """Each gradient alone has the bits it has beside the others."""
    t = make(3, 40, 56, 5, 7, "bf16", "nchw", "relu", scale=True, shift=True)
    layer = t["layer"]
    every = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    d = layer.desc(t["x"].shape)
    ws = torch.empty(layer.backward_workspace_bytes(t["x"].shape), dtype=torch.uint8, device="cuda")
    for name, want in every.items():
        got = torch.full_like(want, float("nan"))
        mb.moce_project_backward(d, t["x"], t["w"], t["scale"], t["z"], t["dy"], mb.make_project_grads(**{name: got}), ws,
                                 ws.numel(), torch.cuda.current_stream())
        assert torch.equal(got, want), name


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype, layout):
    t = make(2, 48, 40, 6, 6, dtype, layout, "gelu", shift=True)
    layer, z = t["layer"], torch.empty_like(t["residual"])
    want = layer.forward(t["x"], residual=t["residual"], z=z)
    y = t["residual"].clone()
    assert torch.equal(layer.forward(t["x"], residual=y, y=y), want)
    zz = t["residual"].clone()
    assert torch.equal(layer.forward(t["x"], residual=zz, z=zz), want) and torch.equal(zz, z)
    every = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    dy, out = t["dy"].clone(), {n: torch.empty_like(every[n]) for n in ("dx", "dweight", "dshift")}
    ws = torch.empty(layer.backward_workspace_bytes(t["x"].shape), dtype=torch.uint8, device="cuda")
    mb.moce_project_backward(layer.desc(t["x"].shape), t["x"], t["w"], None, t["z"], dy,
                             mb.make_project_grads(dresidual=dy, **out), ws, ws.numel(), torch.cuda.current_stream())
    assert torch.equal(dy, every["dresidual"])
    assert all(torch.equal(out[n], every[n]) for n in out)


@pytest.mark.parametrize("size", [(1, 72, 50, 37, 1, "nhwc"), (3, 72, 48, 7, 9, "nchw"), (2, 40, 64, 8, 4, "nchw"),
                                  (1, 1030, 13, 3, 1, "nhwc")], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_outside_the_tensors(size, dtype):
    """Inputs lie in memory full of NaN, outputs between guards that stay."""
    B, C, O, H, W, layout = size
    t = make(B, C, O, H, W, dtype, layout, "gelu", shift=True)
    pad = 512

    def framed(v):
        f = torch.full((v.numel() + 2 * pad,), float("nan"), dtype=v.dtype, device="cuda")
        f[pad:pad + v.numel()] = v.reshape(-1)
        return f, f[pad:pad + v.numel()].view(v.shape)

    x, w, res, zin, dy = (framed(t[n])[1] for n in ("x", "w", "residual", "z", "dy"))
    layer = ProjectLayer(w, None, t["shift"], act="gelu", layout=layout)
    (fy, y), (fz, z) = framed(t["z"]), framed(t["z"])
    layer.forward(x, residual=res, y=y, z=z)
    check_forward(t, dtype, layout, "gelu", t["residual"], y, z)
    fdx, dx = framed(t["x"])
    out = layer.backward(x, dy, z=zin, residual=True, dx=dx)
    check_backward(t, dtype, layout, "gelu", out)
    for f, n in ((fy, y.numel()), (fz, z.numel()), (fdx, dx.numel())):
        assert torch.isnan(f[:pad]).all() and torch.isnan(f[pad + n:]).all()


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_at_their_position(dtype, layout):
    t = make(2, 40, 24, 5, 5, dtype, layout, "relu", shift=True)
    clean = t["layer"].forward(t["x"])
    x = t["x"].clone()
    (x[1, :, 2, 3] if layout == "nchw" else x[1, 2, 3])[7] = float("nan")
    (x[0, :, 4, 4] if layout == "nchw" else x[0, 4, 4])[0] = float("inf")
    y = t["layer"].forward(x)
    at = torch.zeros_like(y, dtype=torch.bool)
    (at[1, :, 2, 3] if layout == "nchw" else at[1, 2, 3])[:] = True
    assert torch.isnan(y[at]).all()
    (at[0, :, 4, 4] if layout == "nchw" else at[0, 4, 4])[:] = True
    assert torch.equal(y[~at], clean[~at])
    inf = y[0, :, 4, 4] if layout == "nchw" else y[0, 4, 4]
    assert torch.equal(torch.isinf(inf), t["w"][:, 0] > 0) and (inf[t["w"][:, 0] < 0] == 0).all()
    # an upstream value at a position that the ReLU closed reaches nothing
    dy, z = t["dy"].clone(), t["z"].clone()
    (dy[0, :, 1, 1] if layout == "nchw" else dy[0, 1, 1])[:] = float("inf")
    (z[0, :, 1, 1] if layout == "nchw" else z[0, 1, 1])[:] = -1.0
    out = t["layer"].backward(t["x"], dy, z=z, residual=True)
    assert all(torch.isfinite(v.float()).all() for v in out.values())


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, 21, 13, 40, 1, "nhwc"), (3, 21, 541, 40, 1, "nhwc"), (2, 21, 13, 7, 7, "nchw"),
                                  (3, 13, 70, 5, 7, "nchw"), (1, 5, 3, 1, 2, "nhwc")], ids=str)
def test_lines_of_any_length_end_where_they_end(size, dtype, act):
    """Upstream values that are not finite at the first element of a line leave the line before it alone."""
    B, C, O, H, W, layout = size
    t = make(B, C, O, H, W, dtype, layout, act, shift=True)
    clean = t["layer"].backward(t["x"], t["dy"], z=t["z"], residual=True)
    dy, z = t["dy"].clone(), t["z"].clone()
    z[B - 1] = 1.0      # open for every activation
    want = t["layer"].backward(t["x"], dy, z=z, residual=True)
    dy[B - 1] = float("nan")
    got = t["layer"].backward(t["x"], dy, z=z, residual=True)
    for name in ("dx", "dresidual"):
        if B > 1:
            assert torch.equal(got[name][:B - 1], clean[name][:B - 1]), name
        assert torch.isnan(got[name][B - 1]).all() and torch.isfinite(want[name].float()).all(), name
    assert torch.isnan(got["dshift"]).all() and torch.isnan(got["dweight"]).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_activations_over_their_range(dtype, act):
    """An identity weight: values from tiny to huge, and the limits at infinity."""
    v = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([-1e30, -300., -100., -40., 0., 1e-30, 40., 300., 1e30])])
    x = v.to(TYPES[dtype]).cuda().reshape(-1, 1)
    w = torch.ones(1, 1, dtype=x.dtype, device="cuda")
    layer = ProjectLayer(w, act=act)
    y = layer.forward(x)
    z64 = x.double()
    want = act64(z64, act)
    # an absolute error of the distribution function of 3e-7 beside the rounding (float32: a few steps)
    check("y", y, want, HALF[dtype] * 1.01 * want.abs() + (3e-7 if dtype == "bf16" else 4 * STEP32) * z64.abs().clamp(max=8) +
          (0 if dtype == "bf16" else 8 * STEP32 * want.abs()))
    dy = torch.ones_like(y)
    g = layer.backward(x, dy, z=x, residual=True)["dresidual"]
    want = act_grad64(z64, act).nan_to_num(0.0)
    check("slope", g, want, HALF[dtype] * 1.01 * want.abs() + ACT_ERR)
    ends = torch.tensor([[float("-inf")], [float("inf")]], dtype=x.dtype, device="cuda")
    one = torch.zeros(2, 1, dtype=x.dtype, device="cuda")
    z = torch.empty_like(ends)
    y = layer.forward(one, residual=ends, z=z)
    assert float(y[0]) == 0.0 and float(y[1]) == float("inf") and torch.equal(z, ends)
    g = layer.backward(one, torch.ones_like(ends), z=ends, residual=True)["dresidual"]
    assert float(g[0]) == 0.0 and float(g[1]) == 1.0


def test_same_bits_every_time_on_any_stream_and_captured():
    t = make(4, 512, 48, 9, 9, "bf16", "nhwc", "gelu", shift=True)
    layer = t["layer"]
    want = layer.forward(t["x"], residual=t["residual"])
    grads = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = layer.forward(t["x"], residual=t["residual"])
        out = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    side.synchronize()
    assert torch.equal(y, want) and all(torch.equal(out[n], grads[n]) for n in grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.forward(t["x"], residual=t["residual"])
        out = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(100 + seed)
        for n in ("x", "dy", "z", "residual"):
            t[n].copy_(torch.randn(t[n].shape, generator=g, device="cuda"))
        want = layer.forward(t["x"], residual=t["residual"])
        grads = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and all(torch.equal(out[n], grads[n]) for n in grads)


def test_tokens_rows_and_empty_batches():
    t = make(2, 24, 40, 5, 3, "bf16", "nhwc", "silu", shift=True)
    layer, want = t["layer"], t["layer"].forward(t["x"])
    assert torch.equal(layer.forward(t["x"].reshape(30, 24)), want.reshape(30, 40))
    assert torch.equal(layer.forward(t["x"].reshape(2, 15, 24)), want.reshape(2, 15, 40))
    empty = torch.empty(0, 7, 24, dtype=torch.bfloat16, device="cuda")
    assert layer.forward(empty).shape == (0, 7, 40)
    out = layer.backward(empty, torch.empty(0, 7, 40, dtype=torch.bfloat16, device="cuda"),
                         z=torch.empty(0, 7, 40, dtype=torch.bfloat16, device="cuda"))
    assert float(out["dweight"].abs().max()) == 0 and float(out["dshift"].abs().max()) == 0


def test_layer_refusals():
    t = make(2, 24, 40, 5, 3, "bf16", "nhwc", "silu", shift=True)
    layer, x = t["layer"], t["x"]
    for bad in (x.float(), x.cpu(), x[..., :23], x.transpose(1, 2), x.reshape(-1)):
        with pytest.raises(ValueError):
            layer.forward(bad)
    with pytest.raises(ValueError):
        layer.forward(x, residual=t["residual"][:1])
    with pytest.raises(ValueError):
        layer.forward(x, y=torch.empty(1, device="cuda"))
    with pytest.raises(ValueError):
        layer.backward(x, t["dy"])                       # no z
    with pytest.raises(ValueError):
        layer.backward(x, t["dy"].float(), z=t["z"])
    with pytest.raises(ValueError):
        ProjectLayer(t["w"], act="tanh")
    with pytest.raises(ValueError):
        ProjectLayer(t["w"].t())
    with pytest.raises(ValueError):
        ProjectLayer(t["w"], shift=t["shift"][:-1])
    with pytest.raises(mb.MoceError):
        layer.backward(x, t["dy"], z=t["z"], ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        layer.forward(x, ws=torch.empty(1 << 20, dtype=torch.uint8))
    odd = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
    with pytest.raises(mb.MoceError):
        layer.forward(odd)                               # not 16-byte aligned


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_many_positions(layout):
    """Sums over 2^18 positions and more: the weight's gradient in many splits."""
    H = W = 257
    t = make(4, 24, 16, H, W, "bf16", layout, "relu", scale=True, shift=True)
    z = torch.empty_like(t["z"])
    y = t["layer"].forward(t["x"], residual=t["residual"], z=z)
    check_forward(t, "bf16", layout, "relu", t["residual"], y, z)
    t["z"] = z
    check_backward(t, "bf16", layout, "relu", t["layer"].backward(t["x"], t["dy"], z=z, residual=True))


def test_rows_of_one_image_beyond_two_gigabytes():
    """2^21 rows of 1024 channels as one sequence, offsets past 32 bits: rows at the ends, and the sums over all."""
    n, C, O, part = (1 << 21) + 3, 1024, 24, 1 << 18
    g = torch.Generator(device="cuda").manual_seed(5)
    # whole numbers: the sums over rows stay below 2^23 and are exact
    x = torch.empty(1, n, C, dtype=torch.bfloat16, device="cuda").random_(-2, 3, generator=g)
    w = (torch.randn(O, C, generator=g, device="cuda") * C ** -0.5).bfloat16()
    dy = torch.empty(1, n, O, dtype=torch.bfloat16, device="cuda").random_(-1, 2, generator=g)
    layer = ProjectLayer(w)
    y, out = layer.forward(x), layer.backward(x, dy)
    wd = w.double()
    for rows in (slice(0, 40), slice(n // 2, n // 2 + 40), slice(n - 40, n)):
        xd, dyd = x[0, rows].double(), dy[0, rows].double()
        want, mag = xd @ wd.t(), xd.abs() @ wd.abs().t()
        check("y", y[0, rows], want, HALF["bf16"] * want.abs() + 2 * C * STEP32 * mag)
        want, mag = dyd @ wd, dyd.abs() @ wd.abs()
        check("dx", out["dx"][0, rows], want, HALF["bf16"] * want.abs() + 2 * O * STEP32 * mag)
    want = torch.zeros(O, C, dtype=torch.float64, device="cuda")
    for i in range(0, n, part):
        want += dy[0, i:i + part].double().t().contiguous() @ x[0, i:i + part].double()
    check("dweight", out["dweight"], want, HALF["bf16"] * want.abs())


# aligned shapes with edges in their tiles, contractions that end inside a stage, images shorter and longer than a
# stage (every kernel that the products can take: test_project_tiles.py)
TILES = [(1, 200, 328, 700, 1, "nhwc"), (3, 136, 264, 40, 24, "nchw"), (2, 1096, 520, 33, 16, "nhwc"),
         (5, 64, 72, 8, 9, "nchw"), (300, 328, 264, 1, 1, "nhwc"), (64, 24, 2056, 72, 1, "nhwc"), (40, 2056, 24, 8, 10, "nchw"),
         (9, 1032, 1544, 1000, 1, "nhwc"), (10, 1544, 1032, 24, 25, "nchw")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", TILES, ids=str)
def test_tiles(size, dtype):
    B, C, O, H, W, layout = size
    act, scale, shift, residual = KINDS[TILES.index(size) % len(KINDS)]
    t = make(B, C, O, H, W, dtype, layout, act, scale, shift, seed=7)
    res, z = t["residual"] if residual else None, torch.empty_like(t["z"])
    y = t["layer"].forward(t["x"], residual=res, z=z)
    check_forward(t, dtype, layout, act, res, y, z)
    check_backward(t, dtype, layout, act, t["layer"].backward(t["x"], t["dy"], z=t["z"], residual=residual))


@pytest.mark.parametrize("size", [(1, 96, 64, 300, 1, "nhwc"), (2, 512, 512, 20, 16, "nchw"), (1, 33, 20, 70, 1, "nhwc"),
                                  (1, 300, 24, 6, 1, "nhwc")], ids=str)
@pytest.mark.parametrize("scale", [1e-35, 1e-20, 1e18])
def test_float32_keeps_its_bits_at_any_size_of_the_values(size, scale):
    """float32 products at the ends of the range, and beside values of ordinary size."""
    B, C, O, H, W, layout = size
    t = make(B, C, O, H, W, "f32", layout, "none", seed=11)
    t["x"].mul_(scale)
    t["dy"].mul_(scale)
    if layout == "nhwc":
        t["x"][..., : C // 2].div_(scale)
    else:
        t["x"][:, : C // 2].div_(scale)
    check_forward(t, "f32", layout, "none", None, t["layer"].forward(t["x"]), None)
    out = t["layer"].backward(t["x"], t["dy"])
    dx, mag = rows(t["dy"], layout) @ t["w"].double(), rows(t["dy"], layout).abs() @ t["w"].double().abs()
    check("dx", rows(out["dx"], layout), dx, HALF["f32"] * 1.01 * dx.abs() + (O + 8) * STEP32 * mag + 2.0 ** -149)


def test_float32_values_that_are_not_finite():
    """Infinities meet weights without lower bits, zeros and each other as in float32 arithmetic."""
    x = torch.randn(200, 64, device="cuda")
    w = torch.randn(72, 64, device="cuda")
    w[5], w[6, 3] = 1.0, 0.0
    x[7, 3], x[8, 3], x[9, 3], x[9, 4] = float("inf"), float("-inf"), float("inf"), float("-inf")
    x[150, 10] = float("nan")
    x[30], w[8] = 3e38, 1.5
    y = ProjectLayer(w).forward(x)
    want = x.cpu() @ w.cpu().t()
    kind = torch.where(torch.isnan(want), 2.0, torch.where(torch.isinf(want), want.sign() * 1.0, torch.zeros_like(want)))
    got = y.cpu()
    kind_got = torch.where(torch.isnan(got), 2.0, torch.where(torch.isinf(got), got.sign() * 1.0, torch.zeros_like(got)))
    rest = torch.ones(200, dtype=torch.bool)
    rest[30] = False          # sums that overflow on the way go by their order
    assert torch.equal(kind_got[rest], kind[rest])
    fine = rest[:, None] & torch.isfinite(want)
    mag = x.cpu().abs().nan_to_num(0.0, 0.0, 0.0).double() @ w.cpu().abs().double().t()
    assert ((got.double() - want.double()).abs()[fine] <= (80 * STEP32 * mag + 1e-30)[fine]).all()


def test_gelu_relative_to_its_value():
    """bfloat16 GELU and its slope at every bfloat16 argument down to where the values leave the normal numbers: half a
    step of the value and 2^-12 of it for the evaluation (the slope, which passes through zero, 3e-7 beside that)."""
    bits = torch.arange(1 << 15, dtype=torch.int32)
    v = (bits << 16).view(torch.float32)
    v = v[(v >= 2.0 ** -60) & (v <= 12.9)]
    v = torch.cat([-v, v])
    v = v[: v.numel() // 8 * 8].cuda().bfloat16()
    want = act64(v.double(), "gelu")
    tol = (HALF["bf16"] * 1.01 + 2.0 ** -12) * want.abs() + 2.0 ** -122
    one = ProjectLayer(torch.ones(1, 1, dtype=v.dtype, device="cuda"), act="gelu")
    eye = ProjectLayer(torch.eye(8, dtype=v.dtype, device="cuda"), act="gelu")
    check("tiles", eye.forward(v.view(-1, 8)).view(-1), want, tol)
    check("elements", one.forward(v.view(-1, 1)).view(-1), want, tol)
    few = v.view(-1, 8)[:: v.numel() // 8 // 30][:30].contiguous()
    w = act64(few.double(), "gelu")
    check("few rows", eye.forward(few), w, (HALF["bf16"] * 1.01 + 2.0 ** -12) * w.abs() + 2.0 ** -122)
    slope = eye.backward(v.view(-1, 8), torch.ones_like(v).view(-1, 8), z=v.view(-1, 8), residual=True)["dresidual"]
    w = act_grad64(v.double(), "gelu")
    check("slope", slope.view(-1), w, (HALF["bf16"] * 1.01 + 2.0 ** -12) * w.abs() + 3e-7)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 8, 8, 1, 1, "nhwc"), (2, 65, 63, 33, 1, "nhwc"), (4, 128, 256, 16, 9, "nhwc"),
                                  (3, 33, 31, 7, 7, "nchw"), (5, 72, 40, 8, 8, "nchw"), (1, 7, 300, 130, 1, "nhwc")], ids=str)
def test_the_scale_of_a_smooth_activation_has_its_gradient(size, dtype, act):
    B, C, O, H, W, layout = size
    t = make(B, C, O, H, W, dtype, layout, act, scale=True, shift=True, seed=3)
    layer = t["layer"]
    out = layer.backward(t["x"], t["dy"], z=t["z"], residual=True)
    assert set(out) == {"dx", "dweight", "dscale", "dshift", "dresidual"}
    check_backward(t, dtype, layout, act, out)
    # the same bits without dresidual, in a workspace of the size that the layer gives, and captured
    ws = torch.empty(layer.backward_workspace_bytes(t["x"].shape), dtype=torch.uint8, device="cuda")
    again = layer.backward(t["x"], t["dy"], z=t["z"], ws=ws)
    assert set(again) == {"dx", "dweight", "dscale", "dshift"}
    assert all(torch.equal(again[n], out[n]) for n in again)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer.backward(t["x"], t["dy"], z=t["z"], ws=ws)
    for f in (1.0, -0.5, 2.0):
        t["dy"].mul_(f)
        want = layer.backward(t["x"], t["dy"], z=t["z"])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[n], want[n]) for n in want)


def test_the_scale_of_a_smooth_activation_against_differences():
    t = make(2, 12, 10, 3, 4, "f32", "nchw", "gelu", scale=True, shift=True)

    def loss(scale):
        y = ProjectLayer(t["w"], scale, t["shift"], act="gelu", layout="nchw").forward(t["x"])
        return float((y.double() * t["dy"].double()).sum())

    z = torch.empty_like(t["dy"])
    t["layer"].forward(t["x"], z=z)
    got = t["layer"].backward(t["x"], t["dy"], z=z)["dscale"]
    h = 2.0 ** -6      # as above: off by h^2 / 6 of a third derivative and by roundings over h
    for i in range(10):
        a, b = t["scale"].clone(), t["scale"].clone()
        a[i] += h
        b[i] -= h
        d = (loss(a) - loss(b)) / (2 * h)
        assert abs(d - float(got[i])) <= 2e-3 * max(1.0, float(got.abs().max())), i


@pytest.mark.parametrize("O,C", [(4, 0), (0, 4), (0, 0)])
def test_a_weight_without_channels_is_refused(O, C):
    """A sum over no channels is none that the kernels form: the call would have to return act(shift + residual)."""
    with pytest.raises(ValueError):
        ProjectLayer(torch.empty(O, C, device="cuda"))


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(4, 24, 16, 257, 257, "nchw"), (4, 24, 16, 256, 260, "nchw"), (7, 40, 24, 200, 200, "nchw"),
                                  (1, 24, 16, 512, 520, "nchw"), (4, 24, 16, 257, 257, "nhwc"), (9, 23, 13, 181, 163, "nhwc"),
                                  (9000, 23, 13, 4, 7, "nchw")], ids=str)
def test_sums_of_whole_numbers_over_many_positions(size, dtype, act):
    """Every partial sum is a whole number below 2^24 (a half of one for dscale and dx) and so exact in float32: a
    position that is lost or counted twice shows, and the gradients are the exact ones rounded once."""
    B, C, O, H, W, layout = size
    g = torch.Generator(device="cuda").manual_seed(B + C)
    dt, xs, ys = TYPES[dtype], (B, C, H, W), (B, O, H, W)
    if layout == "nhwc":
        xs, ys = (B, H, W, C), (B, H, W, O)

    def whole(shape, lo, hi, t):
        return torch.empty(shape, device="cuda").random_(lo, hi + 1, generator=g).to(t)

    # means that are not zero, so that no part of the positions adds up to nothing
    x, dy, z = whole(xs, -1, 3, dt), whole(ys, -1, 2, dt), whole(ys, -1, 1, dt)
    w, shift = whole((O, C), -2, 2, dt), whole((O,), -3, 3, torch.float32)
    scale = 2.0 ** whole((O,), -1, 1, torch.float32) * torch.where(whole((O,), 0, 1, torch.float32) > 0, 1.0, -1.0)
    layer = ProjectLayer(w, scale, shift, act=act, layout=layout)
    out = layer.backward(x, dy, z=z if act == "relu" else None, residual=True)
    xd, wd, dz = rows(x, layout), w.double(), rows(dy, layout)
    if act == "relu":
        dz = torch.where(rows(z, layout) > 0, dz, torch.zeros_like(dz))
    assert float((dz.abs().t() @ xd.abs()).max()) < 2.0 ** 24
    G = dz.t() @ xd
    assert float((wd.abs() * G.abs()).sum(1).max()) < 2.0 ** 24
    assert torch.equal(out["dshift"], dz.sum(0).float())
    assert torch.equal(out["dscale"], (wd * G).sum(1).float())
    assert torch.equal(out["dweight"], (scale.double()[:, None] * G).to(dt))
    assert torch.equal(rows(out["dresidual"], layout), dz)
    assert torch.equal(rows(out["dx"], layout), ((dz * scale.double()) @ wd).to(dt).double())


def arena(nbytes, guard=4096):
    """nbytes of device memory between guards of a fixed pattern, aligned to 256 bytes: the whole, and the middle."""
    whole = torch.full((nbytes + 2 * guard + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    at = guard + -(whole.data_ptr() + guard) % 256
    return whole, whole[at:at + nbytes], at


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 72, 50, 37, 1, "nhwc"), (3, 72, 48, 7, 9, "nchw"), (2, 40, 64, 8, 4, "nchw"),
                                  (1, 1030, 13, 3, 1, "nhwc"), (2, 45, 541, 19, 1, "nhwc"), (5000, 9, 17, 2, 3, "nchw"),
                                  (4100, 8, 16, 4, 2, "nchw"), (1, 100, 700, 1, 1, "nhwc"), (2, 700, 20, 13, 11, "nchw"),
                                  (3, 260, 68, 60, 70, "nhwc"), (1, 1036, 516, 40, 1, "nhwc")], ids=str)
def test_every_output_and_the_workspace_end_where_they_end(size, dtype):
    """The calls themselves, with every output in memory of its own size and the workspace in what the query says."""
    B, C, O, H, W, layout = size
    for act, scale in (("relu", True), ("gelu", False), ("none", True), ("silu", True)):
        t = make(B, C, O, H, W, dtype, layout, act, scale, True, seed=2)
        layer, x, st = t["layer"], t["x"], torch.cuda.current_stream()
        d = layer.desc(x.shape)
        smooth = act in ("gelu", "silu")
        like = {"y": t["dy"], "z": t["dy"], "dx": x, "dweight": t["w"], "dshift": t["shift"], "dresidual": t["dy"]}
        if scale and not smooth:
            like["dscale"] = t["scale"]
        sizes = {n: v.numel() * v.element_size() for n, v in like.items()}
        sizes.update(ws=layer.workspace_bytes(x.shape), bws=layer.backward_workspace_bytes(x.shape))
        held = {n: arena(b) for n, b in sizes.items()}
        out = {n: held[n][1].view(v.dtype).view(v.shape) for n, v in like.items()}
        ws, bws = held["ws"][1], held["bws"][1]
        mb.moce_project(d, x, t["w"], t["scale"], t["shift"], t["residual"], out["y"], out["z"], ws if sizes["ws"] else None,
                        sizes["ws"], st)
        grads = {n: out[n] for n in out if n not in ("y", "z")}
        mb.moce_project_backward(d, x, t["w"], t["scale"], t["z"], t["dy"], mb.make_project_grads(**grads), bws,
                                 sizes["bws"], st)
        torch.cuda.synchronize()
        for n, (whole, _, at) in held.items():
            assert (whole[:at] == 0xA5).all() and (whole[at + sizes[n]:] == 0xA5).all(), n
        check_forward(t, dtype, layout, act, t["residual"], out["y"], out["z"])
        check_backward(t, dtype, layout, act, grads)
