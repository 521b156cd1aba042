"""Group norm with an activation and its gradients on the GPU, against float64."""
import math

import pytest
import torch

from paper_2608_23794_amd import binding as mb
from paper_2608_23794_amd.layer import GroupNormLayer

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
# What the float32 sums lose, relative to a standard deviation.  A sum of m
# values is off by at most m 2^-24 of the sum of their sizes; a thread adds up
# to 64 of them before sums are joined, the deviations from the value it takes
# them about are up to about 8 standard deviations on average in an unlucky
# thread (so the mean is off by 64 x 8 x 2^-24 = 2^-15 of one), and the squares'
# sum by as much of itself.
SUMS = 2.0 ** -14

SHAPES = [
    # B, C, G, H, W
    (1, 1, 1, 1, 1), (1, 1, 1, 7, 3), (2, 8, 8, 1, 1), (3, 12, 4, 1, 1), (1, 64, 1, 1, 1), (5, 7, 7, 5, 3),
    (2, 6, 3, 2, 2), (1, 512, 32, 7, 7), (2, 330, 11, 9, 9), (3, 32, 32, 16, 16), (2, 256, 32, 14, 14),
    (1, 96, 3, 197, 1), (4, 768, 1, 5, 1), (2, 40, 5, 33, 17), (1, 17, 1, 64, 65), (1, 24, 2, 300, 301),
    (70, 16, 4, 3, 3), (1, 2056, 8, 4, 4), (2, 8, 2, 128, 256), (9, 100, 50, 12, 1), (1, 5000, 5000, 2, 3),
]


def act64(z, kind):
    if kind == "relu":
        return z.clamp(min=0), (z > 0).double()
    if kind == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)


def channels_first(t, layout):
    """[B, C, positions]"""
    return t.reshape(t.shape[0], t.shape[1], -1) if layout == "nchw" else t.reshape(
        t.shape[0], -1, t.shape[-1]).transpose(1, 2)


def reference(x, dy, scale, shift, G, eps, act, layout, stats=None):
    """In float64, [B, C, positions] each, beside the statistics [B, C, 1]."""
    x, dy = channels_first(x.double(), layout), channels_first(dy.double(), layout)
    B, C, P = x.shape
    v = x.reshape(B, G, -1)
    mean = v.mean(2, keepdim=True)
    rstd = 1 / torch.sqrt((v - mean).square().mean(2, keepdim=True) + eps)

    def wide(t):
        return t.reshape(B, G, 1).expand(B, G, C // G).reshape(B, C, 1)

    def grouped_mean(t):
        return wide(t.reshape(B, G, -1).mean(2))

    m, r = wide(mean), wide(rstd)
    h = (x - m) * r
    a = scale.double().reshape(1, C, 1) if scale is not None else torch.ones(1, C, 1, dtype=torch.float64, device="cuda")
    b = shift.double().reshape(1, C, 1) if shift is not None else torch.zeros_like(a)
    z = a * h + b
    y, slope = act64(z, act)
    dz = slope * dy
    t = a * dz
    dx = r * (t - grouped_mean(t) - h * grouped_mean(t * h))
    return dict(mean=mean.reshape(B, G), rstd=rstd.reshape(B, G), m=m, r=r, h=h, z=z, y=y, dz=dz, t=t, dx=dx, a=a, dy=dy,
                grouped_mean=grouped_mean)


def make(shape, dtype, layout, seed=0, mean=1.0, affine=True):
    B, C, G, H, W = shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = (B, C, H, W) if layout == "nchw" else (B, H, W, C)
    x = torch.randn(s, generator=g, device="cuda") + mean
    dy = torch.randn(s, generator=g, device="cuda")
    scale = 1 + 0.3 * torch.randn(C, generator=g, device="cuda") if affine else None
    shift = 0.3 * torch.randn(C, generator=g, device="cuda") if affine else None
    return x.to(TYPES[dtype]), dy.to(TYPES[dtype]), scale, shift


def tolerances(ref, dtype, act, G):
    """h, z and y of a forward whose mean and rstd are float32."""
    h = SUMS * (1 + ref["h"].abs()) + ref["m"].abs() * ref["r"] * 2.0 ** -23
    z = ref["a"].abs() * h + 2.0 ** -23 * ref["z"].abs()
    # slopes of the activations are below 1.13; bfloat16 evaluates them to 2^-12, float32 to a few steps
    y = 1.13 * z + (2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -21) * ref["y"].abs()
    return h, z, y + HALF[dtype] * (ref["y"].abs() + y) + 2.0 ** -100


def check_forward(y, stats, ref, dtype, act, G, layout):
    h, z, tol = tolerances(ref, dtype, act, G)
    assert ((channels_first(y.double(), layout) - ref["y"]).abs() <= tol).all()
    std = 1 / ref["rstd"]
    assert ((stats[0].double() - ref["mean"]).abs() <= SUMS * std + 2.0 ** -24 * ref["mean"].abs()).all()
    assert ((stats[1].double() - ref["rstd"]).abs() <= SUMS * ref["rstd"]).all()


def check_backward(out, ref, dtype, act, layout):
    h, z, _ = tolerances(ref, dtype, act, None)
    mean = ref["grouped_mean"]
    # slopes' own slopes are below 1.3; at the corner of ReLU either side is right
    corner = (ref["z"].abs() <= z).double() if act == "relu" else torch.zeros_like(z)
    dz = ref["dy"].abs() * (corner + (0 if act in ("none", "relu") else 1.3 * z + 2.0 ** -12)) + 2.0 ** -22 * ref["dz"].abs()
    t, e = ref["t"].abs(), ref["a"].abs() * dz
    th = t * h + e * (ref["h"].abs() + h)
    tol = ref["r"] * (e + mean(e) + h * mean(t * ref["h"].abs()) + (ref["h"].abs() + h) * mean(th)
                      + 2.0 ** -18 * (t + mean(t) + ref["h"].abs() * mean(t * ref["h"].abs())))
    dx = channels_first(out["dx"].double(), layout)
    assert ((dx - ref["dx"]).abs() <= tol + HALF[dtype] * (ref["dx"].abs() + tol) + 2.0 ** -100).all()
    if "dshift" in out:
        w = (ref["dz"].abs() * 2.0 ** -18 + dz).sum((0, 2))
        assert ((out["dshift"].double() - ref["dz"].sum((0, 2))).abs() <= w).all()
    if "dscale" in out:
        dzh = ref["dz"] * ref["h"]
        w = (dzh.abs() * 2.0 ** -18 + ref["dz"].abs() * h + dz * (ref["h"].abs() + h)).sum((0, 2))
        assert ((out["dscale"].double() - dzh.sum((0, 2))).abs() <= w).all()


ACTS = ["none", "relu", "gelu", "silu"]

# Larger ones, through parts of an image: parts joined by their readers or by a launch, groups that end inside a
# workgroup's channels, whole and ragged rows, many and few parts, groups of all channels.
PARTS = [
    (2, 64, 8, 120, 130), (1, 256, 8, 100, 90), (3, 36, 9, 150, 60), (1, 512, 2, 90, 90), (20, 128, 32, 80, 80),
    (1, 1030, 103, 40, 41), (1, 520, 65, 64, 70), (1, 768, 1, 300, 20), (4, 33, 3, 200, 100), (300, 24, 3, 60, 70),
    (2, 2, 1, 700, 700), (1, 1024, 1024, 80, 80), (70, 256, 32, 56, 56), (64, 512, 32, 28, 28), (16, 100, 5, 64, 64),
]


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PARTS)
def test_larger_ones(shape, dtype, layout):
    i = PARTS.index(shape)
    act = ACTS[(i + (dtype == "bf16") + 2 * (layout == "nchw")) % 4]
    x, dy, scale, shift = make(shape, dtype, layout, seed=100 + i)
    layer = GroupNormLayer(shape[2], scale, shift, act=act, layout=layout)
    stats = layer.new_stats(x.shape)
    y = layer.forward(x, stats=stats)
    ref = reference(x, dy, scale, shift, shape[2], 1e-5, act, layout)
    check_forward(y, stats, ref, x.dtype, act, shape[2], layout)
    out = layer.backward(x, dy, stats)
    check_backward(out, ref, x.dtype, act, layout)
    again = layer.backward(x, dy, stats)
    assert torch.equal(layer.forward(x), y) and all(torch.equal(again[n], out[n]) for n in out)
    # the parameters' gradients without dx
    n = mb.moce_group_norm_backward_workspace_bytes(layer.desc(x.shape, x.dtype))
    ws, some = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.full_like(scale, 7.0)
    mb.moce_group_norm_backward(layer.desc(x.shape, x.dtype), x, scale, shift, stats, dy,
                                mb.make_group_norm_grads(dscale=some), ws, n, torch.cuda.current_stream())
    assert torch.equal(some, out["dscale"])


@pytest.mark.parametrize("shape,layout", [((600, 64, 8, 65536, 1), "nhwc"), ((40, 32, 4, 1400, 1300), "nchw")])
def test_offsets_past_32_bits(shape, layout):
    """Images behind 2^31 elements as they are by themselves: a copy of the first ones at the end."""
    B, C, G, H, W = shape
    assert B * C * H * W > 1 << 31
    s = (B, C, H, W) if layout == "nchw" else (B, H, W, C)
    x = torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_()
    x[-1] = x[0]
    layer = GroupNormLayer(G, torch.rand(C, device="cuda") + 0.5, torch.rand(C, device="cuda"), act="relu", layout=layout)
    stats = layer.new_stats(x.shape)
    y = layer.forward(x, stats=stats)
    assert torch.equal(y[-1], y[0]) and torch.equal(stats[:, -1], stats[:, 0])
    ref = reference(x[-1:], x[-1:], layer.scale, layer.shift, G, 1e-5, "relu", layout)
    check_forward(y[-1:], stats[:, -1:], ref, x.dtype, "relu", G, layout)
    del ref
    out = layer.backward(x, x, stats, dx=y)
    assert torch.equal(out["dx"][-1], out["dx"][0])


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype, layout):
    i = SHAPES.index(shape)
    act, affine = ACTS[(i + (dtype == "bf16") + 2 * (layout == "nchw")) % 4], i % 3 != 2
    x, dy, scale, shift = make(shape, dtype, layout, seed=i, affine=affine)
    layer = GroupNormLayer(shape[2], scale, shift, eps=1e-5, act=act, layout=layout)
    stats = layer.new_stats(x.shape)
    y = layer.forward(x, stats=stats)
    ref = reference(x, dy, scale, shift, shape[2], 1e-5, act, layout)
    check_forward(y, stats, ref, x.dtype, act, shape[2], layout)
    out = layer.backward(x, dy, stats)
    assert set(out) == ({"dx", "dscale", "dshift"} if affine else {"dx"})
    check_backward(out, ref, x.dtype, act, layout)
    # the same bits again, without statistics kept, in place
    assert torch.equal(layer.forward(x), y)
    keep, up = x.clone(), dy.clone()
    assert torch.equal(layer.backward(x, up, stats, dx=up)["dx"], out["dx"])
    assert torch.equal(layer.backward(keep, dy, stats, dx=keep)["dx"], out["dx"])
    assert torch.equal(layer.forward(x, y=x), y)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, layout):
    shape = (2, 48, 6, 10, 11)
    for dtype in TYPES:
        x, dy, scale, shift = make(shape, dtype, layout, seed=7)
        layer = GroupNormLayer(6, scale * 3, None, act=act, layout=layout)
        stats = layer.new_stats(x.shape)
        y = layer.forward(x, stats=stats)
        ref = reference(x, dy, scale * 3, None, 6, 1e-5, act, layout)
        check_forward(y, stats, ref, x.dtype, act, 6, layout)
        out = layer.backward(x, dy, stats)
        assert set(out) == {"dx", "dscale"}
        check_backward(out, ref, x.dtype, act, layout)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape", [(2, 64, 8, 28, 28), (1, 32, 4, 160, 160), (3, 64, 64, 9, 1)])
def test_a_mean_that_is_large_against_the_deviation(shape, layout):
    x, dy, scale, shift = make(shape, "f32", layout, seed=3, mean=4096.0)
    layer = GroupNormLayer(shape[2], scale, shift, layout=layout)
    stats = layer.new_stats(x.shape)
    y = layer.forward(x, stats=stats)
    check_forward(y, stats, reference(x, dy, scale, shift, shape[2], 1e-5, "none", layout), x.dtype, "none", shape[2],
                  layout)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("size", [(3, 64, 8, 7, 7), (2, 32, 8, 90, 90)])
def test_groups_apart(size, layout):
    """Constant groups, an outlier, and values that are not finite: each in its own group only."""
    B, C, G, H, W = size
    x, dy, scale, shift = make(size, "f32", layout, seed=5)
    v = channels_first(x, layout).unflatten(1, (G, C // G))     # views of x
    base = GroupNormLayer(G, scale, shift, act="silu", layout=layout)
    clean = base.forward(x)
    v[0, 0] = 2.5                       # no deviation: h is 0
    v[0, 1, 0, 0] = 1e6                 # an outlier, where a thread begins
    v[1, 2, 1, 3] = math.nan
    v[1, 3, 0, 1] = math.inf
    v[1, 4, 2, 5] = -math.inf
    stats = base.new_stats(x.shape)
    y = base.forward(x, stats=stats)
    out = channels_first(y, layout).unflatten(1, (G, C // G))
    want = channels_first(clean, layout).unflatten(1, (G, C // G))
    z = shift.reshape(G, C // G)[0].double()
    tol = 2.0 ** -20 * (1 + z.abs())
    assert ((out[0, 0].double() - (z * torch.sigmoid(z))[:, None]).abs() <= tol[:, None]).all()
    for g in (2, 3, 4):
        assert out[1, g].isnan().all()
    touched = {(0, 0), (0, 1), (1, 2), (1, 3), (1, 4)}
    for b in range(B):
        for g in range(G):
            if (b, g) not in touched:
                assert torch.equal(out[b, g], want[b, g])
    one = v[0, 1].double()
    mean = one.mean()
    rstd = 1 / torch.sqrt((one - mean).square().mean() + 1e-5)
    assert abs(float(stats[0, 0, 1]) - float(mean)) <= SUMS / float(rstd)
    assert abs(float(stats[1, 0, 1] / rstd) - 1) <= SUMS


def test_differences():
    """The gradients against differences of the forward along a direction, float32."""
    for layout in ("nchw", "nhwc"):
        x, dy, scale, shift = make((2, 12, 3, 6, 5), "f32", layout, seed=11)
        layer = GroupNormLayer(3, scale, shift, act="gelu", layout=layout)
        stats = layer.new_stats(x.shape)
        layer.forward(x, stats=stats)
        out = layer.backward(x, dy, stats)
        g = torch.Generator(device="cuda").manual_seed(1)
        d = torch.randn(x.shape, generator=g, device="cuda")
        e = 2.0 ** -7
        # differences are right to e^2 of the third derivative (of order 10 |dy| |d|^3), and lose 2^-24 |y| / e a value
        n = x.numel()
        tol = 10 * e * e * float(dy.abs().sum()) + 2.0 ** -21 / e * n ** 0.5 * 3

        def diff(f):
            return float((dy.double() * (f(e).double() - f(-e).double())).sum()) / (2 * e)

        assert abs(diff(lambda s: layer.forward(x + s * d)) - float((out["dx"].double() * d).sum())) <= tol
        c = torch.randn(12, generator=g, device="cuda")
        got = diff(lambda s: GroupNormLayer(3, scale + s * c, shift, act="gelu", layout=layout).forward(x))
        assert abs(got - float((out["dscale"].double() * c).sum())) <= tol
        got = diff(lambda s: GroupNormLayer(3, scale, shift + s * c, act="gelu", layout=layout).forward(x))
        assert abs(got - float((out["dshift"].double() * c).sum())) <= tol


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape", [(2, 24, 3, 5, 7), (1, 33, 11, 13, 9), (2, 64, 8, 40, 40), (3, 16, 4, 1, 1)])
def test_memory_around_stays(shape, layout):
    """Outputs and workspace between guards of 256 bytes."""
    for dtype in TYPES:
        x, dy, scale, shift = make(shape, dtype, layout, seed=2)
        layer = GroupNormLayer(shape[2], scale, shift, act="relu", layout=layout)

        def guarded(t, dt, shape):
            n = math.prod(shape)
            pad = 256 // torch.empty(0, dtype=dt).element_size()
            buf = torch.full((n + 2 * pad,), 77, dtype=dt, device="cuda")
            return buf, buf[pad:pad + n].reshape(shape), pad

        bufs = []

        def new(dt, shape):
            buf, view, pad = guarded(None, dt, shape)
            bufs.append((buf, pad, view.numel()))
            return view

        y, stats = new(x.dtype, x.shape), new(torch.float32, (2, shape[0], shape[2]))
        ws = new(torch.uint8, (layer.workspace_bytes(x.shape, x.dtype),))
        layer.forward(x, y=y, stats=stats, ws=ws)
        dx, wb = new(x.dtype, x.shape), new(torch.uint8, (layer.backward_workspace_bytes(x.shape, x.dtype),))
        layer.backward(x, dy, stats, dx=dx, ws=wb)
        torch.cuda.synchronize()
        assert torch.equal(y, layer.forward(x)) and torch.equal(dx, layer.backward(x, dy, stats)["dx"])
        for buf, pad, n in bufs:
            assert (buf[:pad] == 77).all() and (buf[pad + n:] == 77).all()


def test_on_another_stream_and_captured():
    x, dy, scale, shift = make((8, 64, 8, 20, 20), "bf16", "nhwc", seed=4)
    layer = GroupNormLayer(8, scale, shift, act="silu")
    stats, y, dx = layer.new_stats(x.shape), torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(layer.workspace_bytes(x.shape, x.dtype), dtype=torch.uint8, device="cuda")
    wb = torch.empty(layer.backward_workspace_bytes(x.shape, x.dtype), dtype=torch.uint8, device="cuda")

    def step():
        layer.forward(x, y=y, stats=stats, ws=ws)
        return layer.backward(x, dy, stats, dx=dx, ws=wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(torch.randn_like(x.float()) * (i + 1) + i)
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone(), stats.clone(), dx.clone(), out["dscale"].clone(), out["dshift"].clone()]
        again = layer.new_stats(x.shape)
        want_y = layer.forward(x, stats=again)
        want = layer.backward(x, dy, again)
        for a, b in zip(got, [want_y, again, want["dx"], want["dscale"], want["dshift"]]):
            assert torch.equal(a, b)


def test_empty_and_refusals():
    dev = "cuda"
    layer = GroupNormLayer(4, torch.ones(8, device=dev), torch.zeros(8, device=dev))
    for shape in [(0, 5, 8), (3, 0, 8)]:
        x = torch.empty(shape, device=dev)
        stats = layer.new_stats(shape)
        assert layer.forward(x, stats=stats).shape == shape
        out = layer.backward(x, x, stats)
        assert out["dx"].shape == shape and float(out["dscale"].abs().sum()) == 0.0
    x = torch.randn(2, 5, 8, device=dev)
    for bad in (x.double(), x.cpu(), x[:, :, :4], x.transpose(0, 1), torch.randn(2, 5, 12, device=dev)):
        with pytest.raises(ValueError):
            layer.forward(bad)
    with pytest.raises(ValueError):
        layer.forward(x, y=torch.empty(2, 5, 8, dtype=torch.bfloat16, device=dev))
    with pytest.raises(ValueError):
        layer.forward(x, stats=torch.empty(2, 2, 8, device=dev))
    with pytest.raises(mb.MoceError):
        layer.forward(x, ws=torch.empty(0, dtype=torch.uint8, device=dev))
    with pytest.raises(ValueError):
        GroupNormLayer(3, torch.ones(8, device=dev))
    with pytest.raises(ValueError):
        GroupNormLayer(4, torch.ones(8, device=dev), torch.ones(4, device=dev))
    with pytest.raises(ValueError):
        GroupNormLayer(4, torch.ones(8))
    with pytest.raises(ValueError):
        GroupNormLayer(3).forward(x)
    for kw in (dict(groups=0), dict(groups=4, eps=-1.0), dict(groups=4, eps=math.inf), dict(groups=4, act="tanh"),
               dict(groups=4, layout="chw")):
        with pytest.raises(ValueError):
            GroupNormLayer(**kw)


@pytest.mark.parametrize("dtype,B,H,W,layout", [
    ("bf16", 1, 46340, 46340, "nchw"), ("bf16", 2, (1 << 31) - 1, 1, "nhwc"), ("f32", 1, (1 << 31) - 1, 1, "nchw"),
])
def test_a_plane_of_all_positions_there_can_be(dtype, B, H, W, layout):
    """One channel whose last part ends at 2^31 - 1 positions, or whose parts' multiples pass it.

    The last 174096 positions hold other values, so that statistics and sums without them are far off: their mean of 40
    adds 0.13 to a variance of 1, their dy of 30 adds 5.2e6 to dshift.  A lane adds up to 2^13 values before its sums
    are joined, so sums are right to 2^13 x 2^-24 = 2^-11 of their values' sizes, which are about one deviation: a mean
    to 2^-10 of one (sums are taken about a lane's first value, itself about one away), rstd to 2^-10 of itself."""
    n, last, chunk = H * W, 174096, 1 << 26
    shape = (B, 1, H, W) if layout == "nchw" else (B, H, W, 1)
    x = torch.empty((B, n), dtype=TYPES[dtype], device="cuda").normal_(0.5, 1.0)
    dy = torch.empty_like(x).normal_()
    x[:, -last:] += 40
    dy[:, -last:] = 30
    scale, shift = torch.full((1,), 1.5, device="cuda"), torch.full((1,), 0.25, device="cuda")
    layer = GroupNormLayer(1, scale, shift, layout=layout)
    stats = layer.new_stats(shape)
    y = torch.full_like(x, math.nan)
    layer.forward(x.view(shape), y=y.view(shape), stats=stats)

    def sums(b, f):
        return sum(f(slice(i, i + chunk)).sum() for i in range(0, n, chunk))

    m = [sums(b, lambda s: x[b, s].double()) / n for b in range(B)]
    r = [1 / torch.sqrt(sums(b, lambda s: (x[b, s].double() - m[b]).square()) / n + 1e-5) for b in range(B)]
    off = 2.0 ** -10
    for b in range(B):
        assert abs(float((stats[0, b, 0].double() - m[b]) * r[b])) <= off
        assert abs(float(stats[1, b, 0].double() / r[b]) - 1) <= off
        for i in range(0, n, chunk):
            h = (x[b, i:i + chunk].double() - m[b]) * r[b]
            z = 1.5 * h + 0.25
            tol = 1.5 * off * (1 + h.abs()) * 1.01
            tol = tol + HALF[x.dtype] * (z.abs() + tol)
            assert ((y[b, i:i + chunk].double() - z).abs() <= tol).all()
    out = layer.backward(x.view(shape), dy.view(shape), stats, dx=y.fill_(math.nan).view(shape))
    sizes, dshift, dscale, worst = 0.0, 0.0, 0.0, 0.0
    for b in range(B):
        m[b], r[b] = stats[0, b, 0].double(), stats[1, b, 0].double()      # the gradients of these
        t0 = sums(b, lambda s: dy[b, s].double())
        t1 = sums(b, lambda s: dy[b, s].double() * (x[b, s].double() - m[b]) * r[b])
        a0 = sums(b, lambda s: dy[b, s].double().abs())
        a1 = sums(b, lambda s: (dy[b, s].double() * (x[b, s].double() - m[b]) * r[b]).abs())
        dshift, dscale, sizes, worst = dshift + t0, dscale + t1, sizes + a0, worst + a1
        for i in range(0, n, chunk):
            h = (x[b, i:i + chunk].double() - m[b]) * r[b]
            d = dy[b, i:i + chunk].double()
            want = r[b] * 1.5 * (d - t0 / n - h * t1 / n)
            tol = r[b] * 1.5 * (2.0 ** -11 * 1.01 * (a0 + h.abs() * a1) / n + 2.0 ** -20 * (d.abs() + h.abs()))
            tol = tol + HALF[x.dtype] * (want.abs() + tol)
            assert ((y[b, i:i + chunk].double() - want).abs() <= tol).all()
    assert abs(float(out["dshift"][0] - dshift)) <= 2.0 ** -11 * float(sizes)
    assert abs(float(out["dscale"][0] - dscale)) <= 2.0 ** -11 * 1.01 * float(worst)


@pytest.mark.parametrize("C,G", [(64, 8), (60, 6), (96, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_of_a_million_rows(dtype, C, G):
    """dscale and dshift where every row adds a value of the same sign and about the same size.

    A row's dz is dy itself, its h is +-k rstd of float32 (one step of rstd, one of the difference, one of each product:
    less than 8 x 2^-24 of the value together), and the sum over the rows adds no more than its last rounding, 2^-24."""
    B = (1 << 20) + 3
    k = 2.0 ** torch.randint(0, 3, (B, 1), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    x = (k * (1 - 2 * (torch.arange(C, device="cuda") % 2))).to(TYPES[dtype])       # every group's mean is 0
    dy = torch.full_like(x, 0.1)
    layer = GroupNormLayer(G, torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"))
    stats = layer.new_stats(x.shape)
    layer.forward(x, stats=stats)
    out = layer.backward(x, dy, stats)
    one = float(dy[0, 0])
    assert ((out["dshift"].double() - B * one).abs() <= 2.0 ** -23 * B * one).all()
    want = one * (x.double() / torch.sqrt(k.double() ** 2 + 1e-5)).sum(0)
    assert ((out["dscale"].double() - want).abs() <= 2.0 ** -21 * want.abs()).all()


# Even numbers of positions; of as many elements a group that one more or less would show.
EXACT = [
    (2, 64, 8, 7, 8), (3, 16, 4, 12, 10), (4, 512, 32, 14, 14), (2, 256, 32, 100, 90), (1, 64, 8, 120, 100),
    (1, 64, 8, 200, 100), (2, 330, 11, 30, 32), (1, 128, 128, 300, 300), (5, 768, 1, 2, 1), (40, 96, 12, 64, 64),
]


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", EXACT)
def test_statistics_of_whole_numbers(shape, dtype, layout):
    """Channels of +-1, +-2 and +-3, the sign turning with the position: mean 0, and all sums of one thread are exact.

    What is off is what joins add.  A join of two counts, means and squared deviations loses at most 8 x 2^-24 of what
    it adds (a reciprocal, a difference, products) and one rounding, 2^-24, of each sum that it holds; a chain of n of
    them (8 + 2 n) 2^-24 of the squares, half of that of rstd.  Means, of at most 3 in size, each lose a rounding and
    the products' few, on weights 1 / 2, 1 / 3, ..: less than (n + 32) 2^-24 of 3.  The longest chains: 256 threads over the
    16-byte vectors of at most 32 across, channels-last; 6 steps of a wave's lanes, channels-first."""
    B, C, G, H, W = shape
    ve = 4 if dtype == "f32" else 8
    across = 1
    while across < 32 and across * ve < C:
        across *= 2
    joins = 256 // across if layout == "nhwc" else 6
    n = C // G * H * W
    tol = (joins + 8) * 2.0 ** -24
    assert tol < 0.5 / n, "a count that is off by one shows"
    size = 1.0 + torch.arange(C, device="cuda") % 3
    sign = 1.0 - 2.0 * (torch.arange(H * W, device="cuda") % 2)
    x = size[:, None] * sign
    x = x.reshape(1, C, H, W) if layout == "nchw" else x.t().reshape(1, H, W, C)
    x = x.expand(B, *x.shape[1:]).to(TYPES[dtype]).contiguous()
    layer = GroupNormLayer(G, layout=layout)
    stats = layer.new_stats(x.shape)
    layer.forward(x, stats=stats)
    rstd = 1 / torch.sqrt((size.double() ** 2).reshape(G, -1).mean(1) + 1e-5)
    assert (stats[0].abs() <= 3 * (joins + 32) * 2.0 ** -24).all()
    assert ((stats[1].double() / rstd - 1).abs() <= tol).all()
