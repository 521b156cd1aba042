"""A training step of the layers together on the GPU: norm, projection, norm, pooled features, a head's losses against
labels and a teacher, all gradients, their clipping; against torch's own differentiation in float64."""
import pytest
import torch

from paper_2608_23794_amd.layer import GroupNormLayer, HeadLoss, ProjectLayer, clip_gradients

pytestmark = pytest.mark.gpu


def act64(z, kind):
    return torch.relu(z) if kind == "relu" else z * torch.sigmoid(z) if kind == "silu" else z


def norm64(x, G, scale, shift, act):
    B, H, W, C = x.shape
    v = x.reshape(B, H * W, G, C // G)
    m = v.mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt((v - m).square().mean((1, 3), keepdim=True) + 1e-5)
    return act64(((v - m) * r).reshape(B, H, W, C) * scale + shift, act)


def parameters(C, O, V, dtype, g):
    def n(*s, scale=1.0):
        return torch.randn(*s, generator=g, device="cuda") * scale
    return {"scale1": 1 + n(C, scale=0.2), "shift1": n(C, scale=0.2), "project": n(O, C, scale=C ** -0.5).to(dtype),
            "scale2": 1 + n(O, scale=0.2), "shift2": n(O, scale=0.2), "head": n(V, O, scale=O ** -0.5).to(dtype),
            "bias": n(V, scale=0.2)}


def step(p, x, labels, cls, logits, T):
    """The losses and the gradients of their sum, by the layers."""
    norm1 = GroupNormLayer(8, p["scale1"], p["shift1"], act="silu")
    project = ProjectLayer(p["project"])
    norm2 = GroupNormLayer(4, p["scale2"], p["shift2"], act="relu")
    head = HeadLoss(p["head"], p["bias"])
    s1 = norm1.new_stats(x.shape)
    a = norm1.forward(x, stats=s1)
    h = project.forward(a)
    s2 = norm2.new_stats(h.shape)
    f = norm2.forward(h, stats=s2)
    feat = f.float().mean((1, 2)).to(x.dtype)
    sl, st = head.new_saved(feat.shape), head.new_saved(feat.shape, cls.shape[1])
    hard = head.cross_entropy(feat, labels, 0.1, saved=sl)
    soft = head.distill(feat, cls, logits, T, saved=st)
    gl = head.cross_entropy_backward(feat, labels, sl, smoothing=0.1)
    gt = head.distill_backward(feat, cls, logits, st, temperature=T)
    n = f.shape[1] * f.shape[2]
    df = ((gl["dx"].float() + gt["dx"].float()) / n)[:, None, None, :].expand(f.shape).to(x.dtype).contiguous()
    g2 = norm2.backward(h, df, s2)
    gp = project.backward(a, g2["dx"])
    g1 = norm1.backward(x, gp["dx"], s1)
    grads = {"scale1": g1["dscale"], "shift1": g1["dshift"], "project": gp["dweight"], "scale2": g2["dscale"],
             "shift2": g2["dshift"], "head": (gl["dweight"].float() + gt["dweight"].float()).to(x.dtype),
             "bias": gl["dshift"] + gt["dshift"]}
    return hard, soft, grads, g1["dx"]


def inputs(dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, C, O, V, K, Hh = 24, 64, 32, 100, 5, 9
    p = parameters(C, O, V, dtype, g)
    x = torch.randn(B, Hh, Hh, C, generator=g, device="cuda").to(dtype)
    labels = torch.randint(0, V, (B,), generator=g, device="cuda")
    labels[3] = -100
    cls = torch.randint(0, V, (B, K), generator=g, device="cuda")
    logits = torch.randn(B, K, generator=g, device="cuda") * 2
    cls[7] = -1
    return p, x, labels, cls, logits


# The 2-norm of a gradient's error over its own.  float32: sums of at most 24 x 81 terms and 64 channels in chains of
# five layers, each within 2^-14 of its values.  bfloat16: each of the five tensors between the layers is rounded to
# 2^-9 in the mean square (half a step of 2^-8 at most), forward and backward, and the products' operands once more:
# 12 roundings of independent signs, 2^-8 sqrt(12) at most.
BOUND = {torch.float32: 5 * 2.0 ** -14, torch.bfloat16: 2.0 ** -8 * 12 ** 0.5}
# And ReLU's corner, for what lies behind it: its argument z, of deviation 1 and a density of at most 0.5 at 0, is off
# by e, in bfloat16 by three roundings of 2^-9 (a, h and the product's operands): 0.0034 in the mean square.  It then
# falls on the other side in a share E|e| 0.5 = 0.0017 of the places, where dz is another value of its own size; half
# of the places have a dz at all, so the error is sqrt(0.0017 / 0.5) = 0.058 of the norm, beside BOUND.
CORNER = {torch.float32: 0.0, torch.bfloat16: 0.058}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_step(dtype):
    p, x, labels, cls, logits = inputs(dtype)
    T = 2.0
    hard, soft, grads, dx = step(p, x, labels, cls, logits, T)
    q = {n: t.double().requires_grad_() for n, t in p.items()}
    xd = x.double().requires_grad_()
    f = norm64(torch.matmul(norm64(xd, 8, q["scale1"], q["shift1"], "silu"), q["project"].t()), 4, q["scale2"],
               q["shift2"], "relu").mean((1, 2))
    z = torch.matmul(f, q["head"].t()) + q["bias"]
    V = z.shape[1]
    t = torch.full_like(z, 0.1 / V).scatter_add_(1, labels.clamp(min=0)[:, None], torch.full((24, 1), 0.9, dtype=z.dtype,
                                                                                          device="cuda"))
    ok = labels >= 0
    hard64 = -(t * torch.log_softmax(z, 1)).sum(1)[ok].mean()
    there = cls[:, 0] >= 0
    t = torch.zeros_like(z).scatter_add_(1, cls.clamp(min=0), torch.softmax(logits.double() / T, 1))
    soft64 = (T * T * (torch.xlogy(t, t) - t * torch.log_softmax(z / T, 1)).sum(1))[there].mean()
    (hard64 + soft64).backward()
    bound = BOUND[dtype]
    assert abs(float(hard) / hard64.item() - 1) <= bound and abs(float(soft) / soft64.item() - 1) <= bound
    for n, g in list(grads.items()) + [("x", dx)]:
        want = xd.grad if n == "x" else q[n].grad
        far = bound if n in ("head", "bias") else (bound ** 2 + CORNER[dtype] ** 2) ** 0.5
        assert float((g.double() - want).norm()) <= far * float(want.norm()), n
    norm = clip_gradients(list(grads.values()), 0.1)
    want = sum(float(q[n].grad.square().sum()) for n in q) ** 0.5
    assert abs(float(norm) / want - 1) <= bound
    after = sum(float(g.double().square().sum()) for g in grads.values()) ** 0.5
    assert after <= 0.1 * (1 + bound)


def test_step_captured():
    """The whole step replayed from a graph, with new inputs: the bits of the eager step."""
    p, x, labels, cls, logits = inputs(torch.bfloat16)

    def run():
        hard, soft, grads, dx = step(p, x, labels, cls, logits, 2.0)
        out = list(grads.values())
        norm = clip_gradients(out, 0.1)
        return [hard, soft, dx, norm] + out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for seed in range(1, 5):
        _, x2, l2, c2, t2 = inputs(torch.bfloat16, seed)
        for a, b in ((x, x2), (labels, l2), (cls, c2), (logits, t2)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, b in zip(got, run()):
            assert torch.equal(a, b)
