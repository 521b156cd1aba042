"""The operators beside the channel-expert layer, as a program that uses them has them done, for timing and comparison.

A case is one pass of one operator:
    "project"   a dense pointwise projection with its epilogue: y = act(scale x W^T + shift + residual)
    "backward"  its gradients for an upstream gradient and the pre-activation that the forward saved
    "clip"      the global norm over a list of gradients, and their clipping to a largest norm

Where ``own`` is false, ``run`` computes them in elementary torch operations in
32 bits; where it is true it calls this package.  ``exact`` has them in 64 bits.

Fields of a projection: B images of C channels over H x W positions (tokens: H
of them, W = 1) to O outputs; dtype "bf16" or "f32"; layout "nchw" or "nhwc";
act "none", "relu", "gelu" or "silu"; scale, shift, residual: what the epilogue
has; save: the pre-activation z is an output too (a training forward).
Fields of a clip: net, the list of gradients ("layer", "resnet" or "blocks",
with width and depth), dtype of its matrices, and ratio, the largest norm over
the gradients' expected one (below 1: they are clipped, into buffers of their
own; above: they stay as they are, in place).
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _project(op, B, C, O, H, W, dtype, layout, act="none", scale=False, shift=True, residual=False, save=False,
             name=None):
    c = {"op": op, "B": B, "C": C, "O": O, "H": H, "W": W, "dtype": dtype, "layout": layout, "act": act,
         "scale": scale, "shift": shift, "residual": residual, "save": save}
    return dict(c, name=name) if name else c


def _clip(net, width, depth, dtype, ratio, name=None):
    c = {"op": "clip", "net": net, "width": width, "depth": depth, "dtype": dtype, "ratio": ratio}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: one token of a ViT block through its projection, all latency
        _project("project", 1, 768, 768, 1, 1, "bf16", "nhwc", act="gelu", name="one_token"),
        # serving: eight tokens through a wide block's output projection with its residual
        _project("project", 8, 4096, 4096, 1, 1, "bf16", "nhwc", residual=True, name="eight_tokens"),
        # the expansion that closes a ResNet-50 stage 1 bottleneck after a reduction to 64 channels: folded batch
        # norm, residual, ReLU; bound by memory
        _project("project", 64, 64, 256, 56, 56, "bf16", "nchw", act="relu", scale=True, residual=True,
                 name="stage1_expand"),
        # the same at stage 4, channels-last, planes of 49 positions
        _project("project", 128, 512, 2048, 7, 7, "bf16", "nhwc", act="relu", scale=True, residual=True,
                 name="stage4_expand"),
        # a training forward over the tokens of a ViT (197 of them, odd), the pre-activation saved
        _project("project", 256, 768, 768, 197, 1, "bf16", "nhwc", act="gelu", save=True, name="vit_tokens"),
        # the largest: the tokens of a long prompt through a wide block
        _project("project", 8, 4096, 4096, 2048, 1, "bf16", "nhwc", act="silu", name="long_prompt"),
        # float32, odd channels and odd planes
        _project("project", 16, 331, 165, 27, 27, "f32", "nchw", act="relu", residual=True, name="ragged_f32"),
        # training: the gradients of a stage 3 expansion, channels-first
        _project("backward", 64, 256, 1024, 14, 14, "bf16", "nchw", act="relu", scale=True, residual=True,
                 name="stage3_backward"),
        # training: the gradients of the ViT projection
        _project("backward", 256, 768, 768, 197, 1, "bf16", "nhwc", act="gelu", name="vit_backward"),
        # the gradients of one channel-expert layer (ResNet-50 stage 3): a few small tensors, all latency
        _clip("layer", 1024, 1, "f32", 0.5, name="clip_layer"),
        # a whole ResNet-50, most of its 161 tensors small, below the largest norm: they stay as they are
        _clip("resnet", 64, 16, "f32", 4.0, name="clip_resnet50"),
        # the gradients of a transformer in bfloat16 with float32 norms and biases, clipped
        _clip("blocks", 2048, 12, "bf16", 0.25, name="clip_blocks"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["project", "project", "project", "backward", "backward", "clip"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "clip":
        net = rng.choice(["layer", "resnet", "blocks"])
        width = {"layer": _log_int(rng, 64, 2048), "resnet": rng.randint(16, 80), "blocks": _log_int(rng, 65, 1536)}[net]
        return _clip(net, width, rng.randint(1, 12), dtype, rng.choice([0.1, 0.5, 3.0]))
    # channels: round ones of real networks, and ragged ones
    C, O = _log_int(rng, 32, 4096), _log_int(rng, 32, 4096)
    if rng.random() < 0.7:
        C, O = max(32, C // 32 * 32), max(32, O // 32 * 32)
    layout = rng.choice(["nhwc", "nhwc", "nchw"])
    if layout == "nhwc" and rng.random() < 0.6:
        H, W = _log_int(rng, 1, 2048), 1     # tokens, from a single one
    else:
        H = W = rng.choice([7, 14, 28, 56, rng.randint(2, 56)])
    # the batch: from one image up, within the work and the memory of the listed cases
    top = (100 if dtype == "bf16" else 20) * 10**9 // (2 * C * O * H * W)
    top = min(top, (256 << 20) // (max(C, O) * H * W * BYTES[dtype]))
    B = _log_int(rng, 1, max(1, min(256, top)))
    act = rng.choice(["none", "relu", "gelu", "silu"])
    scale = act in ("none", "relu") and rng.random() < 0.5
    return _project(op, B, C, O, H, W, dtype, layout, act=act, scale=scale, shift=scale or rng.random() < 0.8,
                    residual=rng.random() < 0.4, save=op == "project" and rng.random() < 0.3)


def _gradients(case):
    """The gradients' shapes: (shape, whether it is a matrix) for every tensor, in the order of the network."""
    w, n = case["width"], case["depth"]
    if case["net"] == "layer":      # a channel-expert layer of w channels, w // 4 experts, k = 64 (or fewer)
        R, k = max(1, w // 4 - 1), min(64, w)
        return n * [((R, k), False), ((R, k), False), ((R,), False), ((R, w), True)]
    if case["net"] == "resnet":     # n bottlenecks of widths w, 2 w, 4 w, 8 w in the ratio 3:4:6:3 and the ends
        s = [((w, 3, 7, 7), True), ((w,), False), ((w,), False)]
        cin = w
        for i, share in enumerate((3, 4, 6, 3)):
            m = w << i
            for j in range(max(1, n * share // 16)):
                s += [((m, cin, 1, 1), True), ((m,), False), ((m,), False), ((m, m, 3, 3), True), ((m,), False),
                      ((m,), False), ((4 * m, m, 1, 1), True), ((4 * m,), False), ((4 * m,), False)]
                if j == 0:
                    s += [((4 * m, cin, 1, 1), True), ((4 * m,), False), ((4 * m,), False)]
                cin = 4 * m
        return s + [((1000, cin), True), ((1000,), False)]
    return n * [((w,), False), ((w,), False), ((w, w), True), ((w, w), True), ((w, w), True), ((w, w), True),
                ((w,), False), ((w,), False), ((4 * w, w), True), ((4 * w,), False), ((w, 4 * w), True), ((w,), False)]


def _buckets(case):
    """For each of the two gradient buckets (of the matrices' type, of float32) its shapes' sizes."""
    sizes = [(math.prod(s), m and case["dtype"] == "bf16") for s, m in _gradients(case)]
    return [n for n, low in sizes if low], [n for n, low in sizes if not low]


def _normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32) * scale


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    if case["op"] == "clip":
        low, full = _buckets(case)
        st = {"case": case}
        # views of a bucket for each type, one after the other as data-parallel buckets hold them; the matrices'
        # gradients are the larger ones
        flats = [_normal(g, sum(low), scale=1e-3).to(torch.bfloat16), _normal(g, sum(full), scale=1e-2)]
        keep = case["ratio"] > 1
        outs = flats if keep else [torch.empty_like(f) for f in flats]
        st["flats"], st["outs"] = flats, outs
        st["src"] = [t for f, n in zip(flats, (low, full)) for t in f.split(n) if n]
        st["dst"] = [t for f, n in zip(outs, (low, full)) for t in f.split(n) if n]
        st["max_norm"] = case["ratio"] * math.sqrt(sum(low) * 1e-6 + sum(full) * 1e-4)
        return st
    B, C, O, H, W = (case[n] for n in ("B", "C", "O", "H", "W"))
    dt, nchw = TYPES[case["dtype"]], case["layout"] == "nchw"
    xs, ys = ((B, C, H, W), (B, O, H, W)) if nchw else ((B, H, W, C), (B, H, W, O))
    st = {"case": case}
    x = _normal(g, *xs)
    st["x"] = (x.relu_() if case["act"] in ("none", "relu") else x).to(dt)
    del x
    st["weight"] = _normal(g, O, C, scale=C ** -0.5).to(dt)
    st["scale"] = 1.0 + _normal(g, O, scale=0.2) if case["scale"] else None
    st["shift"] = _normal(g, O, scale=0.2) if case["shift"] else None
    if case["op"] == "project":
        st["residual"] = _normal(g, *ys).relu_().to(dt) if case["residual"] else None
        st["y"] = torch.empty(ys, dtype=dt, device=DEVICE)
        st["z"] = torch.empty(ys, dtype=dt, device=DEVICE) if case["save"] else None
    else:
        st["dy"] = _normal(g, *ys).to(dt)
        st["z"] = _normal(g, *ys).to(dt) if case["act"] != "none" else None
    return st


def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _rows(t, nchw):
    """[positions, channels] in 32 bits."""
    t = t.float()
    return (t.movedim(1, -1) if nchw else t).reshape(-1, t.shape[1] if nchw else t.shape[-1])


def _laid_out(rows, like, nchw):
    """The rows [positions, channels] in the type and the order of `like`'s positions."""
    n = rows.shape[1]
    if nchw:
        B, _, H, W = like.shape
        return rows.reshape(B, H, W, n).movedim(-1, 1).to(like.dtype).contiguous()
    return rows.reshape(*like.shape[:-1], n).to(like.dtype)


def _run_project(st):
    case = st["case"]
    nchw = case["layout"] == "nchw"
    if own:
        from paper_2608_23794_amd.layer import ProjectLayer
        layer = ProjectLayer(st["weight"], st["scale"], st["shift"], act=case["act"], layout=case["layout"])
        y = layer.forward(st["x"], residual=st["residual"], y=st["y"], z=st["z"])
        return {"y": y, "z": st["z"]} if case["save"] else y
    z = torch.matmul(_rows(st["x"], nchw), st["weight"].float().t())
    if case["scale"]:
        z = z * st["scale"]
    if case["shift"]:
        z = z + st["shift"]
    if case["residual"]:
        z = z + _rows(st["residual"], nchw)
    y = _laid_out(_act(z, case["act"]), st["x"], nchw)
    return {"y": y, "z": _laid_out(z, st["x"], nchw)} if case["save"] else y


def _run_backward(st):
    case = st["case"]
    nchw = case["layout"] == "nchw"
    if own:
        from paper_2608_23794_amd.layer import ProjectLayer
        layer = ProjectLayer(st["weight"], st["scale"], st["shift"], act=case["act"], layout=case["layout"])
        return layer.backward(st["x"], st["dy"], z=st["z"], residual=case["residual"])
    x, w, dz = _rows(st["x"], nchw), st["weight"].float(), _rows(st["dy"], nchw)
    if case["act"] != "none":
        dz = dz * _act_grad(_rows(st["z"], nchw), case["act"])
    G = torch.matmul(dz.t(), x)
    out = {"dweight": G, "dx": torch.matmul(dz, w)}
    if case["scale"]:
        out["dx"] = torch.matmul(dz * st["scale"], w)
        out["dweight"] = st["scale"].unsqueeze(1) * G
        out["dscale"] = (w * G).sum(1)
    if case["shift"]:
        out["dshift"] = dz.sum(0)
    if case["residual"]:
        out["dresidual"] = _laid_out(dz, st["dy"], nchw)
    out["dx"], out["dweight"] = _laid_out(out["dx"], st["x"], nchw), out["dweight"].to(st["weight"].dtype)
    return out


def _run_clip(st):
    if own:
        from paper_2608_23794_amd.layer import clip_gradients
        norm = clip_gradients(st["src"], st["max_norm"], out=st["dst"])
        return {"norm": norm, "clipped": st["outs"]}
    norm = torch.stack([t.double().square().sum() for t in st["src"]]).sum().sqrt().float().reshape(1)
    coef = (st["max_norm"] / norm).clamp(max=1.0)
    [d.copy_(t.float() * coef) for t, d in zip(st["src"], st["dst"])]
    return {"norm": norm, "clipped": st["outs"]}


def run(st):
    return {"project": _run_project, "backward": _run_backward, "clip": _run_clip}[st["case"]["op"]](st)


def work(case):
    if case["op"] == "clip":
        low, full = (sum(n) for n in _buckets(case))
        b = 2 * low + 4 * full
        return {"bytes": b if case["ratio"] > 1 else 2 * b, "flops": 3 * (low + full)}
    M, C, O, el = case["B"] * case["H"] * case["W"], case["C"], case["O"], BYTES[case["dtype"]]
    x, y, w, v = M * C * el, M * O * el, O * C * el, 4 * O * (case["scale"] + case["shift"])
    if case["op"] == "project":
        return {"bytes": x + w + v + y * (1 + case["residual"] + case["save"]), "flops": 2 * M * C * O}
    saved = y if case["act"] != "none" else 0
    return {"bytes": 2 * x + 2 * w + 2 * v + y + saved + y * case["residual"], "flops": 4 * M * C * O}


def _exact_act(z, kind):
    """act(z) and its derivative in 64 bits."""
    if kind == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))
    if kind == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.special.expit(z)
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "clip":
        d = [f.double() for f in st["flats"]]
        norm = torch.sqrt(sum((f * f).sum() for f in d))
        coef = min(1.0, st["max_norm"] / float(norm))
        return {"norm": norm.reshape(1), "clipped": [f.mul_(coef) for f in d]}
    nchw, kind, w = case["layout"] == "nchw", case["act"], st["weight"].double()
    per = [1, -1, 1] if nchw else [1, 1, -1]
    B, C, O = case["B"], case["C"], case["O"]
    y_shape = (B, O, case["H"], case["W"]) if nchw else (B, case["H"], case["W"], O)
    scale = st["scale"].double() if case["scale"] else torch.ones(O, dtype=torch.float64, device=DEVICE)
    parts, dW, dshift = [], 0.0, 0.0
    step = max(1, (1 << 27) // (max(C, O) * case["H"] * case["W"]))
    for b in range(0, B, step):          # images at a time, for the memory of the 64-bit values
        def take(t, n):                  # [b, channels, positions] or [b, positions, channels]
            t = t[b:b + step].double()
            return t.reshape(t.shape[0], n, -1) if nchw else t.reshape(t.shape[0], -1, n)

        x = take(st["x"], C)
        if case["op"] == "project":
            z = torch.matmul(w, x) if nchw else torch.matmul(x, w.t().contiguous())
            z = z * scale.reshape(per)
            if case["shift"]:
                z = z + st["shift"].double().reshape(per)
            if case["residual"]:
                z = z + take(st["residual"], O)
            parts.append((_exact_act(z, kind)[0], z))
        else:
            dz = take(st["dy"], O)
            if kind != "none":
                dz = dz * _exact_act(take(st["z"], O), kind)[1]
            g = dz * scale.reshape(per)
            if nchw:
                dx = torch.matmul(w.t().contiguous(), g)
                dW = dW + torch.matmul(dz, x.transpose(1, 2).contiguous()).sum(0)
            else:
                dx = torch.matmul(g, w)
                dW = dW + torch.matmul(dz.transpose(1, 2).contiguous(), x).sum(0)
            dshift = dshift + dz.sum((0, 2) if nchw else (0, 1))
            parts.append((dx, dz))
    first, second = (torch.cat([p[i] for p in parts]) for i in (0, 1))
    if case["op"] == "project":
        return {"y": first.reshape(y_shape), "z": second.reshape(y_shape)} if case["save"] else first.reshape(y_shape)
    out = {"dx": first.reshape(st["x"].shape), "dweight": dW * scale.unsqueeze(1)}
    if case["scale"]:
        out["dscale"] = (w * dW).sum(1)
    if case["shift"]:
        out["dshift"] = dshift
    if case["residual"]:
        out["dresidual"] = second.reshape(y_shape)
    return out
