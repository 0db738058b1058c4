"""The operators on weight matrices that a training or serving program calls, to be timed and compared.

Four operators: the orthogonalisation of matrices by Newton-Schulz products
("ortho"), the optimiser step around it ("muon"), the quantisation of rows to
8-bit integers ("quantize") and the product of such rows with an 8-bit weight
matrix ("linear").  With `own` false, run() computes them in elementary torch
operations in 32 bits; with `own` true it makes the library's calls.
"""
import math

import torch

own = False

A, B, C = 3.4445, -4.7750, 2.0315  # the quintic X <- aX + (bS + cSS)X, S = XX^T
STEPS = 5

# ResNet-50's 53 convolution filters, [K][R*S*C], in forward order: width, blocks, input channels of each stage
STAGES = ((64, 3, 64), (128, 4, 256), (256, 6, 512), (512, 3, 1024))


def _resnet50():
    out = [(64, 147)]
    for width, blocks, cin in STAGES:
        for b in range(blocks):
            c = cin if b == 0 else 4 * width
            out += [(width, c), (width, 9 * width), (4 * width, width)] + ([(4 * width, c)] if b == 0 else [])
    return _text(out)


def _text(shapes):
    return " ".join("%dx%d" % s for s in shapes)


def _shapes(case):
    """The (rows, cols) of a case's matrices."""
    return [tuple(map(int, s.split("x"))) for s in case["shapes"].split()]


def listed():
    return [
        # one 1x1 filter of the first stage: nothing but latency
        {"name": "ortho_64x64", "op": "ortho", "shapes": "64x64"},
        # the classifier's weight, whose rows are no multiple of a tile
        {"name": "ortho_1000x2048", "op": "ortho", "shapes": "1000x2048"},
        # one large square matrix, bound by the products
        {"name": "ortho_4096x4096", "op": "ortho", "shapes": "4096x4096"},
        # the stem's filter, alone: an odd row length, and latency
        {"name": "muon_64x147", "op": "muon", "shapes": "64x147", "nesterov": True},
        # the last stage's three 3x3 filters
        {"name": "muon_3x_512x4608", "op": "muon", "shapes": "512x4608 512x4608 512x4608", "nesterov": False},
        # every convolution filter of a ResNet-50 in one call: the whole step's update
        {"name": "muon_resnet50", "op": "muon", "shapes": _resnet50(), "nesterov": True},
        # a batch's pooled features, before the classifier
        {"name": "quantize_256x2048", "op": "quantize", "m": 256, "k": 2048},
        # a batch's activations at 56x56, 256 channels, each pixel a row
        {"name": "quantize_802816x256", "op": "quantize", "m": 802816, "k": 256},
        # the classifier for a single image
        {"name": "linear_1x2048x1000", "op": "linear", "m": 1, "k": 2048, "n": 1000, "bias": True},
        # a few rows against a large weight, bound by the weight's bytes
        {"name": "linear_16x8192x8192", "op": "linear", "m": 16, "k": 8192, "n": 8192, "bias": False},
        # a 1x1 convolution at 14x14, batch 256: many rows, few channels
        {"name": "linear_50176x1024x256", "op": "linear", "m": 50176, "k": 1024, "n": 256, "bias": True},
        # a large layer, bound by the products
        {"name": "linear_8192x4096x8192", "op": "linear", "m": 8192, "k": 4096, "n": 8192, "bias": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("ortho", "muon", "quantize", "linear"))
    if op == "ortho":
        return {"op": op, "shapes": _text([(_log(rng, 1, 2048), _log(rng, 1, 2048)) for _ in range(rng.randint(1, 8))])}
    if op == "muon":
        shapes = []
        for _ in range(rng.randint(1, 6)):
            shapes += [(_log(rng, 16, 1024), _log(rng, 9, 4608))] * rng.randint(1, 3)
        return {"op": op, "shapes": _text(shapes), "nesterov": rng.random() < 0.5}
    if op == "quantize":
        k = _log(rng, 1, 16384)
        return {"op": op, "m": _log(rng, 1, min(800000, 200_000_000 // k)), "k": k}
    k, n = _log(rng, 16, 8192), _log(rng, 8, 8192)
    if rng.random() < 0.6:  # most layers' sizes are multiples of 64
        k, n = (k + 63) // 64 * 64, (n + 63) // 64 * 64
    return {"op": op, "m": _log(rng, 1, 60000 if k * n < 1 << 22 else 4096), "k": k, "n": n, "bias": rng.random() < 0.5}


def _gradient(gen, rows, cols):
    """A filter's gradient: a few strong directions over noise, at a gradient's size."""
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    r = max(1, min(rows, cols) // 16)
    return ((n(rows, r) @ n(r, cols) / math.sqrt(r) + n(rows, cols)) * 1e-2).half()


def _arena(parts):
    """A flat arena, as programs keep their parameters, and the matrices in it, each from a multiple of 8 elements on."""
    starts, size = [], 0
    for p in parts:
        starts.append(size)
        size += (p.numel() + 7) // 8 * 8
    flat = torch.zeros(size, dtype=parts[0].dtype, device=parts[0].device)
    views = [flat[at:at + p.numel()].view(p.shape) for at, p in zip(starts, parts)]
    for view, p in zip(views, parts):
        view.copy_(p)
    return flat, views


def _rows(x):
    """8-bit rows and their scales of what a layer before has left."""
    top = x.abs().amax(1, keepdim=True).float()
    return torch.round(x.float() * 127 / top).to(torch.int8), (top / 127).flatten()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    s = dict(case)
    if case["op"] == "ortho":
        s["g"] = [_gradient(gen, r, c) for r, c in _shapes(case)]
    elif case["op"] == "muon":
        s["flat_g"], s["g"] = _arena([_gradient(gen, r, c) for r, c in _shapes(case)])
        s["flat_v"], s["v"] = _arena([(_gradient(gen, r, c).float() * 3).half() for r, c in _shapes(case)])
        s["flat_w"], s["w"] = _arena([(n(r, c) * math.sqrt(2 / c)).half() for r, c in _shapes(case)])
        s["lr"], s["momentum"], s["decay"] = 0.02, 0.95, 0.01
        s["scale"] = [math.sqrt(max(1.0, r / c)) for r, c in _shapes(case)]
    elif case["op"] == "quantize":
        s["x"] = torch.randn(case["m"], case["k"], generator=gen, device="cuda", dtype=torch.float16).relu_().mul_(1.5)
        s["x"] += 0.01  # (activations behind a ReLU, moved off zero by a bias)
    else:
        s["xq"], s["xs"] = _rows(n(case["m"], case["k"]).half())
        s["wq"], s["ws"] = _rows((n(case["n"], case["k"]) * math.sqrt(2 / case["k"])).half())
        s["bias"] = (n(case["n"]) * 0.1).half() if case["bias"] else None
    return s


def _step(x):
    a = x @ x.T
    return A * x + (B * a + C * (a @ a)) @ x


def _polar(u):
    x = u.T if u.shape[0] > u.shape[1] else u
    size = torch.linalg.vector_norm(x)
    x = x / torch.where(size == 0, 1.0, size)
    for _ in range(STEPS):
        x = _step(x)
    return x.T if u.shape[0] > u.shape[1] else x


def _plain(s):
    if s["op"] == "ortho":
        return [_polar(g.float()).half().contiguous() for g in s["g"]]
    if s["op"] == "muon":
        for w, v, g, scale in zip(s["w"], s["v"], s["g"], s["scale"]):
            v.copy_(s["momentum"] * v.float() + g.float())
            u = g.float() + s["momentum"] * v.float() if s["nesterov"] else v.float()
            w.copy_(w.float() - s["lr"] * (scale * _polar(u) + s["decay"] * w.float()))
        return [s["flat_w"], s["flat_v"]]
    if s["op"] == "quantize":
        x = s["x"].float()
        top = x.abs().amax(1, keepdim=True)
        q = torch.round(x * 127 / torch.where(top == 0, 1.0, top))
        return [q.to(torch.int8), (top / 127).flatten()]
    y = (s["xq"].float() @ s["wq"].float().T) * (s["xs"][:, None] * s["ws"][None, :])
    return [(y + s["bias"].float() if s["bias"] is not None else y).half()]


def _own(s):
    from paper_1911_07384_gb300 import pf16

    if s["op"] == "ortho":
        if "plan" not in s:  # the list and the workspace, which a program keeps
            s["o"] = [torch.empty_like(g) for g in s["g"]]
            s["plan"] = pf16.ortho_list(zip(s["g"], s["o"], *zip(*_shapes(s))))
            s["space"] = torch.empty(pf16.ortho_workspace_size(s["plan"]), dtype=torch.uint8, device="cuda")
        pf16.orthogonalize(s["plan"], s["space"])
        return s["o"]
    if s["op"] == "muon":
        if "plan" not in s:
            s["plan"] = pf16.muon_list(zip(s["w"], s["v"], s["g"], *zip(*_shapes(s)), s["scale"]))
            s["space"] = torch.empty(pf16.muon_workspace_size(s["plan"]), dtype=torch.uint8, device="cuda")
        pf16.muon_update(s["plan"], s["lr"], s["momentum"], s["decay"], s["space"],
                         flags=pf16.PF16_MUON_NESTEROV if s["nesterov"] else 0)
        return [s["flat_w"], s["flat_v"]]
    m, k = s["m"], s["k"]
    if s["op"] == "quantize":
        if "q" not in s:
            s["q"] = torch.empty(m, k, dtype=torch.int8, device="cuda")
            s["qs"] = torch.empty(m, dtype=torch.float32, device="cuda")
        pf16.quantize_i8(s["x"], s["q"], s["qs"], m, k)
        return [s["q"], s["qs"]]
    if "y" not in s:
        s["y"] = torch.empty(m, s["n"], dtype=torch.float16, device="cuda")
    pf16.linear_i8(s["xq"], s["xs"], s["wq"], s["ws"], s["bias"], s["y"], m, s["n"], k)
    return [s["y"]]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    if case["op"] in ("ortho", "muon"):
        size = sum(r * c for r, c in _shapes(case))
        # XX^T and SS are symmetric: half of their products; then (bS + cSS)X
        flops = sum(STEPS * (3 * min(r, c) ** 2 * max(r, c) + min(r, c) ** 3) for r, c in _shapes(case))
        return {"bytes": size * (4 if case["op"] == "ortho" else 10), "flops": flops}
    m, k = case["m"], case["k"]
    if case["op"] == "quantize":
        return {"bytes": 3 * m * k + 4 * m, "flops": 3 * m * k}
    n = case["n"]
    return {"bytes": m * k + n * k + 2 * m * n + 4 * (m + n) + (2 * n if case["bias"] else 0), "flops": 2 * m * n * k}


def _orthogonal64(u):
    """The definition, from the left for wide matrices and from the right for tall ones."""
    size = u.square().sum().sqrt()
    x = u / size if size > 0 else u
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            s = torch.mm(x, x.t())
            x = torch.mm(A * torch.eye(len(s), dtype=x.dtype, device=x.device) + B * s + C * torch.mm(s, s), x)
        else:
            s = torch.mm(x.t(), x)
            x = torch.mm(x, A * torch.eye(len(s), dtype=x.dtype, device=x.device) + B * s + C * torch.mm(s, s))
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ortho":
        return [_orthogonal64(g.double()) for g in s["g"]]
    if case["op"] == "muon":
        ws, vs = [], []
        for w, v, g, scale in zip(s["w"], s["v"], s["g"], s["scale"]):
            g, w = g.double(), w.double()
            new = torch.add(g, v.double(), alpha=s["momentum"])
            kept = new.half().double()  # (the update is taken of the momentum as it is stored)
            o = _orthogonal64(g + s["momentum"] * kept if case["nesterov"] else kept)
            ws.append((1 - s["lr"] * s["decay"]) * w - s["lr"] * scale * o)
            vs.append(new)
        return [_arena(ws)[0], _arena(vs)[0]]
    if case["op"] == "quantize":
        # row blocks: the 64-bit copies of the largest case are large
        q, scale = [], []
        for x in s["x"].split(max(1, (1 << 26) // case["k"])):
            top = x.double().abs().max(dim=1).values
            q.append(torch.round(127.0 * x.double() / torch.where(top > 0, top, torch.ones_like(top))[:, None]).to(torch.int8))
            scale.append(top / 127.0)
        return [torch.cat(q), torch.cat(scale)]
    y = torch.mm(s["xq"].double(), s["wq"].double().t())
    y *= s["xs"].double()[:, None]
    y *= s["ws"].double()[None, :]
    return [y + s["bias"].double() if s["bias"] is not None else y]
