"""Performance cases of the matrix-product operators beside the convolutions:

  orth        orthogonalising matrices by Newton-Schulz products, the result
              rounded to binary16 (products of 22-bit operands);
  muon        one update of a set of binary16 weight matrices by orthogonalised
              momentum (binary16 weights, gradients and momentum, in place);
  int8_fwd    a dense layer's forward in 8-bit integers with a scale for each
              token and each output channel, the weights quantised beforehand;
  int8_train  a dense layer's whole training pass in 8-bit integers: weights
              quantised, forward, and the gradients of input, weights and bias.

Each is defined by the plain form below, in elementary operations.  With `own`
set, run() makes this library's calls instead.
"""

from __future__ import annotations

import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)  # the quintic X <- aX + (bA + cA^2)X, A = X X^T
STEPS = 5

# the convolution filters and the classifier of ResNet-50 as matrices
# [filters][taps * channels], count x rows x cols
RESNET50 = ("1x64x147,1x64x64,2x64x256,3x64x576,4x256x64,1x128x256,3x128x512,4x128x1152,4x512x128,"
            "1x512x256,1x256x512,5x256x1024,6x256x2304,6x1024x256,1x1024x512,1x512x1024,2x512x2048,"
            "3x512x4608,3x2048x512,1x2048x1024,1x1000x2048")
MOST_ELEMS = 4096 * 4096                 # of a matrix set
MOST_FLOPS = 5 * 4 * 4096 ** 3           # of its products (muon_4096)
MOST_MACS = 8192 * 4096 * 4096           # of one product of a dense layer


def listed():
    return [
        # one 3x3 filter of the narrowest stage: launches and latency count
        dict(name="orth_64x576", kind="orth", shapes="1x64x576"),
        # the classifier of ResNet-50, rows no multiple of a tile
        dict(name="orth_1000x2048", kind="orth", shapes="1x1000x2048"),
        # square projections of one width, orthogonalised together
        dict(name="orth_4x1024", kind="orth", shapes="4x1024x1024"),
        # every weight matrix of ResNet-50 in one update
        dict(name="muon_resnet50", kind="muon", shapes=RESNET50),
        # a wide, a tall and an odd matrix of a network with other widths
        dict(name="muon_ragged", kind="muon", shapes="1x333x1111,1x2049x517,2x77x90"),
        # the largest square matrix
        dict(name="muon_4096", kind="muon", shapes="1x4096x4096"),
        # one token at a time through a wide layer: the weights are read once
        dict(name="fwd_1_4096", kind="int8_fwd", tokens=1, inputs=4096, outputs=4096, bias=False),
        # a few tokens through ResNet-50's classifier
        dict(name="fwd_13_classifier", kind="int8_fwd", tokens=13, inputs=2048, outputs=1000,
             bias=True),
        # many tokens through a wide layer
        dict(name="fwd_8192_4096", kind="int8_fwd", tokens=8192, inputs=4096, outputs=4096,
             bias=False),
        # ResNet-50's classifier at the benchmark's batch
        dict(name="train_128_classifier", kind="int8_train", tokens=128, inputs=2048,
             outputs=1000, bias=True),
        # sizes that end inside every tile and are no multiple of a vector
        dict(name="train_ragged", kind="int8_train", tokens=1111, inputs=1337, outputs=2501,
             bias=True),
        # a wide layer's training pass
        dict(name="train_4096", kind="int8_train", tokens=4096, inputs=4096, outputs=4096,
             bias=True),
    ]


# ---- drawn cases: the same kinds over their ranges -----------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """As it falls, or a multiple of 8, or of 64."""
    v, t = _log(rng, lo, hi), rng.random()
    step = 1 if t < 0.4 else 8 if t < 0.7 else 64
    return max(lo, min(hi, (v + step // 2) // step * step))


def _shapes(text):
    return [tuple(int(v) for v in s.split("x")) for s in text.split(",")]


def _products(shapes):
    """Multiplications and additions of the Newton-Schulz products: X X^T and A^2
    are symmetric, so half of each is enough."""
    f = 0
    for count, rows, cols in shapes:
        m, n = min(rows, cols), max(rows, cols)
        f += count * STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
    return f


def draw(rng):
    t = rng.random()
    if t < 0.5:
        kind = "orth" if t < 0.25 else "muon"
        shapes = []
        for _ in range(rng.choice((1, 1, 1, 2, 3))):
            shapes.append([rng.choice((1, 1, 1, 2, 5)), _size(rng, 4, 4096), _size(rng, 4, 4096)])
        for s in shapes:  # no larger than the largest listed one
            while _products(shapes) > MOST_FLOPS or sum(a * b * c for a, b, c in shapes) > MOST_ELEMS:
                s[0] = max(1, s[0] // 2)
                i = 1 if s[1] >= s[2] else 2
                if s[i] <= 64:
                    break
                s[i] = s[i] * 2 // 3
        return dict(kind=kind, shapes=",".join("x".join(map(str, s)) for s in shapes))
    c = dict(kind="int8_fwd" if t < 0.75 else "int8_train", tokens=_log(rng, 1, 8192),
             inputs=_size(rng, 16, 8192), outputs=_size(rng, 16, 8192), bias=rng.random() < 0.5)
    most = MOST_MACS if c["kind"] == "int8_fwd" else MOST_MACS // 2
    while c["tokens"] * c["inputs"] * c["outputs"] > most:
        c["tokens"] = c["tokens"] * 3 // 4
    return c


# ---- inputs ----------------------------------------------------------------------

def _gradient(g, count, rows, cols):
    """A weight gradient as training gives it: a few strong directions over noise,
    of a size at which no loss scaling keeps it from small values."""
    r = max(1, min(rows, cols) // 16)
    dev = dict(device="cuda", generator=g)
    u, v = torch.randn((count, rows, r), **dev), torch.randn((count, r, cols), **dev)
    s = torch.logspace(0, -1, r, device="cuda")
    x = (u * s) @ v / math.sqrt(r) + 0.1 * torch.randn((count, rows, cols), **dev)
    return (1e-3 * x).half()


def _tokens(g, rows, cols):
    """Activations: each token of a size of its own, a few channels far larger."""
    dev = dict(device="cuda", generator=g)
    x = torch.randn((rows, cols), **dev) * torch.exp(0.5 * torch.randn((rows, 1), **dev))
    return (x * torch.where(torch.rand(cols, **dev) < 0.01, 8.0, 1.0)).half()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dev = dict(device="cuda", generator=g)
    kind = case["kind"]
    if kind in ("orth", "muon"):
        shapes = _shapes(case["shapes"])
        st = {"kind": kind, "g": [_gradient(g, *s) for s in shapes]}
        if kind == "orth":
            st["y"] = [torch.empty_like(t) for t in st["g"]]
        else:
            st["m"] = [_gradient(g, *s) for s in shapes]
            st["w"] = [(torch.randn(s, **dev) * math.sqrt(2.0 / s[2])).half() for s in shapes]
            st["scale"] = [math.sqrt(max(1.0, s[1] / s[2])) for s in shapes]
            st.update(lr=0.02, momentum=0.95, weight_decay=0.01)
        return st
    t, i, o = case["tokens"], case["inputs"], case["outputs"]
    st = {"kind": kind, "x": _tokens(g, t, i), "sizes": (t, i, o),
          "bias": (0.1 * torch.randn(o, **dev)).half() if case["bias"] else None}
    w = (torch.randn((o, i), **dev) / math.sqrt(i)).half()
    st["y"] = torch.empty((t, o), dtype=torch.float16, device="cuda")
    if kind == "int8_fwd":
        # the weights of a program that serves: quantised once, each row padded
        # with zeros to whole 16 bytes
        q, s = _quantised(w.float())
        st["wq"] = torch.zeros((o, -(-i // 16) * 16), dtype=torch.int8, device="cuda")
        st["wq"][:, :i] = q.to(torch.int8)
        st["sw"] = s.reshape(-1).contiguous()
    else:
        st["w"] = w
        st["dy"] = _tokens(g, t, o) * 1e-2
        st["dx"], st["dw"] = torch.empty_like(st["x"]), torch.empty_like(w)
        st["dbias"] = torch.empty(o, dtype=torch.float16, device="cuda") if case["bias"] else None
    return st


# ---- the plain forms ---------------------------------------------------------------

def _newton_schulz(u):
    """Matrices [count][rows][cols] in float32: each over its Frobenius norm (0
    stays 0), then STEPS times X <- aX + (bA + cA^2)X with A = X X^T taken over
    the shorter side."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = x * torch.where(norm > 0, 1.0 / norm, norm).float()
    a, b, c = COEF
    for _ in range(STEPS):
        p = x @ x.transpose(1, 2)
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.transpose(1, 2) if tall else x


def _muon(st):
    mu, keep = st["momentum"], 1.0 - st["lr"] * st["weight_decay"]
    for w, g, m, scale in zip(st["w"], st["g"], st["m"], st["scale"]):
        m.copy_((mu * m.float() + g.float()).half())
        o = _newton_schulz(mu * m.float() + g.float())
        w.copy_((keep * w.float() - st["lr"] * scale * o).half())
    return st["w"] + st["m"]


def _quantised(x):
    """Whole numbers and a scale for each row of x: s = max |x| / 127 and
    q = 127 x / max |x| to the nearest, ties to even (0 where the row is 0).  127 x
    of a binary16 x is exact, so the quotient is halfway where the numbers are."""
    top = x.abs().amax(1, keepdim=True)
    return torch.where(top > 0, torch.round(127.0 * x / top), 0.0), top / 127.0


def _product(a, b):
    (qa, sa), (qb, sb) = a, b
    return (qa @ qb.t()) * (sa * sb.t())


def _int8_fwd(st, wq, sw):
    y = _product(_quantised(st["x"].float()), (wq, sw))
    return (y if st["bias"] is None else y + st["bias"].float()).half()


def _int8_train(st):
    w, x, dy = st["w"].float(), st["x"].float(), st["dy"].float()
    y = _int8_fwd(st, *_quantised(w))
    dx = _product(_quantised(dy), _quantised(w.t().contiguous())).half()
    dw = _product(_quantised(dy.t().contiguous()), _quantised(x.t().contiguous())).half()
    return [y, dx, dw] + ([] if st["bias"] is None else [dy.sum(0).half()])


# ---- this library's calls ------------------------------------------------------------

def _own_matrices(st):
    import paper_1911_07384_amd as F
    if "ws" not in st:  # what a program keeps beside its weights
        scale = st.get("scale", [1.0] * len(st["g"]))
        st["descs"] = F.muon_descs([(t.shape[1], t.shape[2], s) for t, s in zip(st["g"], scale)
                                    for _ in range(t.shape[0])])
        for k in ("g", "y", "w", "m"):
            st["each_" + k] = [v for t in st.get(k, []) for v in t]
        products = 3 if st["kind"] == "orth" else 1
        st["ws"] = F.workspace(F.fp16_muon_workspace_bytes(st["descs"], products))
    if st["kind"] == "orth":
        F.fp16_orthogonalize(st["descs"], st["each_g"], st["each_y"], steps=STEPS, coef=COEF,
                             products=3, ws=st["ws"])
        return st["y"]
    F.fp16_muon_step(st["descs"], st["each_w"], st["each_g"], st["each_m"], st["lr"],
                     st["momentum"], st["weight_decay"], nesterov=True, steps=STEPS, coef=COEF,
                     products=1, ws=st["ws"])
    return st["w"] + st["m"]


def _own_dense(st):
    import paper_1911_07384_amd as F
    t, i, o = st["sizes"]
    if "ws" not in st:
        st["desc"] = d = F.int8_dense_desc(t, i, o)
        st["ws"] = F.workspace(F.fp16_int8_dense_workspace_bytes(d))
        if st["kind"] == "int8_train":
            st["wq"], st["sw"] = F.int8_operand(o, i)
            st["wqt"], st["swt"] = F.int8_operand(i, o)
    d = st["desc"]
    if st["kind"] == "int8_fwd":
        F.fp16_int8_dense_fwd(d, st["x"], st["wq"], st["sw"], st["bias"], st["y"], st["ws"])
        return st["y"]
    F.fp16_int8_dense_weights(d, st["w"], st["wq"], st["sw"], st["wqt"], st["swt"], st["ws"])
    F.fp16_int8_dense_fwd(d, st["x"], st["wq"], st["sw"], st["bias"], st["y"], st["ws"])
    F.fp16_int8_dense_bwd(d, st["x"], st["dy"], st["wqt"], st["swt"], st["dx"], st["dw"],
                          st["dbias"], st["ws"])
    return [st["y"], st["dx"], st["dw"]] + ([] if st["bias"] is None else [st["dbias"]])


def run(state):
    kind = state["kind"]
    if own:
        return _own_matrices(state) if kind in ("orth", "muon") else _own_dense(state)
    if kind == "orth":
        return [_newton_schulz(t.float()).half() for t in state["g"]]
    if kind == "muon":
        return _muon(state)
    if kind == "int8_fwd":
        i = state["sizes"][1]
        return _int8_fwd(state, state["wq"][:, :i].float(), state["sw"][:, None])
    return _int8_train(state)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("orth", "muon"):
        shapes = _shapes(case["shapes"])
        elems = sum(a * b * c for a, b, c in shapes)
        return {"bytes": elems * (4 if kind == "orth" else 10), "flops": _products(shapes)}
    t, i, o = case["tokens"], case["inputs"], case["outputs"]
    bias = 2 * o if case["bias"] else 0
    if kind == "int8_fwd":
        return {"bytes": 2 * t * i + o * i + 4 * o + 2 * t * o + bias, "flops": 2 * t * i * o}
    return {"bytes": 2 * (2 * t * i + 2 * t * o + 2 * o * i) + 2 * bias, "flops": 6 * t * i * o}


# ---- the definitions in 64 bits ------------------------------------------------------

def _orthogonal64(u):
    a, b, c = COEF
    x = u / u.square().sum().sqrt()
    if x.shape[0] > x.shape[1]:
        x = x.mT
    eye = torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
    for _ in range(STEPS):
        p = x.matmul(x.mT)
        x = (a * eye + b * p + c * p.matmul(p)).matmul(x)
    return x if u.shape[0] <= u.shape[1] else x.mT


def _whole64(x, dim):
    top = x.abs().amax(dim, keepdim=True)
    return torch.nan_to_num(torch.round(x * 127 / top)) * (top / 127)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "orth":
        return [torch.stack([_orthogonal64(v.double()) for v in t]) for t in st["g"]]
    if kind == "muon":
        mu, ws, ms = st["momentum"], [], []
        for w, g, m, scale in zip(st["w"], st["g"], st["m"], st["scale"]):
            new = mu * m.double() + g.double()
            kept = new.half().double()  # what the momentum buffer holds from now on
            o = torch.stack([_orthogonal64(v) for v in g.double() + mu * kept])
            ws.append((1 - st["lr"] * st["weight_decay"]) * w.double() - st["lr"] * scale * o)
            ms.append(new)
        return ws + ms
    x = st["x"].double()
    bias = 0.0 if st["bias"] is None else st["bias"].double()
    if kind == "int8_fwd":
        w = st["wq"][:, :case["inputs"]].double() * st["sw"].double()[:, None]
        return _whole64(x, 1) @ w.mT + bias
    w, dy = st["w"].double(), st["dy"].double()
    out = [_whole64(x, 1) @ _whole64(w, 1).mT + bias, _whole64(dy, 1) @ _whole64(w, 0),
           _whole64(dy, 0).mT @ _whole64(x, 0)]
    return out if st["bias"] is None else out + [dy.sum(0)]
