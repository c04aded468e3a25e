"""Performance cases of the operators of a network's dense head and of what is read
from its logits:

  dense_fwd      a dense layer whose bias, activation, dropout and residual join
                 the product before its only rounding;
  dense_train    that layer's forward, which keeps the values before the activation,
                 and its backward from such values of an earlier forward;
  dropout        dropout from a counter-based generator, its mask never stored, with
                 an optional residual; forward and backward;
  logprob        log probabilities of given classes with each row's entropy and its
                 most probable classes;
  logprob_train  log probabilities and entropies, and the logits' gradient from the
                 gradients of both.

Each is defined by the plain form below, in elementary operations.  With `own`
set, run() makes this library's calls instead.

Dropout of an element: element i takes 16-bit word i % 8 of the Philox4x32-10 block
(Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) of
counter (i / 8, site, step low, step high) and key (seed low, seed high), and is kept
where the word is at least round(65536 p).
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

MOST_MACS = 8192 * 4096 * 4096   # of a layer's forward (fwd_8192_4096); half in training
MOST_DROP = 8192 * 16384         # elements of a dropout
MOST_LOGITS = 4096 * 50048


def listed():
    return [
        # one image through ResNet-50's classifier: launches and latency count
        dict(name="fwd_1_classifier", kind="dense_fwd", tokens=1, inputs=2048, outputs=1000,
             act="none", bias=True, residual=False),
        # one token at a time through the first layer of a wide block: the weights are
        # read once
        dict(name="fwd_1_wide", kind="dense_fwd", tokens=1, inputs=4096, outputs=16384,
             act="gelu", bias=True, residual=False),
        # a few sequences' tokens through the block's second layer
        dict(name="fwd_24_wide", kind="dense_fwd", tokens=24, inputs=16384, outputs=4096,
             act="none", bias=True, residual=True),
        # sizes that end inside every tile and are no multiple of a vector
        dict(name="fwd_ragged", kind="dense_fwd", tokens=1111, inputs=1337, outputs=2501,
             act="silu", bias=True, residual=True),
        # many tokens through a wide layer
        dict(name="fwd_8192_4096", kind="dense_fwd", tokens=8192, inputs=4096, outputs=4096,
             act="gelu", bias=True, residual=False),
        # ResNet-50's classifier in training at the benchmark's batch
        dict(name="train_128_classifier", kind="dense_train", tokens=128, inputs=2048,
             outputs=1000, act="none", bias=True, residual=False, p=0.0),
        # a wide layer's training pass with everything the epilogue takes
        dict(name="train_4096", kind="dense_train", tokens=4096, inputs=4096, outputs=4096,
             act="gelu", bias=True, residual=True, p=0.1),
        # the features before the classifier at the benchmark's batch
        dict(name="dropout_features", kind="dropout", n=128 * 2048, p=0.2, residual=False),
        # activations of a wide layer joining the residual stream
        dict(name="dropout_wide", kind="dropout", n=8192 * 16384, p=0.1, residual=True),
        # validation of the benchmark's batch: top-1 and top-5 of 1000 classes
        dict(name="logprob_128_1000", kind="logprob", rows=128, classes=1000, stride=1000,
             top=5, scale=1.0),
        # one sequence's next token over a large vocabulary, with its alternatives
        dict(name="logprob_1_131071", kind="logprob", rows=1, classes=131071, stride=131072,
             top=20, scale=1.25),
        # a batch of sequences in training, rows padded past an odd vocabulary
        dict(name="logprob_train_4096", kind="logprob_train", rows=4096, classes=50001,
             stride=50048, top=0, scale=1.0),
    ]


# ---- drawn cases: the same kinds over their ranges -----------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """As it falls, or a multiple of 8, or of 64."""
    v, t = _log(rng, lo, hi), rng.random()
    step = 1 if t < 0.35 else 8 if t < 0.65 else 64
    return max(lo, min(hi, (v + step // 2) // step * step))


def draw(rng):
    t = rng.random()
    if t < 0.55:
        c = dict(kind="dense_fwd" if t < 0.3 else "dense_train", tokens=_log(rng, 1, 8192),
                 inputs=_size(rng, 16, 16384), outputs=_size(rng, 16, 16384),
                 act=rng.choice(("none", "relu", "gelu", "silu")), bias=rng.random() < 0.7,
                 residual=rng.random() < 0.5)
        most = MOST_MACS
        if c["kind"] == "dense_train":
            c["p"] = rng.choice((0.0, 0.0, 0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)))
            most //= 2
        while c["tokens"] * c["inputs"] * c["outputs"] > most:
            c["tokens"] = c["tokens"] * 3 // 4
        return c
    if t < 0.7:
        n = _log(rng, 64, MOST_DROP)
        return dict(kind="dropout", n=n if rng.random() < 0.5 else max(8, n // 8 * 8),
                    p=rng.choice((0.1, 0.2, 0.5, round(rng.uniform(0.01, 0.95), 3))),
                    residual=rng.random() < 0.5)
    kind = "logprob" if t < 0.85 else "logprob_train"
    classes = _size(rng, 16, 262144)
    c = dict(kind=kind, rows=_log(rng, 1, 8192), classes=classes,
             stride=classes + rng.choice((0, 0, rng.randrange(1, 70))),
             top=rng.choice((0, 1, 5, 8)) if kind == "logprob" else 0,
             scale=rng.choice((1.0, 1.0, round(rng.uniform(0.5, 2.0), 3))))
    if kind == "logprob" and classes > 1000:
        c["top"] = rng.choice((1, 5, 20, 64))
    while c["rows"] * c["stride"] > MOST_LOGITS:
        c["rows"] = c["rows"] * 3 // 4
    return c


# ---- inputs ----------------------------------------------------------------------

def _tokens(g, rows, cols):
    """Activations: each token of a size of its own, a few channels far larger."""
    dev = dict(device="cuda", generator=g)
    x = torch.randn((rows, cols), **dev) * torch.exp(0.5 * torch.randn((rows, 1), **dev))
    return (x * torch.where(torch.rand(cols, **dev) < 0.01, 8.0, 1.0)).half()


def _rng_state(seed):
    """Seed and step of the generator, as a program has them after some steps."""
    return torch.tensor([0x9E3779B97F4A7C15 % (1 << 62) + seed, (1 << 33) + 7 * seed],
                        dtype=torch.int64, device="cuda")


def _prepare_dense(case, g, dev, st):
    t, i, o = case["tokens"], case["inputs"], case["outputs"]
    st.update(sizes=(t, i, o), act=case["act"], x=_tokens(g, t, i), bias=None, residual=None)
    # weights that keep most sums near 1, where activations bend
    st["w"] = (torch.randn((o, i), **dev) / math.sqrt(2 * i)).half()
    if case["bias"]:
        st["bias"] = (0.1 * torch.randn(o, **dev)).half()
    if case["residual"]:
        st["residual"] = torch.randn((t, o), **dev).half()
    if st["kind"] == "dense_train":
        # of an earlier forward, so that no gradient hangs on a sum's last bit at 0
        st["z"] = torch.randn((t, o), **dev).half()
        st["dy"] = _tokens(g, t, o) * 1e-2


def _prepare_logits(case, g, dev, st):
    n, k, ld = case["rows"], case["classes"], case["stride"]
    z = torch.empty((n, ld), dtype=torch.float16, device="cuda")
    z[:, k:] = 0.0
    for a in range(0, n, 1024):  # (by parts: float32 copies of all rows are large)
        b = min(n, a + 1024)
        z[a:b, :k] = torch.randn((b - a, k), **dev) * 3.0
    # a class that most rows favour, and classes that are not allowed in every fourth
    at = torch.randint(k, (n,), **dev)
    z[torch.arange(n, device="cuda"), at] += torch.rand(n, **dev).half() * 16.0
    if k > 200:
        z[::4, k // 3:k // 3 + k // 16] = -math.inf
    token = torch.where(torch.rand(n, **dev) < 0.5, at, torch.randint(k // 3, (n,), **dev))
    token = torch.where((token >= k // 3) & (token < k // 3 + k // 16), 0, token)
    if n > 1:  # rows behind the end of a sequence ask for no class
        token = torch.where(torch.rand(n, **dev) < 0.1, -1, token)
    st.update(sizes=(n, k, ld), z=z, token=token.int(), top=case["top"], scale=case["scale"])
    if st["kind"] == "logprob_train":
        st["dlogp"] = torch.randn(n, **dev)
        st["dentropy"] = 0.01 * torch.ones(n, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dev = dict(device="cuda", generator=g)
    st = {"kind": case["kind"], "rng": _rng_state(int(seed) % 100003), "site": 3,
          "p": case.get("p", 0.0)}
    if case["kind"] in ("dense_fwd", "dense_train"):
        _prepare_dense(case, g, dev, st)
    elif case["kind"] == "dropout":
        n = case["n"]
        st["x"] = torch.randn(n, **dev).half()
        st["residual"] = torch.randn(n, **dev).half() if case["residual"] else None
        st["dy"] = (0.01 * torch.randn(n, **dev)).half()
    else:
        _prepare_logits(case, g, dev, st)
    return st


# ---- the plain forms ---------------------------------------------------------------

LOW = 0xFFFFFFFF


def _philox(c, k):
    """Ten rounds on tensors of 32-bit values in 64 bits."""
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # (low 64 bits, also past the sign)
        c = ((b >> 32) & LOW ^ c[1] ^ k[0], b & LOW, (a >> 32) & LOW ^ c[3] ^ k[1], a & LOW)
        k = ((k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW)
    return c


def _dropped(v, st):
    """v (float32) under the mask of its elements' numbers, kept ones over the
    probability of being kept."""
    t = int(math.floor(st["p"] * 65536 + 0.5))
    if t == 0:
        return v
    n = v.numel()
    seed, step = st["rng"][0], st["rng"][1]
    i = torch.arange(-(-n // 8), device=v.device)
    c = _philox((i, torch.full_like(i, st["site"]), step & LOW, (step >> 32) & LOW),
                (seed & LOW, (seed >> 32) & LOW))
    keep = torch.empty((i.numel(), 8), dtype=torch.bool, device=v.device)
    for j in range(8):
        keep[:, j] = ((c[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= t
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    return torch.where(keep.view(-1)[:n].view(v.shape), v * scale, 0.0)


def _active(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * (0.5 * torch.special.erfc(z * -math.sqrt(0.5)))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "gelu":
        return (0.5 * torch.special.erfc(z * -math.sqrt(0.5))
                + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _dense(st):
    z = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    y = _dropped(_active(z, st["act"]), st)
    y = (y if st["residual"] is None else y + st["residual"].float()).half()
    if st["kind"] == "dense_fwd":
        return y
    dz = _dropped(st["dy"].float(), st) * _slope(st["z"].float(), st["act"])
    dx, dw = dz @ st["w"].float(), dz.t() @ st["x"].float()
    return [y, z.half(), dx.half(), dw.half()] + ([] if st["bias"] is None
                                                  else [dz.sum(0).half()])


def _dropout(st):
    y = _dropped(st["x"].float(), st)
    y = y if st["residual"] is None else y + st["residual"].float()
    return [y.half(), _dropped(st["dy"].float(), st).half()]


def _logprob(st):
    n, k, _ = st["sizes"]
    z = st["z"][:, :k]
    top = z.float().amax(1, keepdim=True)
    d = (z.float() - top) * st["scale"]
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    log = torch.log(s)
    entropy = log[:, 0] - torch.where(e > 0, e * d, 0.0).sum(1) / s[:, 0]
    at = st["token"].long().clamp(min=0)[:, None]
    asked = st["token"] >= 0
    logp = torch.where(asked, (d.gather(1, at) - log)[:, 0], 0.0)
    out = [logp, entropy]
    if st["top"]:
        # whole-number keys, larger for larger values, then for lower places
        bits = z.contiguous().view(torch.int16).long()
        key = torch.where(bits < 0, -(bits & 0x7FFF), bits) << 32
        key = key + (k - torch.arange(k, device=z.device))
        best = k - (key.topk(st["top"], 1, largest=True, sorted=True).values & LOW)
        out += [best.int(), d.gather(1, best) - log]
    if st["kind"] == "logprob_train":
        p, given = e / s, d - log
        g = -st["dlogp"][:, None] * torch.where(asked[:, None], p, 0.0)
        g.scatter_add_(1, at, torch.where(asked, st["dlogp"], 0.0)[:, None])
        g -= st["dentropy"][:, None] * torch.where(p > 0, p * (given + entropy[:, None]), 0.0)
        out.append((g * st["scale"]).half())
    return out


# ---- this library's calls ------------------------------------------------------------

def _own_dense(st):
    import paper_1911_07384_amd as F
    t, i, o = st["sizes"]
    train = st["kind"] == "dense_train"
    if "ws" not in st:  # what a program keeps beside its weights
        st["desc"] = d = F.dense_desc(t, i, o, act=st["act"], drop=st["p"], site=st["site"])
        st["ws"] = F.workspace(F.fp16_dense_workspace_bytes(d, None if train else F.DENSE_FWD))
        st["y"] = torch.empty((t, o), dtype=torch.float16, device="cuda")
        if train:
            st["kept"] = torch.empty_like(st["y"])
            st["dx"], st["dw"] = torch.empty_like(st["x"]), torch.empty_like(st["w"])
            st["dbias"] = None if st["bias"] is None else torch.empty_like(st["bias"])
    d = st["desc"]
    F.fp16_dense_fwd(d, st["x"], st["w"], st["bias"], st["residual"], st["y"], st.get("kept"),
                     rng=st["rng"], ws=st["ws"])
    if not train:
        return st["y"]
    F.fp16_dense_bwd(d, st["x"], st["w"], st["z"], st["dy"], st["dx"], st["dw"], st["dbias"],
                     rng=st["rng"], ws=st["ws"])
    return [st["y"], st["kept"], st["dx"], st["dw"]] + ([] if st["bias"] is None
                                                        else [st["dbias"]])


def _own_dropout(st):
    import paper_1911_07384_amd as F
    if "y" not in st:
        st["y"], st["dx"] = torch.empty_like(st["x"]), torch.empty_like(st["x"])
    F.fp16_dropout(st["x"], st["residual"], st["y"], st["p"], st["rng"], site=st["site"])
    F.fp16_dropout(st["dy"], None, st["dx"], st["p"], st["rng"], site=st["site"])
    return [st["y"], st["dx"]]


def _own_logprob(st):
    import paper_1911_07384_amd as F
    n, k, ld = st["sizes"]
    if "ws" not in st:
        st["desc"] = d = F.logprob_desc(n, k, stride=ld, scale=st["scale"], top=st["top"])
        st["ws"] = F.workspace(F.fp16_logprobs_workspace_bytes(d))
        f32 = dict(dtype=torch.float32, device="cuda")
        st["logp"], st["stats"] = torch.empty(n, **f32), torch.empty((n, 3), **f32)
        st["top_id"] = st["top_logp"] = None
        if st["top"]:
            st["top_id"] = torch.empty((n, st["top"]), dtype=torch.int32, device="cuda")
            st["top_logp"] = torch.empty((n, st["top"]), **f32)
        if st["kind"] == "logprob_train":
            st["dz"] = torch.empty_like(st["z"])
    d = st["desc"]
    F.fp16_logprobs(d, st["z"], st["token"], st["logp"], st["stats"], st["top_id"],
                    st["top_logp"], ws=st["ws"])
    out = [st["logp"], st["stats"][:, 2]]
    if st["top"]:
        out += [st["top_id"], st["top_logp"]]
    if st["kind"] == "logprob_train":
        F.fp16_logprobs_bwd(d, st["z"], st["token"], st["stats"], st["dlogp"], st["dentropy"],
                            st["dz"])
        out.append(st["dz"][:, :k])
    return out


def run(state):
    kind = state["kind"]
    if kind in ("dense_fwd", "dense_train"):
        return _own_dense(state) if own else _dense(state)
    if kind == "dropout":
        return _own_dropout(state) if own else _dropout(state)
    return _own_logprob(state) if own else _logprob(state)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("dense_fwd", "dense_train"):
        t, i, o = case["tokens"], case["inputs"], case["outputs"]
        elems = t * i + o * i + t * o + (o if case["bias"] else 0)
        elems += t * o if case["residual"] else 0
        if kind == "dense_fwd":
            return {"bytes": 2 * elems, "flops": 2 * t * i * o}
        # z written and an earlier one read, dy, dx, dw, dbias
        elems += t * o * (2 if case["act"] != "none" else 1) + t * o + t * i + o * i
        elems += o if case["bias"] else 0
        return {"bytes": 2 * elems, "flops": 6 * t * i * o}
    if kind == "dropout":
        n = case["n"]
        return {"bytes": 2 * n * (5 if case["residual"] else 4),
                "flops": n * (3 if case["residual"] else 2)}
    n, k = case["rows"], case["classes"]
    if kind == "logprob":
        return {"bytes": 2 * n * k + n * 12 + 8 * n * case["top"], "flops": 5 * n * k}
    return {"bytes": 4 * n * k + n * 20, "flops": 11 * n * k}


# ---- the definitions in 64 bits ------------------------------------------------------

def _keep64(n, p, seed, step, site):
    """Which of n elements are kept: the generator in numpy's unsigned integers."""
    u = np.uint64
    ctr = np.zeros((4, -(-n // 8)), dtype=u)
    ctr[0] = np.arange(ctr.shape[1], dtype=u)
    ctr[1], ctr[2], ctr[3] = site, step % 2 ** 32, step >> 32
    for r in range(10):
        key = [(seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32,
               ((seed >> 32) + r * 0xBB67AE85) % 2 ** 32]
        m = ctr[0] * u(0xD2511F53)
        q = ctr[2] * u(0xCD9E8D57)
        ctr[0] = (q >> u(32)) ^ ctr[1] ^ u(key[0])
        ctr[1] = q & u(LOW)
        ctr[2] = (m >> u(32)) ^ ctr[3] ^ u(key[1])
        ctr[3] = m & u(LOW)
    words = np.ascontiguousarray(ctr.astype("<u4").T).view("<u2").reshape(-1)[:n]
    return words >= int(p * 65536 + 0.5)


def _mask64(st, shape):
    """What each element is multiplied with."""
    t = int(st["p"] * 65536 + 0.5)
    if t == 0:
        return 1.0
    seed, step = (int(v) for v in st["rng"].tolist())
    keep = torch.from_numpy(_keep64(int(np.prod(shape)), st["p"], seed, step, st["site"]))
    return keep.to("cuda").view(shape).double() * (65536 / max(1, 65536 - t))


def _phi64(z):
    return torch.special.ndtr(z)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "dropout":
        m = _mask64(st, st["x"].shape)
        y = st["x"].double() * m
        return [y if st["residual"] is None else y + st["residual"], st["dy"].double() * m]
    if kind in ("dense_fwd", "dense_train"):
        t, _, o = st["sizes"]
        z = torch.nn.functional.linear(st["x"].double(), st["w"].double())
        z = z if st["bias"] is None else z + st["bias"]
        act = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * _phi64(v),
               "silu": lambda v: v * torch.sigmoid(v)}[case["act"]]
        m = _mask64(st, (t, o))
        y = act(z) * m
        y = y if st["residual"] is None else y + st["residual"]
        if kind == "dense_fwd":
            return y
        kept = st["z"].double().requires_grad_()
        act(kept).backward(m * st["dy"].double())
        dz = kept.grad
        out = [y, z, dz.matmul(st["w"].double()), dz.mT.contiguous().matmul(st["x"].double())]
        return out if st["bias"] is None else out + [dz.sum(0)]
    n, k, _ = st["sizes"]
    if n * k > 1 << 28:
        return None
    logits = st["z"][:, :k].double() * st["scale"]
    lp = torch.log_softmax(logits, 1)
    p = lp.exp()
    entropy = torch.special.entr(p).sum(1)
    asked = st["token"] >= 0
    at = st["token"].long().clamp(min=0)[:, None]
    out = [torch.where(asked, lp.gather(1, at)[:, 0], 0.0), entropy]
    if st["top"]:
        out += [None, lp.sort(1, descending=True).values[:, :st["top"]]]
    if kind == "logprob_train":
        dl = torch.where(asked, st["dlogp"].double(), 0.0)
        g = torch.zeros_like(p).scatter_(1, at, dl[:, None]) - dl[:, None] * p
        g += st["dentropy"].double()[:, None] * (torch.special.entr(p) - p * entropy[:, None])
        out.append(g * st["scale"])
    return out
