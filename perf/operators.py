"""The cases that the language-model operators are measured on: layer norm, embedding
lookup, the stable embedding layer, and the global gradient norm with clipping.

Each is what a training program runs around an 8-bit optimizer step, or what a
serving program runs for a few tokens, through the public entry points: ``nn``'s
functions with torch's autograd for the gradients, ``bq``'s forward calls where
no gradient is wanted, and ``optim.clip_grad_norm_``.  ``run`` computes the same in
elementary torch operations where ``own`` is false.

Sizes are those of the package's own lists (GPT-2-shaped: d 1024 and 1600, vocabulary
50257, context 1024; ResNet-50) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

ALIGN = 512       # elements between the starts of a flat buffer's tensors
EPS = 1e-5
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
ACTIVE, IDLE = 1.0, 1e9   # limits of the clipped norm: always, and never reached


def listed():
    return [
        # generating text: the final layer norm for one new token of each of 8 sequences
        dict(name="ln_token_1600", kind="ln_fwd", rows=8, cols=1600, x="bfloat16", w="float32"),
        # scoring prompts: 8 sequences of 1024 tokens, all in fp16
        dict(name="ln_prompt_1600", kind="ln_fwd", rows=8192, cols=1600, x="float16", w="float16"),
        # training the 1.5B-parameter model: 32 sequences, bf16 activations, fp32 parameters
        dict(name="ln_train_1600", kind="ln_train", rows=32768, cols=1600, x="bfloat16",
             w="float32"),
        # training the 354.8M-parameter model in fp32: 16 sequences
        dict(name="ln_train_1024", kind="ln_train", rows=16384, cols=1024, x="float32",
             w="float32"),
        # rows of an odd length (a feature vector with its length appended), a ragged batch
        dict(name="ln_train_odd", kind="ln_train", rows=4999, cols=1001, x="float16", w="float16"),
        # generating text: the embeddings of 8 new tokens, scaled by sqrt(d)
        dict(name="emb_token_1600", kind="emb_fwd", tokens=8, vocab=50257, dim=1600, w="float32",
             y="bfloat16", scale=40.0, pad=False),
        # training the 354.8M-parameter model: 16 sequences, bf16 weights and gradients
        dict(name="emb_train_1024", kind="emb_train", tokens=16384, vocab=50257, dim=1024,
             w="bfloat16", y="bfloat16", scale=32.0, pad=False),
        # training the 1.5B-parameter model: 64 padded sequences, fp32 weights, bf16 activations
        dict(name="emb_train_1600", kind="emb_train", tokens=65536, vocab=50257, dim=1600,
             w="float32", y="bfloat16", scale=1.0, pad=True),
        # a small model on a small vocabulary: one sequence of 509 tokens
        dict(name="stable_train_small", kind="stable_train", tokens=509, vocab=1000, dim=256,
             w="float32", y="float32", pad=False),
        # the stable embedding of the 1.5B-parameter model: 32 padded sequences, all fp32
        dict(name="stable_train_1600", kind="stable_train", tokens=32768, vocab=50257, dim=1600,
             w="float32", y="float32", pad=True),
        # vision training: the norm of the ResNet-50 list's fp32 gradients, below the limit
        dict(name="clip_resnet50", kind="clip", model="resnet50", grad="float32", limit=IDLE,
             norm="2"),
        # training the 1.5B-parameter model: its 580 fp16 gradients, above the limit
        dict(name="clip_lm1p5b", kind="clip", model="lm", layers=48, d=1600, vocab=50257, ctx=1024,
             grad="float16", limit=ACTIVE, norm="2"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["ln_fwd", "ln_train", "ln_train", "emb_fwd", "emb_train", "stable_train",
                       "clip"])
    if kind in ("ln_fwd", "ln_train"):
        x, w = rng.choice([("float32", "float32"), ("float16", "float16"),
                           ("bfloat16", "bfloat16"), ("float16", "float32"),
                           ("bfloat16", "float32")])
        cols = _log_int(rng, 40, 20000)
        return dict(kind=kind, rows=_log_int(rng, 1, max(2, min(40000, 50_000_000 // cols))),
                    cols=cols, x=x, w=w)
    if kind == "clip":
        grad = rng.choice(["float32", "float16", "bfloat16"])
        c = dict(kind=kind, grad=grad, norm=rng.choice(["2", "2", "2", "inf"]),
                 # an fp32 list is below the limit after its first pass, whatever that is
                 limit=IDLE if grad == "float32" else rng.choice([ACTIVE, IDLE]))
        if rng.random() < 0.5:
            c.update(model="ragged", count=_log_int(rng, 1, 700), total=_log_int(rng, 1e4, 1e9) | 1,
                     shape_seed=rng.randrange(1 << 20))
        else:
            c.update(model="lm", layers=rng.randint(1, 24), d=rng.randint(64, 1024),
                     vocab=_log_int(rng, 1000, 60000), ctx=_log_int(rng, 64, 2048))
        return c
    w, y = rng.choice([("float32", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"),
                       ("float32", "float16"), ("float32", "bfloat16")])
    dim = _log_int(rng, 40, 2000)
    c = dict(kind=kind, tokens=_log_int(rng, 1, 65000), vocab=_log_int(rng, 50, 130000 // (1 + dim // 800)),
             dim=dim, w=w, y=y, pad=rng.random() < 0.5)
    if kind != "stable_train":
        c["scale"] = rng.choice([1.0, math.sqrt(dim)])
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 64 + what) & ((1 << 62) - 1))
    return g


def _normal(shape, std, seed, what):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(
        0.0, std, generator=_gen(seed, what))


def _cast(x, dtype):
    return x.to(getattr(torch, dtype))


def _hidden(case, seed):
    """A residual stream: unit values around an offset, a few channels twenty times larger."""
    x = _normal((case["rows"], case["cols"]), 1.0, seed, 0) + 0.25
    at = torch.randint(0, case["cols"], (max(1, case["cols"] // 400),), device="cuda",
                       generator=_gen(seed, 1))
    x[:, at] *= 20.0
    return _cast(x, case["x"])


def _affine(n, dtype, seed):
    return (_cast(_normal((n,), 0.1, seed, 2) + 1.0, dtype), _cast(_normal((n,), 0.02, seed, 3), dtype))


def _ids(case, seed):
    """Tokens whose frequency falls with their rank, the last tenth of them padding if asked."""
    t, v = case["tokens"], case["vocab"]
    u = torch.rand(t, dtype=torch.float64, device="cuda", generator=_gen(seed, 4))
    ids = (torch.exp(u * math.log(v + 1)) - 1).long().clamp_(0, v - 1)
    if case["pad"]:
        ids[t - t // 10:] = v - 1
    return ids


def _padding(case):
    return case["vocab"] - 1 if case["pad"] else None


def _numels(case):
    if case["model"] == "ragged":  # sizes spread over two decades, summing to total
        rng = random.Random(case["shape_seed"])
        share = [math.exp(rng.uniform(0.0, math.log(100.0))) for _ in range(case["count"])]
        out = [max(1, int(case["total"] * s / sum(share))) for s in share]
        out[0] += max(0, case["total"] - sum(out))
        return out
    if case["model"] == "resnet50":
        out = [64 * 3 * 49, 64, 64]
        cin = 64
        for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                out += [width * cin, width, width, width * width * 9, width, width,
                        4 * width * width, 4 * width, 4 * width]
                if b == 0:
                    out += [4 * width * cin, 4 * width, 4 * width]
                cin = 4 * width
        return out + [1000 * 2048, 1000]
    d = case["d"]
    layer = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
    return [case["vocab"] * d, case["ctx"] * d] + case["layers"] * layer + [d, d]


def _places(case):
    place, e = [], 0
    for n in _numels(case):
        place.append((e, n))
        e += -(-n // ALIGN) * ALIGN
    return place, e


def _grads(case, seed):
    """One flat buffer of N(0, 1e-3), one value in ten thousand a hundred times larger."""
    place, n = _places(case)
    g = _normal((n,), 1e-3, seed, 5)
    at = torch.randint(0, n, (max(1, n // 10_000),), device="cuda", generator=_gen(seed, 6))
    g[at] *= 100.0
    return place, _cast(g, case["grad"])


def prepare(case, seed):
    kind = case["kind"]
    s = dict(case=case)
    if kind == "clip":
        place, s["flat"] = _grads(case, seed)
        s["grads"] = [s["flat"][e:e + n] for e, n in place]
        s["params"] = []
        for g in s["grads"]:
            # fp32 master weights with gradients of their own type: only the gradients count here
            p = torch.nn.Parameter(torch.empty(1, device="cuda").expand(g.numel()))
            p.grad_dtype = None
            p.grad = g
            s["params"].append(p)
        return s
    train = kind.endswith("train")
    if kind.startswith("ln"):
        s["x"] = _hidden(case, seed).requires_grad_(train)
        w, b = _affine(case["cols"], case["w"], seed)
        shape, dtype = (case["rows"], case["cols"]), case["x"]
    else:
        s["ids"] = _ids(case, seed)
        s["table"] = _cast(_normal((case["vocab"], case["dim"]), 0.02, seed, 0),
                           case["w"]).requires_grad_(train)
        w, b = _affine(case["dim"], case["w"], seed)
        shape, dtype = (case["tokens"], case["dim"]), case["y"]
    if not kind.startswith("emb"):
        s["w"], s["b"] = w.requires_grad_(train), b.requires_grad_(train)
    if train:
        s["dy"] = _cast(_normal(shape, 1e-2, seed, 7), dtype)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2110_02861_amd import bq, nn, optim
    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        norm = optim.clip_grad_norm_(s["params"], case["limit"], norm_type=float(case["norm"]))
        return {"norm": norm, "grads": s["flat"]}
    if kind == "ln_fwd":
        return {"y": bq.bq_layer_norm_forward(s["x"], s["w"], s["b"], EPS)}
    if kind == "emb_fwd":
        return {"y": bq.bq_embedding_forward(s["table"], s["ids"], scale=case["scale"],
                                             out_dtype=getattr(torch, case["y"]))}
    if kind == "ln_train":
        y = nn.layer_norm(s["x"], s["w"], s["b"], EPS)
        dx, dw, db = torch.autograd.grad(y, (s["x"], s["w"], s["b"]), s["dy"])
        return {"y": y.detach(), "dx": dx, "dw": dw, "db": db}
    out = getattr(torch, case["y"])
    if kind == "emb_train":
        y = nn.embedding(s["ids"], s["table"], padding_idx=_padding(case), scale=case["scale"],
                         out_dtype=out)
        dtable, = torch.autograd.grad(y, (s["table"],), s["dy"])
        return {"y": y.detach(), "dtable": dtable}
    y = nn.stable_embedding(s["ids"], s["table"], s["w"], s["b"], EPS, padding_idx=_padding(case),
                            out_dtype=out)
    dtable, dw, db = torch.autograd.grad(y, (s["table"], s["w"], s["b"]), s["dy"])
    return {"y": y.detach(), "dtable": dtable, "dw": dw, "db": db}


def _plain_norm(x):
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / torch.sqrt(xc.square().mean(-1, keepdim=True) + EPS)
    return xc * rstd, rstd


def _plain_norm_grad(xh, rstd, w, dy):
    g = dy * w
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _plain_scatter(rows, s, case):
    d = torch.zeros(case["vocab"], case["dim"], dtype=torch.float32, device="cuda")
    d.index_add_(0, s["ids"], rows)
    if case["pad"]:
        d[case["vocab"] - 1] = 0.0
    return d


@torch.no_grad()
def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        if case["norm"] == "2":
            norm = torch.stack([g.float().square().sum(dtype=torch.float64)
                                for g in s["grads"]]).sum().sqrt()
        else:
            norm = torch.stack([g.abs().max() for g in s["grads"]]).max().double()
        coef = (case["limit"] / (norm + 1e-6)).clamp(max=1.0).float()
        for g in s["grads"]:
            g.copy_(g.float() * coef)
        return {"norm": norm.float(), "grads": s["flat"]}
    if kind.startswith("ln"):
        x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
        xh, rstd = _plain_norm(x)
        out = {"y": _cast(xh * w + b, case["x"])}
        if kind == "ln_train":
            dx, dw, db = _plain_norm_grad(xh, rstd, w, s["dy"].float())
            out.update(dx=_cast(dx, case["x"]), dw=_cast(dw, case["w"]), db=_cast(db, case["w"]))
        return out
    rows = s["table"][s["ids"]].float()
    if kind.startswith("emb"):
        out = {"y": _cast(rows * case["scale"], case["y"])}
        if kind == "emb_train":
            out["dtable"] = _cast(_plain_scatter(s["dy"].float() * case["scale"], s, case), case["w"])
        return out
    w, b, dy = s["w"].float(), s["b"].float(), s["dy"].float()
    xh, rstd = _plain_norm(rows)
    dx, dw, db = _plain_norm_grad(xh, rstd, w, dy)
    return {"y": _cast(xh * w + b, case["y"]), "dtable": _cast(_plain_scatter(dx, s, case), case["w"]),
            "dw": _cast(dw, case["w"]), "db": _cast(db, case["w"])}


# ---------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------

def _distinct(case):
    """The expected number of distinct tokens (their probabilities: log((i + 2) / (i + 1)))."""
    v = case["vocab"]
    i = torch.arange(v, dtype=torch.float64)
    p = torch.log((i + 2) / (i + 1)) / math.log(v + 1)
    t = case["tokens"] * (0.9 if case["pad"] else 1.0)
    return min(float((1.0 - torch.exp(t * torch.log1p(-p))).sum()), case["tokens"])


def work(case):
    kind = case["kind"]
    if kind == "clip":
        n = sum(_numels(case))
        times = 1 if case["limit"] == IDLE else 2
        return {"bytes": times * n * SIZE[case["grad"]] + 4, "flops": (1 + times) * n}
    if kind.startswith("ln"):
        m, n, sx, sw = case["rows"], case["cols"], SIZE[case["x"]], SIZE[case["w"]]
        if kind == "ln_fwd":
            return {"bytes": 2 * m * n * sx + 2 * n * sw, "flops": 8 * m * n}
        return {"bytes": 4 * m * n * sx + 4 * n * sw, "flops": 20 * m * n}
    t, v, d = case["tokens"], case["vocab"], case["dim"]
    sw, sy = SIZE[case["w"]], SIZE[case["y"]]
    forward = 8 * t + _distinct(case) * d * sw + t * d * sy
    if kind == "emb_fwd":
        return {"bytes": int(forward), "flops": t * d}
    if kind == "emb_train":
        return {"bytes": int(forward + t * d * sy + v * d * sw), "flops": 3 * t * d}
    return {"bytes": int(forward + t * d * sy + v * d * sw + 4 * d * sw), "flops": 20 * t * d}


def _exact_rows(ids, values, vocab):
    """Sums of the values' rows by id: differences of the running sums of the sorted rows."""
    order = torch.argsort(ids, stable=True)
    run = values[order].cumsum(0)
    last = torch.bincount(ids, minlength=vocab).cumsum(0)
    at = torch.cat([torch.zeros(1, values.shape[1], dtype=torch.float64, device="cuda"), run])[last]
    return torch.diff(at, dim=0, prepend=torch.zeros_like(at[:1]))


def _exact_layer_norm(x, w, b):
    """Value, and a function of dy that gives the gradients: x's from the projection onto
    what is orthogonal to the constant vector and to the normalized row."""
    n = x.shape[1]
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    inv = torch.rsqrt(var + EPS)
    xh = (x - mean) * inv

    def grads(dy):
        g = dy * w
        along = g.mul(xh).sum(1, keepdim=True) / n
        return inv * (g - g.sum(1, keepdim=True) / n - along * xh), (dy * xh).sum(0), dy.sum(0)
    return torch.addcmul(b, xh, w), grads


@torch.no_grad()
def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "clip":
        flat = s["flat"].double()
        if case["norm"] == "2":
            norm = math.sqrt(sum(float(torch.dot(flat[e:e + n], flat[e:e + n]))
                                 for e, n in _places(case)[0]))
        else:
            norm = max(float(flat[e:e + n].abs().max()) for e, n in _places(case)[0])
        coef = min(1.0, case["limit"] / (norm + 1e-6))
        for e, n in _places(case)[0]:
            flat[e:e + n] *= coef
        return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "grads": flat}
    if kind.startswith("ln"):
        y, grads = _exact_layer_norm(s["x"].double(), s["w"].double(), s["b"].double())
        if kind == "ln_fwd":
            return {"y": y}
        dx, dw, db = grads(s["dy"].double())
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    rows = s["table"].double()[s["ids"]]
    if kind.startswith("emb"):
        if kind == "emb_fwd":
            return {"y": rows * case["scale"]}
        d = _exact_rows(s["ids"], s["dy"].double(), case["vocab"]) * case["scale"]
        if case["pad"]:
            d[-1] = 0.0
        return {"y": rows * case["scale"], "dtable": d}
    y, grads = _exact_layer_norm(rows, s["w"].double(), s["b"].double())
    dx, dw, db = grads(s["dy"].double())
    d = _exact_rows(s["ids"], dx, case["vocab"])
    if case["pad"]:
        d[-1] = 0.0
    return {"y": y, "dtable": d, "dw": dw, "db": db}
