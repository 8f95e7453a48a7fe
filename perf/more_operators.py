"""The two ends of a language model in a training step, as cases that can be timed and checked.

A step goes from tokens into rows of an embedding table and ends in a layer norm, a product with the vocabulary and the loss; on the
way back the gradients of both ends are the largest tensors of the buckets that are reduced.  A case is one pass through one of these:

  op "embed"        rows of a table by token, scaled
  op "embed_grad"   the table's gradient: the sums of the rows of each token, the whole table or added onto what the gradient holds
  op "norm"         layer norm over rows
  op "norm_grad"    the gradients of its input, weight and bias
  op "vocab"        log-probabilities and loss of given tokens under softmax(hidden weight^T), the logits never being kept
  op "vocab_grad"   the same, and the gradients of hidden and weight

With `own` false `run` computes them in elementary torch operations in 32 bits; with `own` true through the entry points of this
repository.  A token or target of -1 stands for a place without one (padding, a prompt).
"""
import functools
import math
import random

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
LOSS_SCALE = 1024.0     # of gradients in f16


def _embed(name, rows, dim, vocab, dtype, masked=0):
    c = {"op": "embed", "rows": rows, "dim": dim, "vocab": vocab, "dtype": dtype, "masked": masked}
    return dict(c, name=name) if name else c


def _embed_grad(name, rows, dim, vocab, dtype, out, onto, masked=0):
    c = {"op": "embed_grad", "rows": rows, "dim": dim, "vocab": vocab, "dtype": dtype, "out": out, "onto": onto, "masked": masked}
    return dict(c, name=name) if name else c


def _norm(name, rows, dim, dtype, param, grad):
    c = {"op": "norm_grad" if grad else "norm", "rows": rows, "dim": dim, "dtype": dtype, "param": param}
    return dict(c, name=name) if name else c


def _vocab(name, rows, dim, vocab, dtype, grad, masked=0, temperature=1.0):
    c = {"op": "vocab_grad" if grad else "vocab", "rows": rows, "dim": dim, "vocab": vocab, "dtype": dtype, "masked": masked, "temperature": temperature}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token while serving: nothing but latency
        _embed("embed 1 token", 1, 2048, 50257, "bf16"),
        # a micro-batch of long sequences, padded
        _embed("embed 16384 x 4096 bf16", 16384, 4096, 131072, "bf16", masked=900),
        # a small model's table, of odd sizes
        _embed_grad("embed grad 300 x 1001 f32", 300, 1001, 5003, "f32", "f32", False, masked=11),
        # a table that the head shares: its gradient is there already, the tokens' rows are added onto it
        _embed_grad("embed grad 16384 x 4096 bf16", 16384, 4096, 131072, "bf16", "bf16", True, masked=900),
        # one row while serving
        _norm("norm 1 x 4096 bf16", 1, 4096, "bf16", "bf16", False),
        # an ordinary micro-batch
        _norm("norm 16384 x 4096 bf16", 16384, 4096, "bf16", "bf16", False),
        # few rows of an odd length, as of a small model in 32 bits
        _norm("norm grad 333 x 1001 f32", 333, 1001, "f32", "f32", True),
        # the backward pass of the ordinary micro-batch, weights in 32 bits
        _norm("norm grad 16384 x 4096 bf16", 16384, 4096, "bf16", "f32", True),
        # the score of one token while serving
        _vocab("vocab 1 x 2048 x 50257 bf16", 1, 2048, 50257, "bf16", False),
        # a small micro-batch of a small model
        _vocab("vocab grad 48 x 1024 x 32000 f16", 48, 1024, 32000, "f16", True, masked=5, temperature=0.7),
        # a model kept in 32 bits, every size odd
        _vocab("vocab grad 1023 x 1001 x 50257 f32", 1023, 1001, 50257, "f32", True, masked=100),
        # the largest: a micro-batch of long sequences over a long vocabulary, prompts masked
        _vocab("vocab grad 8192 x 4096 x 131072", 8192, 4096, 131072, "bf16", True, masked=1500),
    ]


def _spread(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _even(rng, n, to=64):
    """Sizes are as often multiples of 64 as not."""
    return max(to, n // to * to) if rng.random() < 0.5 else n


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    op = rng.choice(("embed", "embed_grad", "norm", "norm_grad", "vocab", "vocab_grad", "vocab_grad"))
    param = rng.choice((dtype, "f32"))
    rows = _spread(rng, 1, 32769)
    if op in ("norm", "norm_grad"):
        dim = _even(rng, _spread(rng, 64, 16385))
        rows = max(1, min(rows, (1 << 28) // (dim * BYTES[dtype])))
        return _norm("", rows, dim, dtype, param, op == "norm_grad")
    vocab = _spread(rng, 1000, 131073)
    dim = _even(rng, _spread(rng, 64, 4097))
    if op == "embed":
        return _embed("", rows, dim, vocab, dtype, masked=rng.randrange(rows) // 4)
    if op == "embed_grad":
        return _embed_grad("", rows, dim, vocab, dtype, param, rng.random() < 0.5, masked=rng.randrange(rows) // 4)
    rows = max(1, min(_spread(rng, 1, 8193), 8192 * 4096 * (131072 // 2) // (vocab * dim)))
    return _vocab("", rows, dim, vocab, dtype, op == "vocab_grad", masked=rng.randrange(rows) // 3, temperature=rng.choice((1.0, 1.0, 0.7)))


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------
def _tokens(case, gen):
    """Tokens as text has them: the k-th most frequent about 1 / k as often as the first, spread over the table; -1 where there is none."""
    n, vocab = case["rows"], case["vocab"]
    rank = (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * math.log(vocab + 1.0)).exp().long().sub(1).clamp(0, vocab - 1)
    t = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    t[torch.randperm(n, generator=gen, device="cuda")[:case["masked"]]] = -1
    return t


def _normal(shape, std, dtype, gen):
    """Normal values of a type, made in parts: the 32-bit ones are never there whole."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // max(1, math.prod(shape[1:])))
    for a in range(0, shape[0], step):
        part = x[a:a + step]
        part.copy_(torch.empty(part.shape, device="cuda").normal_(0.0, std, generator=gen))
    return x


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    op, rows, dim, kind = case["op"], case["rows"], case["dim"], TORCH[case["dtype"]]
    if op in ("norm", "norm_grad"):
        # a residual stream: rows of different sizes around a small offset, a few channels far larger than the others
        size = torch.empty(rows, 1, device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
        channel = torch.ones(dim, device="cuda")
        channel[torch.randint(0, dim, (1 + dim // 200,), generator=gen, device="cuda")] = 12.0
        x = torch.empty(rows, dim, device="cuda").normal_(generator=gen).mul_(channel).add_(0.1).mul_(size)
        s = {"x": x.to(kind), "w": (1.0 + 0.1 * torch.randn(dim, generator=gen, device="cuda")).to(TORCH[case["param"]])}
        if op == "norm":
            s["b"] = _normal((dim,), 0.1, TORCH[case["param"]], gen)
        else:
            s["dy"] = _normal((rows, dim), 0.05, kind, gen)
        return s
    t = _tokens(case, gen)
    if op == "embed":
        return {"t": t, "table": _normal((case["vocab"], dim), 0.02, kind, gen)}
    if op == "embed_grad":
        s = {"t": t, "g": _normal((rows, dim), 0.01, kind, gen)}
        if case["onto"]:
            s["G"] = _normal((case["vocab"], dim), 0.02, TORCH[case["out"]], gen)
        return s
    # logits of a spread of 2.5; a token that comes next is expected more or less
    std = 2.5 / math.sqrt(dim)
    s = {"t": t, "W": _normal((case["vocab"], dim), std, kind, gen)}
    x = torch.empty(rows, dim, device="cuda").normal_(generator=gen)
    x += torch.rand(rows, 1, generator=gen, device="cuda") * 2.0 * s["W"][t.clamp(min=0)].float()
    s["X"] = x.to(kind)
    s["weight"] = (t >= 0).float()
    s["scale"] = (LOSS_SCALE if case["dtype"] == "f16" else 1.0) / s["weight"].sum().clamp(min=1.0)
    return s


def prepare(case, seed):
    """The inputs, the buffers that outputs go to and the workspaces: what a training program lays out once."""
    s = _inputs(case, seed)
    op, rows, dim, kind = case["op"], case["rows"], case["dim"], TORCH[case["dtype"]]
    dev = {"device": "cuda"}
    s["case"] = case
    if op in ("embed", "norm"):
        s["out"] = torch.empty(rows, dim, dtype=kind, **dev)
    elif op == "embed_grad" and not case["onto"]:
        s["G"] = torch.empty(case["vocab"], dim, dtype=TORCH[case["out"]], **dev)
    elif op == "norm_grad":
        s["out"] = {"x": torch.empty(rows, dim, dtype=kind, **dev), "w": torch.empty(dim, dtype=TORCH[case["param"]], **dev),
                    "b": torch.empty(dim, dtype=TORCH[case["param"]], **dev)}
    elif op in ("vocab", "vocab_grad"):
        s["out"] = {"logp": torch.empty(rows, **dev)}
        if op == "vocab_grad":
            s["out"].update(loss=torch.empty(rows, **dev), sums=torch.empty(2, **dev), X=torch.empty(rows, dim, dtype=kind, **dev),
                            W=torch.empty(case["vocab"], dim, dtype=kind, **dev))
    if own:
        import paper_2303_06324_amd as dfx
        s["dfx"] = dfx
        kinds = {"f32": dfx.F32, "bf16": dfx.BF16, "f16": dfx.F16}
        s["kind"] = kinds[case["dtype"]]
        s["other"] = kinds[case.get("out", case.get("param", case["dtype"]))]
        n = 0
        if op == "embed_grad":
            n = dfx.embed_grad_workspace(rows, dim, case["vocab"], s["kind"])
        elif op == "norm_grad":
            n = dfx.layer_norm_grad_workspace(rows, dim, s["kind"])
        elif op in ("vocab", "vocab_grad"):
            n = dfx.vocab_loss_workspace(rows, dim, case["vocab"], s["kind"], grad=op == "vocab_grad")
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, **dev)
    return s


# --------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state, state["case"]) if own else globals()["_plain_" + state["case"]["op"]](state, state["case"])


def _run_own(s, case):
    dfx, op, rows, dim, stream = s["dfx"], case["op"], case["rows"], case["dim"], torch.cuda.current_stream().cuda_stream
    if op == "embed":
        dfx.embed(rows, dim, case["vocab"], s["kind"], s["t"].data_ptr(), s["table"].data_ptr(), s["out"].data_ptr(), scale=math.sqrt(dim), stream=stream)
        return s["out"]
    work = {"workspace": s["work"].data_ptr(), "workspace_bytes": s["work"].numel(), "stream": stream}
    if op == "embed_grad":
        dfx.embed_grad(rows, dim, case["vocab"], s["kind"], s["t"].data_ptr(), s["g"].data_ptr(), s["G"].data_ptr(), out_dtype=s["other"],
                       scale=math.sqrt(dim), accumulate=case["onto"], **work)
        return s["G"]
    if op == "norm":
        dfx.layer_norm(rows, dim, s["kind"], s["x"].data_ptr(), s["out"].data_ptr(), weight=s["w"].data_ptr(), bias=s["b"].data_ptr(),
                       param_dtype=s["other"], eps=EPS, stream=stream)
        return s["out"]
    out = s["out"]
    if op == "norm_grad":
        dfx.layer_norm_grad(rows, dim, s["kind"], s["x"].data_ptr(), s["dy"].data_ptr(), out["x"].data_ptr(), weight=s["w"].data_ptr(),
                            grad_weight=out["w"].data_ptr(), grad_bias=out["b"].data_ptr(), param_dtype=s["other"], eps=EPS, **work)
        return out
    more = {"loss": out["loss"].data_ptr(), "sums": out["sums"].data_ptr(), "scale": s["scale"].data_ptr(), "grad_hidden": out["X"].data_ptr(),
            "grad_weight": out["W"].data_ptr()} if op == "vocab_grad" else {}
    dfx.vocab_loss(rows, dim, case["vocab"], s["kind"], s["X"].data_ptr(), s["W"].data_ptr(), s["t"].data_ptr(), row_weight=s["weight"].data_ptr(),
                   logp=out["logp"].data_ptr(), inv_temperature=1.0 / case["temperature"], **more, **work)
    return out


def _plain_embed(s, case):
    t = s["t"]
    return (s["table"][t.clamp(min=0)].float() * ((t >= 0).float() * math.sqrt(case["dim"]))[:, None]).to(s["table"].dtype)


def _plain_embed_grad(s, case):
    t = s["t"]
    g = s["g"].float() * ((t >= 0).float() * math.sqrt(case["dim"]))[:, None]
    if not case["onto"]:
        return torch.zeros(s["G"].shape, device="cuda").index_add_(0, t.clamp(min=0), g).to(s["G"].dtype)
    G = s["G"].float().index_add_(0, t.clamp(min=0), g)
    s["G"].copy_(G)
    return s["G"]


def _plain_stats(x):
    x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    return x * r, r


def _plain_norm(s, case):
    h, _ = _plain_stats(s["x"].float())
    return (h * s["w"].float() + s["b"].float()).to(s["x"].dtype)


def _plain_norm_grad(s, case):
    h, r = _plain_stats(s["x"].float())
    dy = s["dy"].float()
    dw, db = (dy * h).sum(0), dy.sum(0)
    g = dy * s["w"].float()
    dx = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return {"x": dx.to(s["x"].dtype), "w": dw.to(s["w"].dtype), "b": db.to(s["w"].dtype)}


def _plain_softmax(s, case):
    """Log-probabilities of the targets (0 where there is none), exponentials around the largest logit, and their sums."""
    z = s["X"].float() @ s["W"].float().t()
    if case["temperature"] != 1.0:
        z *= 1.0 / case["temperature"]
    top = z.amax(1, keepdim=True)
    zt = z.gather(1, s["t"].clamp(min=0)[:, None])
    e = z.sub_(top).exp_()
    total = e.sum(1, keepdim=True)
    return (zt - top - total.log())[:, 0] * s["weight"], e, total


def _plain_vocab(s, case):
    return {"logp": _plain_softmax(s, case)[0]}


def _plain_vocab_grad(s, case):
    logp, e, total = _plain_softmax(s, case)
    per = s["weight"] * s["scale"] * (1.0 / case["temperature"])
    dz = e.mul_(per[:, None] / total).scatter_add_(1, s["t"].clamp(min=0)[:, None], -per[:, None])
    loss = -logp * s["weight"]
    return {"logp": logp, "loss": loss, "sums": torch.stack([loss.sum(), s["weight"].sum()]), "X": (dz @ s["W"].float()).to(s["X"].dtype),
            "W": (dz.t() @ s["X"].float()).to(s["W"].dtype)}


# --------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# --------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _distinct(n, vocab):
    """How many different tokens n draws of _tokens have, on average."""
    k = np.arange(1, vocab + 1, dtype=np.float64)
    return int(np.sum(-np.expm1(n * np.log1p(-np.log1p(1.0 / k) / math.log(vocab + 1.0)))))


def work(case):
    op, rows, dim, e = case["op"], case["rows"], case["dim"], BYTES[case["dtype"]]
    if op == "norm":
        return {"bytes": 2 * rows * dim * e + 2 * dim * BYTES[case["param"]], "flops": 8 * rows * dim}
    if op == "norm_grad":
        return {"bytes": 3 * rows * dim * e + 3 * dim * BYTES[case["param"]], "flops": 16 * rows * dim}
    read, vocab = rows - case["masked"], case["vocab"]
    if op == "embed":
        return {"bytes": (_distinct(read, vocab) + rows) * dim * e + 8 * rows, "flops": read * dim}
    if op == "embed_grad":
        rows_of_table = 2 * _distinct(read, vocab) if case["onto"] else vocab
        return {"bytes": read * dim * e + rows_of_table * dim * BYTES[case["out"]] + 8 * rows, "flops": 2 * read * dim}
    if op == "vocab":
        return {"bytes": (read + vocab) * dim * e + 16 * rows, "flops": 2 * read * vocab * dim}
    return {"bytes": (read + rows + 2 * vocab) * dim * e + 20 * rows, "flops": 6 * read * vocab * dim}


def _exact_vocab(s, case):
    c, rows = 1.0 / case["temperature"], case["rows"]
    grad, W = case["op"] == "vocab_grad", s["W"].double()
    logp = torch.zeros(rows, dtype=torch.float64, device="cuda")
    dX = torch.zeros(rows, case["dim"], dtype=torch.float64, device="cuda") if grad else None
    dW = torch.zeros_like(W) if grad else None
    places = torch.nonzero(s["t"] >= 0)[:, 0]
    for at in places.split(max(1, (1 << 27) // case["vocab"])):
        X, t = s["X"][at].double(), s["t"][at]
        z = torch.mm(X, W.t()).mul_(c)
        lse = torch.logsumexp(z, 1)
        i = torch.arange(len(at), device="cuda")
        logp[at] = z[i, t] - lse
        if not grad:
            continue
        p = z.sub_(lse[:, None]).exp_()
        p[i, t] -= 1.0
        p *= c * float(s["scale"])
        dX[at] = torch.mm(p, W)
        dW.addmm_(p.t(), X)
    if not grad:
        return {"logp": logp}
    n = torch.tensor(float(len(places)), dtype=torch.float64, device="cuda")
    return {"logp": logp, "loss": -logp, "sums": torch.stack([-logp.sum(), n]), "X": dX, "W": dW}


def exact(case, seed):
    s = _inputs(case, seed)
    op, dim = case["op"], case["dim"]
    if op in ("vocab", "vocab_grad"):
        return _exact_vocab(s, case)
    if op == "embed":
        out = torch.zeros(case["rows"], dim, dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["t"] >= 0)[:, 0]
        out[at] = s["table"][s["t"][at]].double() * dim ** 0.5
        return out
    if op == "embed_grad":
        G = s["G"].double() if case["onto"] else torch.zeros(case["vocab"], dim, dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["t"] >= 0)[:, 0]
        return G.index_add_(0, s["t"][at], s["g"][at].double(), alpha=dim ** 0.5)
    x, w = s["x"].double(), s["w"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    root = torch.sqrt(var + EPS)
    h = (x - mean) / root
    if op == "norm":
        return torch.addcmul(s["b"].double(), h, w)
    dy = s["dy"].double()
    g = dy * w
    dx = (g - torch.sum(g, 1, keepdim=True) / dim - h * (torch.sum(g * h, 1, keepdim=True) / dim)) / root
    return {"x": dx, "w": torch.sum(dy * h, 0), "b": torch.sum(dy, 0)}
