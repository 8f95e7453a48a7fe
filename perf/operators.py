"""The training step around the collectives, as cases that can be timed and checked.

A data-parallel step has a loss in front of its gradient all-reduce and, behind it, the norm of all gradients, the clipping
and the update.  A case is one pass through one of these:

  op "loss"    the clipped policy loss with its KL term over rows of logits: forward alone (the log-probabilities of given
               tokens), or forward and the gradient of the logits
  op "norm"    the norm of all gradients of a list
  op "clip"    that norm, and the gradients scaled by the clip factor into the buffers that the optimizer reads
  op "adamw"   the update of 32-bit parameters and moments by gradients that are clipped on the way, with a 16-bit copy of
               the parameters where the model computes in 16 bits

With `own` false `run` computes them in elementary torch operations in 32 bits; with `own` true through the entry points of
this repository.  Gradients are lists of tensors that lie one behind the other in a flat bucket, as a bucketed all-reduce
leaves them: their places are multiples of the element's size and of nothing else.  The plain form works on whole buckets.
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
RANKS = 8               # the sum of so many ranks' gradients becomes their mean on the way
LOSS_SCALE = 1024.0     # of gradients in f16
MAX_NORM = 1.0
LR, BETA1, BETA2, EPS, DECAY, STEP = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1000
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
MIB = 1 << 20


def _list(name, op, tensors, elems, dtype, even=False, spec=0, **more):
    c = {"op": op, "tensors": tensors, "elems": elems, "dtype": dtype, "even": even, "spec": spec, **more}
    return dict(c, name=name) if name else c


def _loss(name, rows, vocab, dtype, grad, masked=0, temperature=1.0):
    c = {"op": "loss", "rows": rows, "vocab": vocab, "dtype": dtype, "grad": grad, "masked": masked, "temperature": temperature}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the biases and norm weights of one small block: nothing but latency
        _list("norm 9 small f32", "norm", 9, 12345, "f32", spec=1),
        # sixteen gradient buckets of the usual 25 MiB, as the disordered all-reduces of the benchmark leave them
        _list("norm 16 buckets 25 MiB bf16", "norm", 16, 16 * 25 * MIB // 2, "bf16", even=True),
        # every gradient of a model kept in 32 bits, of all sizes
        _list("norm 148 ragged 1 GiB f32", "norm", 148, 256 * MIB + 77, "f32", spec=2),
        # a small model's gradients, clipped
        _list("clip 24 small f32", "clip", 24, 200003, "f32", spec=3, out="f32"),
        # the buckets again, their mean clipped into the 32-bit gradients of the optimizer
        _list("clip 16 buckets 25 MiB bf16", "clip", 16, 16 * 25 * MIB // 2, "bf16", even=True, out="f32"),
        # the update of a small model
        _list("adamw 24 small f32", "adamw", 24, 500009, "f32", spec=4, copy=""),
        # the update of a model that computes in 16 bits, all its parameters
        _list("adamw 148 ragged bf16", "adamw", 148, 124 * 1000 * 1000 * 3 + 1, "bf16", spec=5, copy="bf16"),
        # the log-probability of one token while serving
        _loss("logp 1 token 50257 bf16", 1, 50257, "bf16", False),
        # scoring a batch of answers by the reference policy
        _loss("logp 2048 x 32000 bf16", 2048, 32000, "bf16", False, masked=300),
        # a small micro-batch over a long vocabulary
        _loss("loss 16 x 128000 f16", 16, 128000, "f16", True, temperature=0.7),
        # an ordinary micro-batch in 32 bits, rows of an odd length
        _loss("loss 1024 x 50257 f32", 1024, 50257, "f32", True, masked=111),
        # the largest: a micro-batch of long answers over a long vocabulary, prompts masked
        _loss("loss 4096 x 131072 bf16", 4096, 131072, "bf16", True, masked=700),
    ]


def _spread(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    op = rng.choice(("loss", "loss", "norm", "clip", "adamw"))
    if op == "loss":
        vocab = _spread(rng, 1000, 131072)
        rows = _spread(rng, 1, 4096)
        rows = max(1, min(rows, 4096 * 131072 * 2 // (vocab * BYTES[dtype])))
        return _loss("", rows, vocab, dtype, rng.random() < 0.6, masked=rng.randrange(rows) // 3, temperature=rng.choice((1.0, 1.0, 0.7)))
    elems = _spread(rng, 5000, {"norm": 256, "clip": 200, "adamw": 350}[op] * MIB)
    tensors = _spread(rng, 1, min(600, elems // 500))
    more = {"out": rng.choice(("f32", dtype))} if op == "clip" else {"copy": rng.choice(("", "bf16", "f16"))} if op == "adamw" else {}
    return _list("", op, tensors, elems, dtype, spec=rng.randrange(1 << 20), **more)


# --------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------
def _sizes(case):
    """Elements of each tensor of the list: equal buckets, or sizes spread over a factor of a thousand (matrices, biases)."""
    n, total = case["tensors"], case["elems"]
    if case["even"]:
        return [total // n] * n
    rng = random.Random(case["spec"])
    share = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(n)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    sizes[sizes.index(max(sizes))] += total - sum(sizes)
    return sizes


def _grad_scale(case):
    return 1.0 / (RANKS * (LOSS_SCALE if case["dtype"] == "f16" else 1.0))


def _inputs(case, seed):
    """What the pass reads and writes, as tensors on the GPU, from the seed alone."""
    gen = torch.Generator("cuda").manual_seed(seed)
    dev = {"device": "cuda"}
    if case["op"] == "loss":
        rows, vocab = case["rows"], case["vocab"]
        s = {"logits": torch.empty(rows, vocab, dtype=TORCH[case["dtype"]], **dev)}
        t, at = torch.empty(rows, dtype=torch.int64, **dev), torch.empty(rows, **dev)
        step = max(1, (1 << 27) // vocab)
        for a in range(0, rows, step):      # tokens are sampled from the policy that gave them, their log-probability is known
            z = torch.empty(min(step, rows - a), vocab, **dev).normal_(0.0, 2.5, generator=gen)
            z = z.to(TORCH[case["dtype"]])
            s["logits"][a:a + step] = z
            z = z.float() / case["temperature"]
            t[a:a + step] = (z - torch.empty_like(z).exponential_(generator=gen).log_()).argmax(1)
            at[a:a + step] = torch.log_softmax(z, 1).gather(1, t[a:a + step, None])[:, 0]
        # how far the policy has moved since the tokens were sampled; by multiples of 1/64 that keep clear of the clip's corners
        # (log 0.8 and log 1.28), where the gradient jumps and the last bit of a ratio would decide
        moved = (torch.randn(rows, generator=gen, **dev) * 0.2).mul(64).floor().add(0.5).div(64)
        s.update(targets=t, old=at - moved, ref=at + 0.1 * torch.randn(rows, generator=gen, **dev), adv=torch.randn(rows, generator=gen, **dev))
        s["weight"] = torch.ones(rows, **dev)
        s["weight"][torch.randperm(rows, generator=gen, **dev)[:case["masked"]]] = 0.0
        s["scale"] = 1.0 / s["weight"].sum()
        return s
    sizes, n = _sizes(case), sum(_sizes(case))
    g = torch.empty(n, dtype=TORCH[case["dtype"]], **dev)
    at, rng = 0, random.Random(case["spec"] + 1)
    for k in sizes:     # the gradients of different tensors have different magnitudes
        g[at:at + k].normal_(0.0, RANKS * 10.0 ** rng.uniform(-4.0, -2.0) * (LOSS_SCALE if case["dtype"] == "f16" else 1.0), generator=gen)
        at += k
    s = {"sizes": sizes, "g": g}
    if case["op"] == "adamw":
        s["p"] = torch.empty(n, **dev).normal_(0.0, 0.02, generator=gen)
        s["m"] = torch.empty(n, **dev).normal_(0.0, 1e-4, generator=gen)
        s["v"] = torch.empty(n, **dev).normal_(0.0, 1e-3, generator=gen).square_().add_(1e-9)
        s["norm"] = torch.full((), 1.75, **dev)
    return s


def prepare(case, seed):
    """The inputs, the buffers that outputs go to, and what names the lists to the library: the handles that a training
    program makes once, when it lays its buckets out (the only thing here that asks for `own`: a plain pass has no use for them)."""
    s = _inputs(case, seed)
    dev = {"device": "cuda"}
    s["case"] = case
    if case["op"] == "loss":
        s["out"] = {k: torch.empty(case["rows"], **dev) for k in ("logp", "loss")} if case["grad"] else {"logp": torch.empty(case["rows"], **dev)}
        if case["grad"]:
            s["out"].update(sums=torch.empty(5, **dev), grad=torch.empty_like(s["logits"]))
    elif case["op"] == "adamw":
        s["copy"] = torch.empty(s["p"].numel(), dtype=TORCH[case["copy"]], **dev) if case["copy"] else None
    else:
        s["norm"] = torch.empty((), **dev)
        if case["op"] == "clip":
            s["clipped"] = torch.empty(s["g"].numel(), dtype=TORCH[case["out"]], **dev)
    if own:
        import paper_2303_06324_amd as dfx
        kinds = {torch.float32: dfx.F32, torch.bfloat16: dfx.BF16, torch.float16: dfx.F16}

        def named(flat):
            at, tensors = flat.data_ptr(), []
            for k in s["sizes"]:
                tensors.append((at, k, kinds[flat.dtype]))
                at += k * flat.element_size()
            return dfx.TensorList(tensors)

        s["dfx"] = dfx
        s["lists"] = {k: named(s[k]) for k in ("g", "p", "m", "v", "copy", "clipped") if s.get(k) is not None}
        if case["op"] == "loss":
            s["kind"] = kinds[s["logits"].dtype]
            s["work"] = torch.empty(dfx.policy_loss_workspace(case["rows"], case["vocab"], s["kind"]), dtype=torch.uint8, **dev)
        elif case["op"] == "adamw":
            s["config"] = dfx.AdamWConfig(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, step=STEP,
                                          grad_scale=_grad_scale(case), max_norm=MAX_NORM)
    return s


# --------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else globals()["_plain_" + state["case"]["op"]](state, state["case"])


def _run_own(s):
    case, dfx, stream = s["case"], s["dfx"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "norm":
        dfx.grad_norm(s["lists"]["g"], s["norm"].data_ptr(), scale=_grad_scale(case), stream=stream)
        return s["norm"]
    if case["op"] == "clip":
        dfx.clip_grad_norm(s["lists"]["g"], s["norm"].data_ptr(), MAX_NORM, out=s["lists"]["clipped"], scale=_grad_scale(case), stream=stream)
        return [s["norm"], s["clipped"]]
    if case["op"] == "adamw":
        x = s["lists"]
        dfx.adamw(x["p"], x["g"], x["m"], x["v"], s["config"], copies=x.get("copy"), norm=s["norm"].data_ptr(), stream=stream)
        return [s["p"], s["m"], s["v"]] + ([s["copy"]] if s["copy"] is not None else [])
    out = s["out"]
    if not case["grad"]:
        dfx.policy_loss(case["rows"], case["vocab"], s["kind"], s["logits"].data_ptr(), s["targets"].data_ptr(), weight=s["weight"].data_ptr(),
                        logp=out["logp"].data_ptr(), inv_temperature=1.0 / case["temperature"],
                        workspace=s["work"].data_ptr(), workspace_bytes=s["work"].numel(), stream=stream)
        return out
    dfx.policy_loss(case["rows"], case["vocab"], s["kind"], s["logits"].data_ptr(), s["targets"].data_ptr(), old_logp=s["old"].data_ptr(),
                    ref_logp=s["ref"].data_ptr(), advantage=s["adv"].data_ptr(), weight=s["weight"].data_ptr(), scale=s["scale"].data_ptr(),
                    logp=out["logp"].data_ptr(), loss=out["loss"].data_ptr(), sums=out["sums"].data_ptr(), grad=out["grad"].data_ptr(),
                    clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL, inv_temperature=1.0 / case["temperature"],
                    workspace=s["work"].data_ptr(), workspace_bytes=s["work"].numel(), stream=stream)
    return out


def _plain_norm(s, case):
    return s["g"].float().square().sum().sqrt() * _grad_scale(case)


def _plain_clip(s, case):
    g = s["g"].float()
    norm = g.square().sum().sqrt() * _grad_scale(case)
    return [norm, (g * ((MAX_NORM / (norm + 1e-6)).clamp(max=1.0) * _grad_scale(case))).to(TORCH[case["out"]])]


def _plain_adamw(s, case):
    p, m, v = s["p"], s["m"], s["v"]
    g = s["g"].float() * ((MAX_NORM / (s["norm"] + 1e-6)).clamp(max=1.0) * _grad_scale(case))
    p.mul_(1.0 - LR * DECAY)
    m.mul_(BETA1).add_(g, alpha=1.0 - BETA1)
    v.mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
    p.addcdiv_(m, (v / (1.0 - BETA2 ** STEP)).sqrt_().add_(EPS), value=-LR / (1.0 - BETA1 ** STEP))
    return [p, m, v] + ([p.to(s["copy"].dtype)] if s["copy"] is not None else [])


def _plain_loss(s, case):
    z, valid = s["logits"].float(), s["weight"] != 0
    if case["temperature"] != 1.0:
        z = z * (1.0 / case["temperature"])
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    logp = (z.gather(1, s["targets"][:, None]) - top - total.log())[:, 0] * valid
    if not case["grad"]:
        return {"logp": logp}
    w, a = s["weight"], s["adv"]
    r = torch.exp(logp - s["old"])
    cut = torch.where(a >= 0, r > 1.0 + CLIP_HIGH, r < 1.0 - CLIP_LOW)
    pg = -a * torch.where(a >= 0, r.clamp(max=1.0 + CLIP_HIGH), r.clamp(min=1.0 - CLIP_LOW))
    d = s["ref"] - logp
    kl = torch.exp(d) - d - 1.0
    loss = w * (pg + KL * kl)
    per = w * s["scale"] * (1.0 / case["temperature"]) * (torch.where(cut, 0.0, -a * r) + KL * (1.0 - torch.exp(d)))
    grad = e.mul_((-per / total[:, 0])[:, None]).scatter_add_(1, s["targets"][:, None], per[:, None])
    return {"logp": logp, "loss": loss, "sums": torch.stack([loss.sum(), (w * pg).sum(), (w * kl).sum(), (w * cut).sum(), w.sum()]),
            "grad": grad.to(s["logits"].dtype)}


# --------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# --------------------------------------------------------------------------------------------
def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "loss":
        rows, vocab, read = case["rows"], case["vocab"], case["rows"] - case["masked"]
        if not case["grad"]:
            return {"bytes": read * vocab * e + rows * 16, "flops": 4 * read * vocab}
        return {"bytes": (read + rows) * vocab * e + rows * 32, "flops": 8 * read * vocab}
    n = case["elems"]
    if case["op"] == "norm":
        return {"bytes": n * e, "flops": 2 * n}
    if case["op"] == "clip":
        return {"bytes": n * (e + BYTES[case["out"]]), "flops": 3 * n}
    return {"bytes": n * (24 + e + (BYTES[case["copy"]] if case["copy"] else 0)), "flops": 14 * n}


def _exact_logp(z, t, c):
    """Logarithm of the softmax of c z in 64 bits at t, and the softmax."""
    z = z.double() * c
    p = torch.softmax(z, 1)
    return z[torch.arange(len(t), device=z.device), t] - torch.logsumexp(z, 1), p


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "loss":
        c, step, logp, grad = 1.0 / case["temperature"], max(1, (1 << 26) // case["vocab"]), [], []
        out = torch.empty(case["rows"], case["vocab"], dtype=torch.float64, device="cuda") if case["grad"] else None
        cols = {k: s[k].double() for k in ("old", "ref", "adv", "weight", "scale")}
        rows = {"loss": [], "pg": [], "kl": [], "cut": []}
        for a in range(0, case["rows"], step):
            at = slice(a, a + step)
            lp, p = _exact_logp(s["logits"][at], s["targets"][at], c)
            on = (cols["weight"][at] != 0).double()
            logp.append(lp * on)
            if out is None:
                continue
            adv, r = cols["adv"][at], torch.exp(lp - cols["old"][at])
            kept = torch.minimum(r * adv, r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv)
            follows = (kept == r * adv).double()
            x = cols["ref"][at] - lp
            rows["pg"].append(-kept * on)
            rows["kl"].append((torch.expm1(x) - x) * on)
            rows["cut"].append((1.0 - follows) * on)
            rows["loss"].append(rows["pg"][-1] + KL * rows["kl"][-1])
            slope = on * cols["weight"][at] * (-adv * r * follows - KL * torch.expm1(x)) * cols["scale"] * c
            p.neg_()
            p[torch.arange(len(lp), device="cuda"), s["targets"][at]] += 1.0
            out[at] = p * slope[:, None]
        if out is None:
            return {"logp": torch.cat(logp)}
        w = cols["weight"]
        per = {k: torch.cat(v) * w for k, v in rows.items()}
        return {"logp": torch.cat(logp), "loss": per["loss"],
                "sums": torch.stack([per["loss"].sum(), per["pg"].sum(), per["kl"].sum(), per["cut"].sum(), w.sum()]), "grad": out}
    scale = _grad_scale(case)
    if case["op"] != "adamw":
        norm = torch.linalg.vector_norm(s["g"].double()) * scale
        return norm if case["op"] == "norm" else [norm, s["g"].double() * (scale * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0))]
    h = s["g"].double() * (scale * min(1.0, MAX_NORM / (float(s["norm"]) + 1e-6)))
    m = BETA1 * s["m"].double() + (1.0 - BETA1) * h
    v = BETA2 * s["v"].double() + (1.0 - BETA2) * h * h
    p = s["p"].double()
    p = p - LR * DECAY * p - LR * (m / (1.0 - BETA1 ** STEP)) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS)
    return [p, m, v] + ([p] if case["copy"] else [])
