"""The worker's operators whose speed counts, each through the public entry
points: layer norm, softmax cross entropy over a vocabulary and distillation
from a teacher's top logits, which end in the fp32 weight gradients that a
worker pushes.

A case is one call sequence of a worker's pass:

  norm          layer norm of hidden states (no gradients: evaluation)
  norm_train    the same, and the backward pass: the gradients of the hidden
                states and, summed over the rows, of weight and bias
  loss          every row's cross entropy, the logits a product of the hidden
                states and the vocabulary's weights that is never kept whole
  loss_train    the same, and the gradients of both
  distill       every row's divergence from a teacher whose ``top`` largest
                logits are known
  distill_train the same, and the gradients of both

``listed`` holds the cases that stand for real use, ``draw`` gives others of
the same ranges: 1 to 16384 rows of 64 to 8192 columns, vocabularies of 100
to 131072, 1 to 128 teacher's logits, three types.  One row in ten of a loss
has no target (padding).  Where ``own`` is false, ``run`` computes the
operators in elementary torch operations in 32 bits.
"""

import math

import torch

own = False  # whether run() makes the framework's calls

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # one token of a model that is being evaluated: the smallest call
        _case("norm_token", "norm", "bf16", 1, 4096),
        # a training batch's hidden states, read and written once
        _case("norm_batch", "norm", "bf16", 16384, 4096),
        # a ragged batch and a width that no vector load divides
        _case("norm_train_odd", "norm_train", "fp16", 2503, 1001),
        # fp32 hidden states: what a worker that keeps everything in the exchange's type has
        _case("norm_train_fp32", "norm_train", "fp32", 4096, 2048),
        # a training batch of a wide model
        _case("norm_train_batch", "norm_train", "bf16", 8192, 8192),
        # a 1000-class layer over 2048 features, a batch of 256, fp32
        _case("loss_train_classes", "loss_train", "fp32", 256, 2048, 1000),
        # a handful of tokens scored against a vocabulary: bound by reading the weights
        _case("loss_few", "loss", "bf16", 5, 4096, 32768),
        # a ragged batch, an odd width and an odd vocabulary
        _case("loss_train_odd", "loss_train", "fp16", 1023, 2047, 50001),
        # an evaluation batch against the largest vocabulary
        _case("loss_large", "loss", "bf16", 4096, 4096, 131072),
        # the ordinary training batch: the largest product
        _case("loss_train_batch", "loss_train", "bf16", 8192, 4096, 32768),
        # scoring a student against stored teacher's logits
        _case("distill_few", "distill", "fp32", 64, 1024, 16384, 64),
        # a student's training batch
        _case("distill_train_batch", "distill_train", "bf16", 4096, 2048, 65536, 32),
    ]


def _case(name, call, kind, rows, cols, vocab=0, top=0):
    return {"name": name, "call": call, "type": kind, "rows": rows, "cols": cols, "vocab": vocab,
            "top": top}


def _spread(rng, low, high):
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    call = rng.choice(["norm", "norm_train", "loss", "loss_train", "loss_train", "distill",
                       "distill_train"])
    kind = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    rows, cols = _spread(rng, 1, 16384), _spread(rng, 64, 8192)
    if rng.random() < 0.6:
        cols = -(-cols // 64) * 64
    vocab = top = 0
    if not call.startswith("norm"):
        vocab = _spread(rng, 100, 131072)
        # no dearer than the listed ones: 2^40 products, fewer where each costs more
        most = 2.0 ** (40 if kind != "fp32" else 37)
        rows = max(1, min(rows, int(most / (vocab * cols))))
        if call.startswith("distill"):
            top = min(_spread(rng, 1, 128), vocab)
    case = _case("", call, kind, rows, cols, vocab, top)
    del case["name"]
    return case


# -------------------------------------------------------------- the inputs

class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.call, kind = case["call"], TYPES[case["type"]]
    n, d, v, top = case["rows"], case["cols"], case["vocab"], case["top"]
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 1000003 + n * 8191 + d)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=DEVICE)

    if s.call.startswith("norm"):
        # a residual stream: rows of unequal scale, off zero
        s.x = (normal(n, d) * (0.5 + 2.0 * uniform(n, 1)) + 0.3 * normal(n, 1)).to(kind)
        s.weight, s.bias = 1.0 + 0.2 * normal(d), 0.1 * normal(d)
        if s.call == "norm_train":
            s.dy = (1e-2 * normal(n, d)).to(kind)
            s.dweight = torch.zeros(d, device=DEVICE)  # a worker's gradients
            s.dbias = torch.zeros(d, device=DEVICE)
        return s
    # the vocabulary's weights, and hidden states that a trained model has
    # turned towards their targets by 0 to 12 units of the logit
    w = normal(v, d) / math.sqrt(d)
    towards = torch.randint(v, (n,), generator=gen, device=DEVICE)
    s.x = (normal(n, d) + 12.0 * uniform(n, 1) * w[towards]).to(kind)
    s.w = w.to(kind)
    live = uniform(n) >= 0.1
    live[0] = True
    if top:
        # the teacher's top entries: the target and others, each once, its logits falling
        s.index = torch.randint(v, (n, 1), generator=gen, device=DEVICE)
        s.index = (s.index + torch.arange(top, device=DEVICE) * max(1, v // top)) % v
        s.index[:, 0] = towards
        twice = s.index[:, 1:] == towards[:, None]
        s.index[:, 1:][twice] = -1
        s.index[~live] = -1
        s.logits = 12.0 * uniform(n, 1) * (1.0 - torch.arange(top, device=DEVICE) / top) + normal(n, top)
        s.temperature = 2.0
    else:
        s.target = torch.where(live, towards, torch.full_like(towards, -100))
    if s.call.endswith("train"):
        # the mean over the rows that count, tokens weighted
        s.dloss = (0.5 + uniform(n)) / live.sum()
        s.dw = torch.zeros(v, d, device=DEVICE)  # a worker's gradients
    return s


def run(s):
    if own:
        return _run_own(s)
    if s.call.startswith("norm"):
        return _plain_norm(s)
    return _plain_loss(s)


# ---------------------------------------------------- the framework's calls

def _run_own(s):
    from paper_1805_07891_amd import layers
    if s.call.startswith("norm"):
        y, mean, rstd = layers.layer_norm(s.x, s.weight, s.bias, EPS)
        if s.call == "norm":
            return {"y": y, "mean": mean, "rstd": rstd}
        dx = layers.layer_norm_grad(s.dy, s.x, s.weight, mean, rstd, s.dweight, s.dbias)
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dweight": s.dweight,
                "dbias": s.dbias}
    if s.call.startswith("loss"):
        loss, lse = layers.vocab_loss(s.x, s.w, s.target)
        if s.call == "loss":
            return {"loss": loss, "lse": lse}
        dx = layers.vocab_loss_grad(s.x, s.w, s.target, lse, s.dloss, s.dw)
    else:
        loss, lse = layers.distill_loss(s.x, s.w, s.index, s.logits, s.temperature)
        if s.call == "distill":
            return {"loss": loss, "lse": lse}
        dx = layers.distill_loss_grad(s.x, s.w, s.index, s.logits, s.temperature, lse, s.dloss,
                                      s.dw)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": s.dw}


# ----------------------------------------------------------- the plain forms

def _plain_norm(s):
    x = s.x.float()
    mean = x.mean(1, keepdim=True)
    off = x - mean
    rstd = 1.0 / torch.sqrt((off * off).mean(1, keepdim=True) + EPS)
    h = off * rstd
    out = {"y": (h * s.weight + s.bias).to(s.x.dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if s.call == "norm_train":
        dy = s.dy.float()
        dh = dy * s.weight
        dx = rstd * (dh - dh.mean(1, keepdim=True) - h * (dh * h).mean(1, keepdim=True))
        out.update(dx=dx.to(s.x.dtype), dweight=(dy * h).sum(0), dbias=dy.sum(0))
    return out


def _plain_loss(s):
    x, w = s.x.float(), s.w.float()
    z = x @ w.t()
    t = 1.0
    if s.call.startswith("distill"):
        t = s.temperature
        z = z / t
    most = z.max(1, keepdim=True).values
    lse = torch.log(torch.exp(z - most).sum(1, keepdim=True)) + most
    if s.call.startswith("loss"):
        live = (s.target >= 0)[:, None]
        index = s.target[:, None].clamp(min=0)
        q = live.float()
        loss = (lse - z.gather(1, index)) * q
    else:
        there = s.index >= 0
        live = there.any(1, keepdim=True)
        index = s.index.clamp(min=0)
        logits = torch.where(there, s.logits / t, -math.inf)
        logits = torch.where(live, logits, 0.0)
        logits = logits - logits.max(1, keepdim=True).values
        logq = logits - torch.log(torch.exp(logits).sum(1, keepdim=True))
        q = torch.where(there, torch.exp(logq), 0.0)
        terms = torch.where(there, q * (logq - z.gather(1, index) + lse), 0.0)
        loss = t * t * terms.sum(1, keepdim=True)
    out = {"loss": loss[:, 0], "lse": lse[:, 0]}
    if s.call.endswith("train"):
        g = torch.exp(z - lse)
        g.scatter_add_(1, index, -q)
        g = torch.where(live, g * (t * s.dloss[:, None]), 0.0)
        out.update(dx=(g @ w).to(s.x.dtype), dw=g.t() @ x)
    return out


# ------------------------------------------------- what a pass cannot avoid

def work(case):
    n, d, v, top, size = case["rows"], case["cols"], case["vocab"], case["top"], BYTES[case["type"]]
    train = case["call"].endswith("train")
    if case["call"].startswith("norm"):
        # x and y, weight and bias, mean and rstd; then dy and dx, and the two gradients
        moved = 2 * n * d * size + 8 * d + 8 * n
        return {"bytes": moved + (2 * n * d * size + 8 * d if train else 0),
                "flops": n * d * (24 if train else 8)}
    # x, w, the targets and the rows' loss and logarithm; then dx, dw and the rows' weights.
    # Two products more for the gradients.
    moved = size * (n + v) * d + n * (12 * top if top else 8) + 8 * n
    return {"bytes": moved + (n * d * size + 4 * v * d + 4 * n if train else 0),
            "flops": 2 * n * v * d * (3 if train else 1)}


# ------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if s.call.startswith("norm"):
        x, weight = s.x.double(), s.weight.double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        h = torch.addcmul(-(mean * rstd)[:, None], x, rstd[:, None])
        out = {"y": torch.addcmul(s.bias.double(), h, weight), "mean": mean, "rstd": rstd}
        if s.call == "norm_train":
            dy = s.dy.double()
            a = torch.mv(dy, weight) / x.shape[1]
            b = torch.mv(dy * h, weight) / x.shape[1]
            out["dx"] = (dy * weight - a[:, None] - b[:, None] * h) * rstd[:, None]
            out["dweight"] = torch.einsum("ij,ij->j", dy, h)
            out["dbias"] = torch.einsum("ij->j", dy)
        return out
    # rows in blocks of about 2^27 logits
    n, v, train = case["rows"], case["vocab"], s.call.endswith("train")
    w, step = s.w.double(), max(1, (1 << 27) // case["vocab"])
    t = s.temperature if case["top"] else 1.0
    loss, lse, dx, dw = [], [], [], torch.zeros_like(w) if train else None
    for i in range(0, n, step):
        x = s.x[i:i + step].double()
        logp = torch.mm(x, w.T) / t
        norm = torch.logsumexp(logp, 1)
        logp -= norm[:, None]
        q = torch.zeros_like(logp)
        if case["top"]:
            for r in range(0, x.shape[0], 512):
                index = s.index[i + r:i + min(r + 512, step)]
                logits = s.logits[i + r:i + min(r + 512, step)].double() / t
                p = torch.softmax(logits.masked_fill(index < 0, -1e300), 1)
                q[r:r + 512].scatter_add_(1, index.clamp(min=0), p.masked_fill(index < 0, 0.0))
        else:
            rows = torch.nonzero(s.target[i:i + step] >= 0)[:, 0]
            q[rows, s.target[i:i + step][rows]] = 1.0
        loss.append(t * t * (torch.xlogy(q, q) - q * logp).sum(1))
        lse.append(norm)
        if train:
            g = (logp.exp_() - q) * (s.dloss[i:i + step].double() * t * (q.sum(1) > 0.5))[:, None]
            dx.append(torch.mm(g, w))
            dw.addmm_(g.T, x)
    out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
    if train:
        out.update(dx=torch.cat(dx), dw=dw)
    return out
