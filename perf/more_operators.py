"""The ends of a training step around the blocks, as cases that can be timed and checked.

Three operators, each through the package's public entry points (``own`` true)
or in elementary torch operations (``own`` false):

* ``loss``     softmax cross entropy of the head's logits h W^T, which are not
               kept, ``ops.head_loss``, and the gradients of h and W,
               ``ops.head_loss_bwd``;
* ``distill``  the same calls with a teacher's top logits: (1 - alpha) times the
               cross entropy plus alpha tau^2 times the divergence from the
               softmax of the teacher's kept logits, both at temperature tau;
* ``norm``     the block's residual sum and RMS norm, ``ops.block_norm``, and its
               gradients, ``ops.block_norm_bwd``.

h and W are bfloat16 or float16, and so are their gradients; losses and the
norm's residual, weight and their gradients are float32, the norm's output is
bfloat16.
"""

import math
import random

import torch

own = False

EPS = 1e-5
DEVICE = "cuda"
IGNORE = -100  # a label of no word: the token has no cross entropy
DTYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16}


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # the next words of 16 running sequences are scored: W is read once
        dict(name="loss 16 tokens", op="loss", tokens=16, vocab=50000, width=2048,
             dtype="bfloat16", masked=0.0, grad=False),
        # the perplexity of one text of 300 tokens, an FP16 head
        dict(name="loss text 300 f16", op="loss", tokens=300, vocab=50000, width=2048,
             dtype="float16", masked=0.0, grad=False),
        # a few tokens of an online update, with the gradients: W is read and written
        dict(name="loss training 64", op="loss", tokens=64, vocab=50000, width=2048,
             dtype="bfloat16", masked=0.0, grad=True),
        # a ragged batch of a smaller model, a third of it prompts and padding without labels
        dict(name="loss training ragged 3001", op="loss", tokens=3001, vocab=32003, width=768,
             dtype="bfloat16", masked=0.33, grad=True),
        # a training batch (8 x 2048 tokens) of the largest model
        dict(name="loss training 8 x 2048", op="loss", tokens=16384, vocab=50000, width=2048,
             dtype="bfloat16", masked=0.0, grad=True),
        # one token against a teacher's 64 best words
        dict(name="distill 1 token", op="distill", tokens=1, vocab=50000, width=2048,
             dtype="bfloat16", masked=0.0, grad=False, top=64, tau=1.0, alpha=0.5),
        # a ragged batch at temperature 2, an FP16 head, tokens without labels or teacher
        dict(name="distill ragged 1000 f16", op="distill", tokens=1000, vocab=32003, width=1000,
             dtype="float16", masked=0.2, grad=True, top=17, tau=2.0, alpha=0.7),
        # the paper's objective (alpha 0.5, temperature 1) on a training batch
        dict(name="distill training 8 x 2048", op="distill", tokens=16384, vocab=50000,
             width=2048, dtype="bfloat16", masked=0.0, grad=True, top=64, tau=1.0, alpha=0.5),
        # the norm of 16 running sequences' tokens
        dict(name="norm 16 tokens", op="norm", tokens=16, width=2048, y=True, grad=False),
        # a short ragged batch, a width that is no power of two, with the gradients
        dict(name="norm training 3001 x 1000", op="norm", tokens=3001, width=1000, y=True,
             grad=True),
        # a training batch of the largest model
        dict(name="norm training 16384", op="norm", tokens=16384, width=2048, y=True, grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    op = rng.choice(("loss", "loss", "distill", "distill", "norm"))
    grad = rng.random() < 0.6
    tokens = _log_int(rng, 1, 16384)
    if op == "norm":
        return dict(op=op, tokens=tokens, width=_log_int(rng, 64, 2048), y=rng.random() < 0.8,
                    grad=grad)
    case = dict(op=op, tokens=tokens, vocab=_log_int(rng, 100, 50000),
                width=8 * _log_int(rng, 8, 256), dtype=rng.choice(("bfloat16", "float16")),
                masked=rng.choice((0.0, 0.0, 0.1, 0.5)), grad=grad)
    if op == "distill":
        case.update(top=min(case["vocab"], _log_int(rng, 1, 64)),
                    tau=rng.choice((1.0, round(rng.uniform(0.5, 4.0), 2))),
                    alpha=round(rng.uniform(0.1, 0.9), 2))
    return case


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std).to(dtype)

    def words(*shape):
        # a text's words: the r-th most frequent one about 1 / r as often as the first
        V = case["vocab"]
        u = torch.rand(*shape, generator=g, device=DEVICE)
        r = torch.exp(u * math.log(V + 1)).long().clamp(1, V) - 1
        return (r * 7919 + 13) % V

    T, D = case["tokens"], case["width"]
    s = dict(case=case)
    if case["op"] == "norm":
        s["residual"] = normal(T, D, std=2.0)
        s["y"] = normal(T, D) if case["y"] else None
        s["w"] = 1.0 + normal(D, std=0.1)
        s["dx"] = normal(T, D, std=0.01, dtype=torch.bfloat16) if case["grad"] else None
        s["dresidual"] = normal(T, D, std=0.01) if case["grad"] else None
        return s
    dt = DTYPES[case["dtype"]]
    s["weight"] = normal(case["vocab"], D, std=2.0 / math.sqrt(D), dtype=dt)
    label = words(T)
    # a model that knows something: the label's logit is raised by 0 to 4 over a spread of 2
    lift = torch.rand(T, 1, generator=g, device=DEVICE)
    s["h"] = (normal(T, D) + lift * s["weight"][label].float()).to(dt)
    none = torch.rand(T, generator=g, device=DEVICE) < case["masked"]
    none[0] = False
    s["targets"] = torch.where(none, IGNORE, label)
    s["ids"] = s["top"] = None
    if case["op"] == "distill":
        K = case["top"]
        s["ids"] = words(T, K)
        s["ids"][:, 0] = label  # (words may come twice)
        s["top"] = torch.sort(normal(T, K, std=3.0), dim=1, descending=True).values
        drop = torch.rand(T, K, generator=g, device=DEVICE) < 0.5 * case["masked"]
        s["ids"][drop | (none & (label % 2 == 0))[:, None]] = -1  # places that hold no word
    # a mean over the batch; an FP16 model's loss is scaled
    scale = 4096.0 if dt == torch.float16 else 1.0
    s["dloss"] = torch.full((T,), scale / T, device=DEVICE) if case["grad"] else None
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return _plain_norm(s) if op == "norm" else _plain_loss(s, op)


def _own(s, op):
    from paper_2606_18114_amd import ops
    if op == "norm":
        x, r = ops.block_norm(s["residual"], s["y"], s["w"], EPS)
        if s["dx"] is None:
            return dict(x=x, residual=r)
        dr, dw = ops.block_norm_bwd(r, s["w"], s["dx"], s["dresidual"], EPS)
        return dict(x=x, residual=r, dresidual=dr, dw=dw)
    teach = {}
    if op == "distill":
        teach = dict(teacher_ids=s["ids"], alpha=s["case"]["alpha"], temperature=s["case"]["tau"])
    loss, stats = ops.head_loss(s["h"], s["weight"], s["targets"], teacher_logits=s["top"],
                                **teach)
    if s["dloss"] is None:
        return dict(loss=loss)
    dh, dw = ops.head_loss_bwd(s["h"], s["weight"], s["targets"], stats, s["dloss"], **teach)
    return dict(loss=loss, dh=dh, dw=dw)


def _plain_norm(s):
    r = s["residual"] if s["y"] is None else s["residual"] + s["y"]
    rho = 1.0 / torch.sqrt((r * r).mean(-1, keepdim=True) + EPS)
    x = (r * rho * s["w"]).to(torch.bfloat16)
    if s["dx"] is None:
        return dict(x=x, residual=r)
    dx = s["dx"].float()
    a = dx * s["w"]
    dr = s["dresidual"] + a * rho - r * rho ** 3 * (a * r).mean(-1, keepdim=True)
    return dict(x=x, residual=r, dresidual=dr, dw=(dx * r * rho).sum(0))


def _log_softmax(z):
    z = z - z.amax(-1, keepdim=True)
    return z - torch.log(torch.exp(z).sum(-1, keepdim=True))


def _plain_loss(s, op):
    c = s["case"]
    h, w = s["h"].float(), s["weight"].float()
    z = h @ w.t()
    has = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    logp = _log_softmax(z)
    loss = torch.where(has, -logp.gather(1, at)[:, 0], 0.0)
    grad = s["dloss"] is not None
    if grad:
        dz = torch.exp(logp)
        dz.scatter_add_(1, at, torch.full_like(loss, -1.0)[:, None])
        dz *= has[:, None]
    if op == "distill":
        alpha, tau = c["alpha"], c["tau"]
        kept = s["ids"] >= 0
        some = kept.any(1)
        ids = s["ids"].clamp(min=0)
        logq = _log_softmax(torch.where(kept, s["top"] / tau, -1e30))
        q = torch.where(kept & some[:, None], torch.exp(logq), 0.0)
        logs = logp if tau == 1.0 else _log_softmax(z / tau)
        kl = (q * (logq - logs.gather(1, ids))).sum(1)
        loss = (1.0 - alpha) * loss + alpha * tau ** 2 * kl
        if grad:
            ds = torch.exp(logs) * some[:, None]
            ds.scatter_add_(1, ids, -q)
            dz = (1.0 - alpha) * dz + alpha * tau * ds
    if not grad:
        return dict(loss=loss)
    dz *= s["dloss"][:, None]
    return dict(loss=loss, dh=(dz @ w).to(s["h"].dtype), dw=(dz.t() @ h).to(s["h"].dtype))


# ---------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once, the products with the logits, and of their gradient, once."""
    T, D, grad = case["tokens"], case["width"], case["grad"]
    if case["op"] == "norm":
        fwd = T * D * (4 + 2 + (8 if case["y"] else 0)) + 4 * D
        bwd = T * D * (2 + 4 + 4) + 4 * D
        return dict(bytes=fwd + (bwd if grad else 0), flops=T * D * (6 + (12 if grad else 0)))
    V, K = case["vocab"], case.get("top", 0)
    n = T * (1.0 - case["masked"]) if case["op"] == "loss" else T
    inputs = 2 * (T + V) * D + 8 * T + 12 * T * K
    flops = 2 * n * V * D + 4 * n * V
    if not grad:
        return dict(bytes=inputs + 4 * T, flops=flops)
    return dict(bytes=inputs + 8 * T + 2 * (T + V) * D, flops=flops + 4 * n * V * D)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"] == "norm" else _exact_loss(s, case)


def _exact_norm(s):
    r = s["residual"].double()
    if s["y"] is not None:
        r = r + s["y"].double()
    var = r.pow(2).mean(-1, keepdim=True) + EPS
    unit = r / var.sqrt()
    out = dict(x=unit * s["w"].double(), residual=r)
    if s["dx"] is not None:
        dx = s["dx"].double()
        du = dx * s["w"].double()
        out["dresidual"] = s["dresidual"].double() \
            + (du - unit * (du * unit).mean(-1, keepdim=True)) / var.sqrt()
        out["dw"] = (dx * unit).sum(0)
    return out


def _exact_loss(s, case, chunk=2048):
    """Runs of tokens, one after another."""
    w = s["weight"].double()
    V = w.shape[0]
    alpha, tau = case.get("alpha", 0.0), case.get("tau", 1.0)
    losses, dhs, dw = [], [], torch.zeros_like(w)
    for lo in range(0, case["tokens"], chunk):
        rows = slice(lo, lo + chunk)
        h, label = s["h"][rows].double(), s["targets"][rows]
        z = h @ w.t()
        i = torch.nonzero(label >= 0)[:, 0]
        y = label[i]
        lse = torch.logsumexp(z, 1)
        loss = torch.zeros(len(h), dtype=torch.float64, device=DEVICE)
        loss[i] = (1.0 - alpha) * (lse[i] - z[i, y])
        dz = torch.zeros_like(z)
        dz[i] = (1.0 - alpha) * torch.softmax(z[i], 1)
        dz[i, y] -= 1.0 - alpha
        if s["ids"] is not None:
            ids, top = s["ids"][rows], s["top"][rows].double() / tau
            t, k = torch.nonzero(ids >= 0, as_tuple=True)
            v = ids[t, k]
            norm = torch.logsumexp(top.masked_fill(ids < 0, -math.inf), 1)
            logq = top[t, k] - norm[t]
            logs = z[t, v] / tau - torch.logsumexp(z / tau, 1)[t]
            loss.index_add_(0, t, alpha * tau * tau * torch.exp(logq) * (logq - logs))
            some = torch.unique(t)
            dz[some] += alpha * tau * torch.softmax(z[some] / tau, 1)
            dz.view(-1).index_add_(0, t * V + v, -alpha * tau * torch.exp(logq))
        losses.append(loss)
        if s["dloss"] is not None:
            dz *= s["dloss"][rows, None].double()
            dhs.append(dz @ w)
            dw += dz.t() @ h
    if s["dloss"] is None:
        return dict(loss=torch.cat(losses))
    return dict(loss=torch.cat(losses), dh=torch.cat(dhs), dw=dw)
