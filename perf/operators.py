"""The sequence forms of the Mamba-2 mixer and the embedding, as cases that can be timed and checked.

Four operators, each through the package's public entry points (``own`` true)
or in elementary torch operations (``own`` false):

* ``conv``   the short causal convolution with SiLU over packed sequences,
             ``ops.mixer_conv``, and its gradients, ``ops.mixer_conv_bwd``;
* ``scan``   the selective state space scan over packed sequences,
             ``ops.mixer_scan``, and its gradients, ``ops.mixer_scan_bwd``;
* ``norm``   the gated RMS norm before out_proj, ``ops.mixer_norm``, and its
             gradients, ``ops.mixer_norm_bwd``;
* ``embed``  rows of an embedding, ``ops.embed``, and the gradient of its
             weight, ``ops.embed_bwd``.

A layer has ``heads`` heads of 64 channels, 128 states and one group of B and
C; in_proj's output ``zxbcdt`` is [tokens, z | x | B | C | dt] in bfloat16 or
float32.  The convolution's output u, the scan's output y, the norm's output
and the gradients of u and y are bfloat16, decode states float16, parameters
and their gradients float32.
"""

import math
import random

import torch

own = False

P, N, TAPS = 64, 128, 4
EPS = 1e-5
DEVICE = "cuda"
DTYPES = {"bfloat16": torch.bfloat16, "float32": torch.float32, "float16": torch.float16}


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # 16 running sequences that each take one token through the prompt path
        dict(name="conv 16 x 1 token", op="conv", tokens=16, seqs=16, ragged=False, heads=64,
             dtype="bfloat16", state=True, grad=False),
        # a training batch (8 x 2048 tokens) of the largest layer, with the gradients
        dict(name="conv training 8 x 2048", op="conv", tokens=16384, seqs=8, ragged=False,
             heads=64, dtype="bfloat16", state=False, grad=True),
        # prompts of many lengths in float32, as in_proj writes them by default
        dict(name="conv ragged 3001 f32", op="conv", tokens=3001, seqs=7, ragged=True, heads=24,
             dtype="float32", state=True, grad=False),
        # 16 running sequences, one token each: the shortest scan
        dict(name="scan 16 x 1 token", op="scan", tokens=16, seqs=16, ragged=False, heads=64,
             dtype="bfloat16", state=True, grad=False),
        # a short prompt before decoding
        dict(name="scan prompt 300", op="scan", tokens=300, seqs=1, ragged=False, heads=64,
             dtype="bfloat16", state=True, grad=False),
        # one long prompt: few rows, a long axis
        dict(name="scan prompt 16384", op="scan", tokens=16384, seqs=1, ragged=False, heads=64,
             dtype="bfloat16", state=True, grad=False),
        # a ragged batch of a smaller model with its gradients, float32 in_proj output
        dict(name="scan training ragged f32", op="scan", tokens=3001, seqs=7, ragged=True,
             heads=24, dtype="float32", state=False, grad=True),
        # a training batch of the largest layer
        dict(name="scan training 8 x 2048", op="scan", tokens=16384, seqs=8, ragged=False,
             heads=64, dtype="bfloat16", state=False, grad=True),
        # the norm of a short prompt
        dict(name="norm prompt 300", op="norm", tokens=300, heads=64, dtype="bfloat16",
             grad=False),
        # the norm of a training batch, with the gradients
        dict(name="norm training 16384", op="norm", tokens=16384, heads=64, dtype="bfloat16",
             grad=True),
        # the tokens of a prompt
        dict(name="embed 300", op="embed", tokens=300, vocab=50000, width=2048, dtype="bfloat16",
             grad=False),
        # the embedding's gradient in a training step; few tokens make up most of a text
        dict(name="embed training 16384", op="embed", tokens=16384, vocab=50000, width=2048,
             dtype="float32", grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    op = rng.choice(("conv", "scan", "scan", "scan", "norm", "embed"))
    grad = rng.random() < 0.5
    dtype = rng.choice(("bfloat16", "bfloat16", "float32"))
    tokens = _log_int(rng, 1, 16384)
    if op == "embed":
        return dict(op=op, tokens=tokens, vocab=_log_int(rng, 100, 50000),
                    width=8 * _log_int(rng, 8, 256),
                    dtype=rng.choice(("float32", "bfloat16", "float16")), grad=grad)
    heads = rng.choice((64, 64, 24, rng.randint(1, 64)))
    if op == "norm":
        return dict(op=op, tokens=tokens, heads=heads, dtype=dtype, grad=grad)
    return dict(op=op, tokens=tokens, seqs=min(tokens, _log_int(rng, 1, 16)),
                ragged=rng.random() < 0.7, heads=heads, dtype=dtype,
                state=not grad and rng.random() < 0.8, grad=grad)


def _offsets(case):
    """Where the sequences begin, and the end; a ragged batch has an empty one."""
    T, S = case["tokens"], case["seqs"]
    if not case["ragged"]:
        return [T * i // S for i in range(S + 1)]
    rng = random.Random(1000 * T + S)
    cuts = sorted(int(T * rng.random() ** 1.5) for _ in range(S - 1))
    if S > 2:
        cuts[1] = cuts[0]
    return [0] + cuts + [T]


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return lo + (hi - lo) * torch.rand(*shape, generator=g, device=DEVICE)

    T = case["tokens"]
    s = dict(case=case)
    if case["op"] == "embed":
        V, D = case["vocab"], case["width"]
        # a text's tokens: the r-th most frequent one about 1 / r as often as the first
        r = torch.exp(uniform(T) * math.log(V + 1)).long().clamp(1, V) - 1
        s["ids"] = (r * 7919 + 13) % V
        s["weight"] = normal(V, D, std=0.02, dtype=dt)
        s["scale"] = 1.5
        s["de"] = normal(T, D, std=0.01) if case["grad"] else None
        return s
    H = case["heads"]
    d = H * P
    cd = d + 2 * N
    s["zx"] = normal(T, d + cd + H, dtype=dt)
    if case["op"] == "norm":
        s["y"] = normal(T, d, dtype=torch.bfloat16)
        s["norm_w"] = 1.0 + normal(d, std=0.1)
        s["dout"] = normal(T, d, std=0.01, dtype=torch.bfloat16) if case["grad"] else None
        return s
    s["offs"] = _offsets(case)
    s["offsets"] = torch.tensor(s["offs"], dtype=torch.int32, device=DEVICE)
    S = case["seqs"]
    if case["op"] == "conv":
        s["conv_w"] = uniform(cd, TAPS, lo=-0.5, hi=0.5)
        s["conv_b"] = uniform(cd, lo=-0.5, hi=0.5)
        s["ring"] = normal(S, cd, TAPS, dtype=torch.float16) if case["state"] else None
        s["slot"] = seed % TAPS  # where the ring's oldest input lies
        s["pos"] = torch.full((1,), s["slot"], dtype=torch.int32, device=DEVICE)
        s["du"] = normal(T, cd, std=0.01, dtype=torch.bfloat16) if case["grad"] else None
        return s
    u = normal(T, cd)
    s["u"] = (u * torch.sigmoid(u)).to(torch.bfloat16)
    step = torch.exp(uniform(H, lo=math.log(1e-3), hi=math.log(1e-1)))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["A_log"] = torch.log(uniform(H, lo=1.0, hi=16.0))
    s["D"] = 1.0 + normal(H, std=0.1)
    s["ssm"] = normal(S, H, P, N, std=0.5, dtype=torch.float16) if case["state"] else None
    s["dy"] = normal(T, d, std=0.01, dtype=torch.bfloat16) if case["grad"] else None
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op, grad = s["case"]["op"], s["case"]["grad"]
    if own:
        return _own(s, op, grad)
    if op == "embed":
        return _plain_embed(s, grad)
    with torch.set_grad_enabled(grad):
        return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[op](s, grad)


def _own(s, op, grad):
    from paper_2606_18114_amd import ops
    if op == "embed":
        if grad:
            return dict(dw=ops.embed_bwd(s["ids"], s["de"], s["case"]["vocab"], s["scale"]))
        return dict(e=ops.embed(s["ids"], s["weight"], s["scale"]))
    zx, H = s["zx"], s["case"]["heads"]
    d = H * P
    dzx = torch.empty_like(zx) if grad else None
    if op == "norm":
        out = ops.mixer_norm(s["y"], zx, s["norm_w"], EPS)
        if not grad:
            return dict(out=out)
        dy, dw = ops.mixer_norm_bwd(s["y"], zx, s["norm_w"], s["dout"], dzx, EPS)
        return dict(out=out, dy=dy, dz=dzx[:, :d], dnorm_w=dw)
    if op == "conv":
        ring = s["ring"]
        new = None if ring is None else torch.empty_like(ring)
        u = ops.mixer_conv(zx, s["conv_w"], s["conv_b"], s["offsets"], ring,
                           None if ring is None else s["pos"], conv_out=new)
        if not grad:
            return dict(u=u) if ring is None else dict(u=u, ring=new)
        dw, db = ops.mixer_conv_bwd(zx, s["conv_w"], s["conv_b"], s["du"], dzx, s["offsets"])
        return dict(u=u, dxbc=dzx[:, d:-H], dconv_w=dw, dconv_b=db)
    new = None if s["ssm"] is None else torch.empty_like(s["ssm"])
    y = ops.mixer_scan(s["u"], zx, s["dt_bias"], s["A_log"], s["D"], s["offsets"], s["ssm"],
                       ssm_out=new)
    if not grad:
        return dict(y=y) if new is None else dict(y=y, ssm=new)
    du, dbias, dalog, dd = ops.mixer_scan_bwd(s["u"], zx, s["dt_bias"], s["A_log"], s["D"],
                                              s["dy"], dzx, s["offsets"])
    return dict(y=y, du=du, ddt=dzx[:, -H:], ddt_bias=dbias, dA_log=dalog, dD=dd)


def _leaf(t, grad):
    return t.detach().float().clone().requires_grad_(True) if grad else t.float()


def _plain_embed(s, grad):
    if not grad:
        return dict(e=s["weight"][s["ids"]].float() * s["scale"])
    dw = torch.zeros(s["case"]["vocab"], s["case"]["width"], device=DEVICE)
    return dict(dw=dw.index_add_(0, s["ids"], s["de"] * s["scale"]))


def _plain_norm(s, grad):
    d = s["case"]["heads"] * P
    y, z, w = (_leaf(t, grad) for t in (s["y"], s["zx"][:, :d], s["norm_w"]))
    g = y * (z / (1.0 + torch.exp(-z)))
    out = g / torch.sqrt((g * g).mean(-1, keepdim=True) + EPS) * w
    if not grad:
        return dict(out=out.to(torch.bfloat16))
    dy, dz, dw = torch.autograd.grad(out, (y, z, w), s["dout"].float())
    return dict(out=out.detach().to(torch.bfloat16), dy=dy.to(torch.bfloat16),
                dz=dz.to(s["zx"].dtype), dnorm_w=dw)


def _positions(s):
    """Of every token its sequence and its place in it; of every sequence its length."""
    off = torch.as_tensor(s["offs"], device=DEVICE)
    length = off[1:] - off[:-1]
    seq = torch.repeat_interleave(torch.arange(len(length), device=DEVICE), length)
    return seq, torch.arange(len(seq), device=DEVICE) - off[seq], length, off


def _plain_conv(s, grad):
    H, T = s["case"]["heads"], s["case"]["tokens"]
    d = H * P
    cd = d + 2 * N
    x, w, b = (_leaf(t, grad) for t in (s["zx"][:, d:d + cd], s["conv_w"], s["conv_b"]))
    seq, at, length, off = _positions(s)
    if s["ring"] is None:
        past = torch.zeros(len(length), TAPS, cd, device=DEVICE)
    else:  # the j-th oldest input of a sequence lies in slot (pos + j) % 4
        past = torch.roll(s["ring"].float(), -s["slot"], dims=2).transpose(1, 2)
    # the inputs of all sequences, each after its past: token t is row t + 4 (seq + 1)
    row = torch.arange(T, device=DEVICE) + TAPS * (seq + 1)
    before = (off[:-1] + TAPS * torch.arange(len(length), device=DEVICE))[:, None] \
        + torch.arange(TAPS, device=DEVICE)
    whole = torch.zeros(T + TAPS * len(length), cd, device=DEVICE)
    whole = whole.index_put((before.reshape(-1),), past.reshape(-1, cd)).index_put((row,), x)
    a = b + w[:, 0] * whole[row - 3] + w[:, 1] * whole[row - 2] + w[:, 2] * whole[row - 1] \
        + w[:, 3] * whole[row]
    u = a / (1.0 + torch.exp(-a))
    if grad:
        dx, dw, db = torch.autograd.grad(u, (x, w, b), s["du"].float())
        return dict(u=u.detach().to(torch.bfloat16), dxbc=dx.to(s["zx"].dtype), dconv_w=dw,
                    dconv_b=db)
    if s["ring"] is None:
        return dict(u=u.to(torch.bfloat16))
    last = whole[before + length[:, None]].transpose(1, 2)  # a sequence's last four inputs
    return dict(u=u.to(torch.bfloat16),
                ring=torch.roll(last, s["slot"], dims=2).to(torch.float16).contiguous())


def _plain_scan(s, grad, Q=64):
    """Chunks of Q tokens: products inside a chunk, the states between chunks
    by the products of their decays (exponents in 64 bits)."""
    H = s["case"]["heads"]
    d = H * P
    u, dt, bias, alog, dskip = (_leaf(t, grad) for t in (
        s["u"], s["zx"][:, -H:], s["dt_bias"], s["A_log"], s["D"]))
    seq, at, length, off = _positions(s)
    S = len(length)
    C = -(-max(1, int(max(b - a for a, b in zip(s["offs"], s["offs"][1:])))) // Q)
    place = torch.arange(C * Q, device=DEVICE)[None, :].expand(S, -1)
    mask = place < length[:, None]
    src = (off[:-1, None] + place).clamp(max=u.shape[0] - 1)
    xbc = (u[src] * mask[..., None]).reshape(S, C, Q, -1)
    x = xbc[..., :d].reshape(S, C, Q, H, P).transpose(2, 3)            # [S, C, H, Q, P]
    Bm, Cm = xbc[..., None, :, d:d + N], xbc[..., None, :, d + N:]     # [S, C, 1, Q, N]
    raw = dt + bias
    step = torch.where(raw > 20.0, raw, torch.log1p(torch.exp(raw.clamp(max=20.0))))
    step = (step[src] * mask[..., None]).reshape(S, C, Q, H).transpose(2, 3)  # [S, C, H, Q]
    cum = -torch.cumsum(step.double() * torch.exp(alog.double())[:, None], -1)
    low = torch.ones(Q, Q, dtype=torch.bool, device=DEVICE).tril()
    diff = (cum[..., :, None] - cum[..., None, :]).masked_fill(~low, -math.inf)
    inner = (Cm @ Bm.transpose(-1, -2)) * torch.exp(diff).float() * step[..., None, :]
    y = inner @ x
    # states at the chunks' ends, from each chunk alone; the initial one first
    w = step * torch.exp(cum[..., -1:] - cum).float()
    part = (x * w[..., None]).transpose(-1, -2) @ Bm                   # [S, C, H, P, N]
    first = torch.zeros(S, 1, H, P, N, device=DEVICE) if s["ssm"] is None \
        else s["ssm"].float()[:, None]
    part = torch.cat([first, part], 1).transpose(1, 2).reshape(S, H, C + 1, P * N)
    total = torch.cumsum(torch.nn.functional.pad(cum[..., -1], (0, 0, 1, 0)), 1).transpose(1, 2)
    low = torch.ones(C + 1, C + 1, dtype=torch.bool, device=DEVICE).tril()
    gap = (total[..., :, None] - total[..., None, :]).masked_fill(~low, -math.inf)
    state = (torch.exp(gap).float() @ part).reshape(S, H, C + 1, P, N).transpose(1, 2)
    y = y + torch.exp(cum).float()[..., None] * (Cm @ state[:, :-1].transpose(-1, -2))
    y = y + dskip[:, None, None] * x
    y = y.transpose(2, 3).reshape(S, C * Q, d)[mask]
    if grad:
        du, ddt, dbias, dalog, dd = torch.autograd.grad(y, (u, dt, bias, alog, dskip),
                                                        s["dy"].float())
        return dict(y=y.detach().to(torch.bfloat16), du=du.to(torch.bfloat16),
                    ddt=ddt.to(s["zx"].dtype), ddt_bias=dbias, dA_log=dalog, dD=dd)
    y = y.to(torch.bfloat16)
    return dict(y=y) if s["ssm"] is None else dict(
        y=y, ssm=state[:, -1].to(torch.float16).contiguous())


# ---------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once, the recurrence's own products."""
    T, grad = case["tokens"], case["grad"]
    if case["op"] == "embed":
        V, D = case["vocab"], case["width"]
        if grad:
            return dict(bytes=8 * T + 4 * T * D + 4 * V * D, flops=2 * T * D)
        es = 4 if case["dtype"] == "float32" else 2
        return dict(bytes=8 * T + (es + 4) * T * D, flops=T * D)
    H = case["heads"]
    es = 4 if case["dtype"] == "float32" else 2
    d = H * P
    cd = d + 2 * N
    if case["op"] == "norm":
        fwd = T * d * (2 + es + 2) + 4 * d
        bwd = T * d * (2 + es + 2 + 2 + es) + 8 * d
        return dict(bytes=fwd + (bwd if grad else 0), flops=T * d * (8 + (20 if grad else 0)))
    S = case["seqs"]
    if case["op"] == "conv":
        fwd = T * cd * (es + 2) + 20 * cd + (16 * S * cd if case["state"] else 0)
        bwd = T * cd * (es + 2 + es) + 40 * cd
        return dict(bytes=fwd + (bwd if grad else 0), flops=T * cd * (12 + (30 if grad else 0)))
    fwd = T * (2 * cd + es * H + 2 * d) + (4 * S * d * N if case["state"] else 0)
    bwd = T * (2 * cd + es * H + 2 * d + 2 * cd + es * H)
    # per token and head: the state's update and the read-out, 2 P N each; backward
    # the state once more, the adjoint's update, dx, dB, dC and the decay's gradient
    return dict(bytes=fwd + (bwd if grad else 0),
                flops=T * H * P * N * (4 + (12 if grad else 0)))


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm,
            "embed": _exact_embed}[case["op"]](s)


def _exact_embed(s):
    if s["de"] is None:
        return dict(e=s["weight"].double()[s["ids"]] * s["scale"])
    dw = torch.zeros(s["weight"].shape, dtype=torch.float64, device=DEVICE)
    return dict(dw=dw.index_add_(0, s["ids"], s["de"].double()) * s["scale"])


def _exact_norm(s):
    d = s["case"]["heads"] * P
    y, z, w = s["y"].double(), s["zx"][:, :d].double(), s["norm_w"].double()
    sig = torch.sigmoid(z)
    g = y * z * sig
    r = ((g * g).mean(-1, keepdim=True) + EPS).rsqrt()
    if s["dout"] is None:
        return dict(out=g * r * w)
    do = s["dout"].double()
    a = do * w
    dg = r * a - g * r ** 3 * (a * g).mean(-1, keepdim=True)
    return dict(out=g * r * w, dy=dg * z * sig, dz=dg * y * sig * (1 + z * (1 - sig)),
                dnorm_w=(do * g * r).sum(0))


def _exact_conv(s):
    d = s["case"]["heads"] * P
    cd = d + 2 * N
    x = s["zx"][:, d:d + cd].double()
    w, b = s["conv_w"].double(), s["conv_b"].double()
    u, ring = torch.empty_like(x), None if s["ring"] is None else s["ring"].double()
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(b)
    for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
        past = torch.zeros(cd, TAPS, dtype=torch.float64, device=DEVICE)
        if ring is not None:
            for j in range(TAPS):
                past[:, j] = ring[i, :, (s["slot"] + j) % TAPS]
        line = torch.cat([past, x[lo:hi].T], 1)
        n = hi - lo
        a = b[:, None] + sum(w[:, j:j + 1] * line[:, 1 + j:1 + j + n] for j in range(TAPS))
        sig = torch.sigmoid(a)
        u[lo:hi] = (a * sig).T
        if s["du"] is not None:
            da = s["du"][lo:hi].double().T * sig * (1 + a * (1 - sig))
            db += da.sum(1)
            for j in range(TAPS):
                dw[:, j] += (da * line[:, 1 + j:1 + j + n]).sum(1)
                back = TAPS - 1 - j  # tap j reads the input `back` tokens before
                if n > back:
                    dx[lo:hi - back] += (w[:, j:j + 1] * da[:, back:]).T
        if ring is not None and n:
            for j in range(TAPS):
                ring[i, :, (s["slot"] + j) % TAPS] = line[:, n + j]
    if s["du"] is not None:
        return dict(u=u, dxbc=dx, dconv_w=dw, dconv_b=db)
    return dict(u=u) if ring is None else dict(u=u, ring=ring)


def _exact_scan(s):
    """The recurrence token by token; backward its adjoint, on states kept
    every 64 tokens and computed again between them."""
    H = s["case"]["heads"]
    d = H * P
    S, L = len(s["offs"]) - 1, max(b - a for a, b in zip(s["offs"], s["offs"][1:]))
    f64 = dict(dtype=torch.float64, device=DEVICE)

    def rows(t):  # [tokens, n] -> [L, S, n], zeros behind a sequence's end
        out = torch.zeros(L, S, t.shape[1], **f64)
        for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:])):
            out[:hi - lo, i] = t[lo:hi].double()
        return out

    def packed(t):
        return torch.cat([t[:hi - lo, i].flatten(1)
                          for i, (lo, hi) in enumerate(zip(s["offs"], s["offs"][1:]))])

    valid = rows(torch.ones(s["u"].shape[0], 1, device=DEVICE))
    u = rows(s["u"])
    x, Bm, Cm = u[..., :d].reshape(L, S, H, P), u[..., d:d + N], u[..., d + N:]
    raw = rows(s["zx"][:, -H:]) + s["dt_bias"].double()
    step = torch.nn.functional.softplus(raw, threshold=200.0) * valid
    rate = torch.exp(s["A_log"].double())
    decay = torch.exp(-step * rate)
    D = s["D"].double()
    xb = x * step[..., None]
    state = torch.zeros(S, H, P, N, **f64) if s["ssm"] is None else s["ssm"].double()
    y, kept = torch.empty(L, S, H, P, **f64), []

    def forward(state, t):
        return state * decay[t][..., None, None] + xb[t][..., None] * Bm[t][:, None, None, :]

    for t in range(L):
        if s["dy"] is not None and t % 64 == 0:
            kept.append(state)
        state = forward(state, t)
        y[t] = (state @ Cm[t][:, None, :, None])[..., 0]
    y += D[:, None] * x
    if s["dy"] is None:
        return dict(y=packed(y)) if s["ssm"] is None else dict(y=packed(y), ssm=state)
    dy = rows(s["dy"]).reshape(L, S, H, P)
    dx, dB, dC = torch.empty_like(x), torch.empty_like(Bm), torch.empty_like(Cm)
    dstep, dlog = torch.empty_like(step), torch.empty_like(step)
    adj = torch.zeros(S, H, P, N, **f64)
    for block in range(len(kept) - 1, -1, -1):
        lo, hi = 64 * block, min(L, 64 * block + 64)
        states = [kept[block]]
        for t in range(lo, hi):
            states.append(forward(states[-1], t))
        for t in range(hi - 1, lo - 1, -1):
            now, before = states[t - lo + 1], states[t - lo]
            adj = adj + dy[t][..., None] * Cm[t][:, None, None, :]
            dC[t] = (dy[t].reshape(S, 1, d) @ now.reshape(S, d, N))[:, 0]
            dB[t] = (xb[t].reshape(S, 1, d) @ adj.reshape(S, d, N))[:, 0]
            dxb = (adj @ Bm[t][:, None, :, None])[..., 0]
            dx[t] = dxb * step[t][..., None] + D[:, None] * dy[t]
            dstep[t] = (dxb * x[t]).sum(-1)
            adj = adj * decay[t][..., None, None]
            dlog[t] = (adj * before).sum((-1, -2))
    dstep = dstep - rate * dlog
    ddt = dstep * torch.sigmoid(raw) * valid
    return dict(y=packed(y), du=torch.cat([packed(dx), packed(dB), packed(dC)], 1),
                ddt=packed(ddt), ddt_bias=ddt.sum((0, 1)),
                dA_log=(-step * rate * dlog).sum((0, 1)), dD=(dy * x).sum((0, 1, 3)))
