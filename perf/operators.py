"""The operators that train a softmax head over embedding rows, as they are timed.

Three kinds of call, each through the package's public entry points:

  norm    layer_norm over rows, and layer_norm_backward with the reduction of
          the two weight gradients;
  loss    SoftmaxLoss.loss: softmax cross entropy against every row of an
          output table, without keeping the logits; and SoftmaxLoss.grad, its
          gradient with respect to rows, table and bias;
  adamw   AdamW.step over a list of tensors, with states in 32 bits or in 8.

Sizes are those of the workloads in synth/gen.py: vocabularies of 10,000 to a
million nodes or the blocks of a block model, rows of 32 to 256 values, batches
from one row to a hundred thousand.  With `own` false the same is computed in
elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256  # elements that share the two scales of a state in 8 bits


# --------------------------------------------------------------------------- #
# Cases
# --------------------------------------------------------------------------- #
def listed():
    return [
        # one small batch of the tiny workload normalised before the head: latency
        dict(name="norm_small", kind="norm", n=1024, dim=32, type="f32", grad=False, pad=0),
        # training on a medium batch, half-width rows
        dict(name="norm_medium", kind="norm", n=65_536, dim=128, type="bf16", grad=True, pad=0),
        # training on a whole batch of wide rows, columns of a wider buffer
        dict(name="norm_large", kind="norm", n=262_144, dim=256, type="f32", grad=True, pad=64),
        # serving: one row's distribution over a million nodes
        dict(name="loss_one", kind="loss", n=1, classes=1_000_000, dim=128, type="f32",
             grad=False, bias=False, weights=False, unlabelled=0.0, masked=0.0, pad=0),
        # a training step on the tiny workload: every node is a class
        dict(name="loss_tiny", kind="loss", n=1024, classes=10_000, dim=32, type="f32",
             grad=True, bias=True, weights=False, unlabelled=0.0, masked=0.0, pad=0),
        # validation: the exact loss of a held-out batch over the medium vocabulary
        dict(name="loss_heldout", kind="loss", n=4096, classes=1_000_000, dim=128, type="bf16",
             grad=False, bias=False, weights=True, unlabelled=0.0, masked=0.0, pad=0),
        # training with the exact softmax over the medium vocabulary
        dict(name="loss_nodes", kind="loss", n=4096, classes=1_000_000, dim=128, type="bf16",
             grad=True, bias=True, weights=True, unlabelled=0.0, masked=0.0, pad=0),
        # wide rows in 32 bits, ragged sizes, some nodes taken out of the vocabulary
        dict(name="loss_wide", kind="loss", n=3001, classes=50_021, dim=256, type="f32",
             grad=True, bias=True, weights=True, unlabelled=0.0, masked=0.02, pad=32),
        # a classifier of the nodes' blocks: few classes, many rows, some without a label
        dict(name="loss_blocks", kind="loss", n=100_003, classes=1000, dim=128, type="bf16",
             grad=True, bias=True, weights=False, unlabelled=0.1, masked=0.0, pad=0),
        # the optimiser on a small head: four tensors, latency
        dict(name="adamw_head", kind="adamw", sizes="32,32,320,10", params="f32", grads="f32",
             states="f32"),
        # a vocabulary table and a head, everything in 32 bits
        dict(name="adamw_table", kind="adamw", sizes="128000000,1000000,128,128", params="f32",
             grads="f32", states="f32"),
        # the same with half-width parameters and states in 8 bits, uneven tensors
        dict(name="adamw_8bit", kind="adamw", sizes="256000000,100003,5120,257,256,1",
             params="bf16", grads="bf16", states="q8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["norm", "loss", "loss", "loss", "adamw"])
    if kind == "norm":
        dim = rng.choice([4 * _log(rng, 4, 256), _log(rng, 9, 1500)])
        return dict(kind=kind, n=_log(rng, 1, min(262_144, 67_000_000 // dim)), dim=dim,
                    type=rng.choice(["f32", "bf16"]), grad=rng.random() < 0.6,
                    pad=rng.choice([0, 0, 64, 3]))
    if kind == "loss":
        dim = 4 * _log(rng, 4, 96)
        classes = _log(rng, 10, 1_000_000)
        grad = rng.random() < 0.65
        kind_of = rng.choice(["f32", "bf16", "bf16"])
        # no more products, and no more logits, than the largest listed case
        most = 4_000_000_000 * 128 // max(dim, 128) // (6 if kind_of == "f32" else 1)
        top = max(1, min(131_072, most // classes))
        n = _log(rng, min(256, top) if grad else 1, top)
        return dict(kind=kind, n=n, classes=classes, dim=dim, type=kind_of, grad=grad,
                    bias=rng.random() < 0.5, weights=rng.random() < 0.5,
                    unlabelled=rng.choice([0.0, 0.0, 0.1, 0.5]), masked=0.0, pad=rng.choice([0, 0, 32, 4]))
    count = rng.randint(1, 12)
    sizes = [_log(rng, 1, 40_000_000 // count) for _ in range(count)]
    params = rng.choice(["f32", "f32", "bf16"])
    return dict(kind=kind, sizes=",".join(str(s) for s in sizes), params=params,
                grads=rng.choice([params, "f32"]), states=rng.choice(["f32", "q8"]))


# --------------------------------------------------------------------------- #
# Inputs
# --------------------------------------------------------------------------- #
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rows(n, dim, pad, dtype, g, scale=1.0):
    """n rows of a buffer with `pad` more columns."""
    t = torch.randn((n, dim + pad), device=DEV, generator=g)
    return t.mul_(scale).to(dtype)[:, :dim]


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "norm":
        dt, dim = TYPES[case["type"]], case["dim"]
        s = dict(x=_rows(case["n"], dim, case["pad"], dt, g, 0.7),
                 gamma=1 + 0.1 * torch.randn(dim, device=DEV, generator=g),
                 beta=0.1 * torch.randn(dim, device=DEV, generator=g))
        s["x"] += 0.3  # embeddings part-way through training have a mean
        if case["grad"]:
            s["dy"] = _rows(case["n"], dim, case["pad"], dt, g)
        return s
    if case["kind"] == "loss":
        dt, n, classes, dim = TYPES[case["type"]], case["n"], case["classes"], case["dim"]
        w = _rows(classes, dim, case["pad"], dt, g, 1.5 / math.sqrt(dim))
        labels = torch.randint(0, classes, (n,), device=DEV, generator=g)
        # normalised rows that lean towards their label's row
        h = torch.randn((n, dim + case["pad"]), device=DEV, generator=g)
        h[:, :dim] += torch.rand((n, 1), device=DEV, generator=g) * 3 * w[labels].float()
        h = h.to(dt)[:, :dim]
        s = dict(h=h, w=w, bias=None, weights=None)
        if case["bias"]:
            s["bias"] = 0.3 * torch.randn(classes, device=DEV, generator=g)
        if case["masked"]:
            s["bias"][torch.rand(classes, device=DEV, generator=g) < case["masked"]] = -math.inf
        if case["weights"]:  # co-occurrence counts
            s["weights"] = torch.randint(1, 6, (n,), device=DEV, generator=g).float()
        if case["unlabelled"]:
            labels[torch.rand(n, device=DEV, generator=g) < case["unlabelled"]] = -1
        s["labels"] = labels.to(torch.int32)
        s["scale"] = 1.0 / n
        return s
    sizes = [int(t) for t in case["sizes"].split(",")]
    s = dict(params=[], grads=[], m=[], v=[])
    for size in sizes:
        p = 0.1 * torch.randn(size, device=DEV, generator=g)
        s["params"].append(p.to(TYPES[case["params"]]))
        # gradients whose scale differs from row to row of 128, as those of rare
        # and of frequent nodes do, and moments that fit them
        rows = torch.exp(2 * torch.randn(-(-size // 128), device=DEV, generator=g))
        rows = (1e-3 * rows).repeat_interleave(128)[:size]
        s["grads"].append((torch.randn(size, device=DEV, generator=g) * rows)
                          .to(TYPES[case["grads"]]))
        s["m"].append(0.2 * torch.randn(size, device=DEV, generator=g) * rows)
        v = torch.randn(size, device=DEV, generator=g).abs_() * rows
        s["v"].append(v.mul_(v))
        if case["states"] == "q8":  # values that 8 bits can hold
            s["m"][-1], s["v"][-1] = _values(*_codes(s["m"][-1], s["v"][-1]), size)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "adamw":
        s["steps"] = 10  # that the moments have seen
        s["state"] = None  # moments in 8 bits, kept in place of m and v
        if case["states"] == "q8":
            s["state"] = [_codes(m, v) for m, v in zip(s["m"], s["v"])]
    if own:
        import paper_2307_14490_amd as P
        s["P"] = P
        if case["kind"] == "loss":
            s["op"] = P.SoftmaxLoss(case["n"], case["classes"], case["dim"], dtype=case["type"],
                                    grad=case["grad"])
        if case["kind"] == "adamw":
            s["op"] = P.AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=EPS,
                              weight_decay=DECAY, states=case["states"])
            s["op"].load(s["m"], s["v"], s["steps"])
            s["state"] = None
    if case["kind"] == "adamw" and (own or case["states"] == "q8"):
        s["m"] = s["v"] = None
    return s


# --------------------------------------------------------------------------- #
# One pass
# --------------------------------------------------------------------------- #
def run(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        return _norm_own(s) if own else _norm_plain(s)
    if kind == "loss":
        return _loss_own(s) if own else _loss_plain(s)
    return _adamw_own(s) if own else _adamw_plain(s)


def _norm_own(s):
    P = s["P"]
    y, mean, rstd = P.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS_NORM)
    out = dict(y=y, mean=mean, rstd=rstd)
    if s["case"]["grad"]:
        dx, dgamma, dbeta = P.layer_norm_backward(s["dy"], s["x"], s["gamma"], mean, rstd)
        out.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return out


def _norm_plain(s):
    x = s["x"].float()
    mean = x.mean(1)
    z = x - mean[:, None]
    rstd = 1 / torch.sqrt((z * z).mean(1) + EPS_NORM)
    z = z * rstd[:, None]
    out = dict(y=(z * s["gamma"] + s["beta"]).to(s["x"].dtype), mean=mean, rstd=rstd)
    if s["case"]["grad"]:
        dy = s["dy"].float()
        a = dy * s["gamma"]
        dx = (a - a.mean(1, keepdim=True) - z * (a * z).mean(1, keepdim=True)) * rstd[:, None]
        out.update(dx=dx.to(s["x"].dtype), dgamma=(dy * z).sum(0), dbeta=dy.sum(0))
    return out


def _loss_own(s):
    op = s["op"]
    loss, lse = op.loss(s["h"], s["w"], s["labels"], bias=s["bias"], weights=s["weights"])
    out = dict(loss=loss, lse=lse)
    if s["case"]["grad"]:
        dh, dw, db = op.grad(s["h"], s["w"], s["labels"], lse, bias=s["bias"],
                             weights=s["weights"], scale=s["scale"])
        out.update(dh=dh, dw=dw, db=db)
    return out


def _loss_plain(s):
    h, w, labels = s["h"].float(), s["w"].float(), s["labels"].long()
    x = h @ w.t()
    if s["bias"] is not None:
        x += s["bias"]
    top = x.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log((x - top).exp_().sum(1))
    y = labels.clamp(min=0)
    at = x.gather(1, y[:, None])[:, 0]
    c = ((labels >= 0) & (at > -math.inf)).float()  # rows with a label that is not masked
    if s["weights"] is not None:
        c *= s["weights"]
    out = dict(loss=torch.where(c > 0, c * (lse - at), torch.zeros_like(c)), lse=lse)
    if s["case"]["grad"]:
        c *= s["scale"]
        x -= lse[:, None]
        p = x.exp_().mul_(c[:, None])
        rows = torch.arange(len(y), device=y.device)
        p[rows, y] -= c
        out.update(dh=(p @ w).to(s["h"].dtype), dw=(p.t() @ h).to(s["w"].dtype), db=p.sum(0))
    return out


def _adamw_own(s):
    op = s["op"]
    op.step(s["grads"])
    m, v = op.values()
    return dict(params=s["params"], m=m, v=v)


def _blocks(x):
    """x as rows of BLOCK values, the last one filled with zeros."""
    rows = x.new_zeros((-(-x.numel() // BLOCK), BLOCK))
    rows.view(-1)[:x.numel()] = x
    return rows


def _codes(m, v):
    """The moments in 8 bits: in blocks, m by s sgn(m) (q / 127)^2 and sqrt(v) by
    t (u / 255)^2, with s and t the block's largest."""
    m, r = _blocks(m), torch.sqrt(_blocks(v))
    s, t = m.abs().amax(1, keepdim=True), r.amax(1, keepdim=True)
    zero = torch.zeros_like(s)
    q = torch.round(torch.sqrt(m.abs() * torch.where(s > 0, torch.reciprocal(s), zero)) * 127.0)
    u = torch.round(torch.sqrt(r * torch.where(t > 0, torch.reciprocal(t), zero)) * 255.0)
    u = torch.where(r > 0, u.clamp(min=1.0), u)
    return (q * m.sign()).to(torch.int8), s, u.to(torch.uint8), t


def _values(q, s, u, t, size):
    a = q.float()
    b = a.abs() * float(np.float32(1) / np.float32(127))
    c = u.float() * float(np.float32(1) / np.float32(255))
    r = t * (c * c)
    return (a.sign() * (s * (b * b))).view(-1)[:size], (r * r).view(-1)[:size]


def _adamw_plain(s):
    s["steps"] += 1
    q8 = s["case"]["states"] == "q8"
    new = [_adamw_one(s, k, q8) for k in range(len(s["params"]))]
    if not q8:
        s["m"], s["v"] = [n[0] for n in new], [n[1] for n in new]
    return dict(params=s["params"], m=[n[0] for n in new], v=[n[1] for n in new])


def _adamw_one(s, k, q8):
    p, g = s["params"][k], s["grads"][k].float()
    m, v = _values(*s["state"][k], p.numel()) if q8 else (s["m"][k], s["v"][k])
    f = np.float32
    rate = float(f(LR / (1 - BETA1 ** s["steps"])))
    fix = float(f(1 / math.sqrt(1 - BETA2 ** s["steps"])))
    m = m * float(f(BETA1)) + g * float(f(1 - BETA1))
    v = v * float(f(BETA2)) + (g * g) * float(f(1 - BETA2))
    step = (m * rate) / (torch.sqrt(v) * fix + float(f(EPS)))
    p.copy_(p.float() * float(f(1 - LR * DECAY)) - step)
    if q8:
        s["state"][k] = _codes(m, v)
        m, v = _values(*s["state"][k], p.numel())
    return m, v


# --------------------------------------------------------------------------- #
# Work and exact values
# --------------------------------------------------------------------------- #
def work(case):
    if case["kind"] == "adamw":
        n = sum(int(t) for t in case["sizes"].split(","))
        p, g = (2 if case[k] == "bf16" else 4 for k in ("params", "grads"))
        # parameter and states read and written, gradient read; the values of
        # states in 8 bits are written out beside them
        state = 16 if case["states"] == "f32" else 4 + 8 + 32 / BLOCK
        return dict(bytes=n * (2 * p + g + state), flops=15 * n)
    e, n, dim = (2 if case["type"] == "bf16" else 4), case["n"], case["dim"]
    if case["kind"] == "norm":
        b, f = 2 * n * dim * e + 8 * n + 8 * dim, 8 * n * dim
        if case["grad"]:
            # x is read again: the backward pass is another call
            b, f = b + 3 * n * dim * e + 8 * n + 12 * dim, f + 12 * n * dim
        return dict(bytes=b, flops=f)
    classes = case["classes"]
    b = (n + classes) * dim * e + 12 * n + (4 * classes if case["bias"] else 0) \
        + (4 * n if case["weights"] else 0)
    f = 2 * n * classes * dim
    if case["grad"]:
        b, f = b + (n + classes) * dim * e + 4 * classes, 3 * f
    return dict(bytes=b, flops=f)


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _norm_exact, "loss": _loss_exact, "adamw": _adamw_exact}[case["kind"]](case, s)


def _norm_exact(case, s):
    x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
    mean = x.sum(1) / case["dim"]
    rstd = ((x - mean[:, None]).square().sum(1) / case["dim"] + EPS_NORM).rsqrt()
    z = torch.addcmul(torch.zeros_like(x), x - mean[:, None], rstd[:, None])
    out = dict(y=z * gamma + beta, mean=mean, rstd=rstd)
    if case["grad"]:
        # (I - 1 1' / dim - z z' / dim) applied to the gradient of z
        dy = s["dy"].double()
        dz = dy * gamma
        along = (dz * z).sum(1, keepdim=True)
        flat = dz.sum(1, keepdim=True)
        out.update(dx=rstd[:, None] * (dz - (flat + z * along) / case["dim"]),
                   dgamma=torch.mv((dy * z).t().contiguous(), torch.ones_like(mean)),
                   dbeta=torch.mv(dy.t().contiguous(), torch.ones_like(mean)))
    return out


def _loss_exact(case, s):
    """In two passes over pieces of the vocabulary, with a running maximum and sum."""
    h, labels = s["h"].double(), s["labels"].long()
    n, classes = case["n"], case["classes"]
    piece = max(1024, min(classes, 400_000_000 // n))
    bias = torch.zeros(classes, device=DEV) if s["bias"] is None else s["bias"]
    have = labels >= 0
    top = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    total = torch.zeros(n, dtype=torch.float64, device=DEV)
    pieces = [(a, min(classes, a + piece)) for a in range(0, classes, piece)]

    def logits(a, b):
        return torch.addmm(bias[a:b].double(), h, s["w"][a:b].double().t())

    for a, b in pieces:
        x = logits(a, b)
        new = torch.maximum(top, x.amax(1))
        total = total * torch.exp(top - new) + torch.exp(x - new[:, None]).sum(1)
        top = new
        del x
    lse = top + torch.log(total)
    y = labels[have]
    at = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    at[have] = (h[have] * s["w"][y].double()).sum(1) + bias[y].double()
    c = torch.ones(n, dtype=torch.float64, device=DEV) if s["weights"] is None \
        else s["weights"].double()
    c = torch.where(at > -math.inf, c, torch.zeros_like(c))
    loss = torch.zeros_like(c)
    loss[c > 0] = (c * (lse - at))[c > 0]
    out = dict(loss=loss, lse=lse)
    if case["grad"]:
        c = c / n
        dh = torch.zeros_like(h)
        dw = torch.empty((classes, case["dim"]), dtype=torch.float64, device=DEV)
        db = torch.empty(classes, dtype=torch.float64, device=DEV)
        for a, b in pieces:
            p = torch.exp(logits(a, b) - lse[:, None]) * c[:, None]
            here = (labels >= a) & (labels < b)
            p[here.nonzero()[:, 0], labels[here] - a] -= c[here]
            dh += p @ s["w"][a:b].double()
            dw[a:b] = p.t() @ h
            db[a:b] = p.sum(0)
            del p
        out.update(dh=dh, dw=dw, db=db)
    return out


def _adamw_exact(case, s):
    t = 11
    out = dict(params=[], m=[], v=[])
    for p, g, m, v in zip(s["params"], s["grads"], s["m"], s["v"]):
        g = g.double()
        m = BETA1 * m.double() + (1 - BETA1) * g
        v = BETA2 * v.double() + (1 - BETA2) * g.square()
        unbiased = v / (1 - BETA2 ** t)
        q = p.double() - LR * (m / (1 - BETA1 ** t) / (unbiased.sqrt() + EPS)
                               + DECAY * p.double())
        if case["states"] == "q8":
            m, v = _nearest(m, v)
        out["params"].append(q)
        out["m"].append(m)
        out["v"].append(v)
    return out


def _nearest(m, v):
    """The values that moments in 8 bits stand for, in 64-bit arithmetic."""
    size, r = m.numel(), v.sqrt()
    fill = -size % BLOCK
    m, r = (torch.nn.functional.pad(x, (0, fill)).view(-1, BLOCK) for x in (m, r))
    s, t = (x.abs().max(1, keepdim=True).values.clamp(min=1e-300) for x in (m, r))
    k = (127 * (m.abs() / s).sqrt()).round() / 127
    j = (255 * (r / t).sqrt()).round()
    j = torch.where(r > 0, j.clamp(min=1), j) / 255
    return (torch.sign(m) * s * k.square()).flatten()[:size], \
        (t * j.square()).square().flatten()[:size]
