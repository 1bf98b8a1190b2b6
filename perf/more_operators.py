"""The operators that normalise rows for a softmax head, answer with it and clip its
gradients, as they are timed.

Three kinds of call, each through the package's public entry points:

  rms     rms_norm over rows with the residual's addition, in the rows' type or in 8
          bits with a scale for each 32 columns, and rms_norm_backward;
  answer  LogProbs.log_probs: log probabilities of given classes over every row of an
          output table (in 32, 16 or 8 bits), with the entropy and the most likely
          classes, without keeping the logits; and LogProbs.grad, the gradient of
          weighted sums of log probabilities and entropies;
  clip    grad_norm over a list of tensors, and AdamW.step with gradients clipped to
          a largest norm.

Sizes are those of the workloads in synth/gen.py: vocabularies of 10,000 to a
million nodes or the blocks of a block model, rows of 32 to 256 values, batches
from one row to a hundred thousand.  With `own` false the same is computed in
elementary torch operations in 32 bits; the logits that decide which classes are the
most likely, and the sum under a norm, in 64.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
MAX_NORM = 1.0
BLOCK = 32    # columns that share a scale of rows in 8 bits
LEAST = -100  # smallest power of two of a scale


# --------------------------------------------------------------------------- #
# Cases
# --------------------------------------------------------------------------- #
def listed():
    return [
        # one small batch of the tiny workload normalised before the head: latency
        dict(name="rms_small", kind="rms", n=1024, dim=32, type="f32", residual=True, q8=False,
             grad=False, pad=0),
        # training on a medium batch, half-width rows on a residual stream
        dict(name="rms_train", kind="rms", n=65_536, dim=128, type="bf16", residual=True, q8=False,
             grad=True, pad=0),
        # training on rows of an odd width, columns of a wider buffer
        dict(name="rms_odd", kind="rms", n=60_417, dim=761, type="f32", residual=True, q8=False,
             grad=True, pad=3),
        # a million nodes' rows normalised and kept in 8 bits, to be answered from
        dict(name="rms_table8", kind="rms", n=1_000_000, dim=128, type="bf16", residual=False,
             q8=True, grad=False, pad=0),
        # serving: one row's distribution over a million nodes in 8 bits, ten best
        dict(name="answer_one", kind="answer", n=1, classes=1_000_000, dim=128, type="q8", top=10,
             labels=False, bias=False, masked=0.0, grad=False, pad=0),
        # serving a few rows in 32 bits, some nodes taken out of the vocabulary
        dict(name="answer_few", kind="answer", n=38, classes=300_007, dim=256, type="f32", top=5,
             labels=True, bias=True, masked=0.02, grad=False, pad=0),
        # evaluation: a held-out batch over the medium vocabulary
        dict(name="answer_batch", kind="answer", n=4096, classes=1_000_000, dim=128, type="bf16",
             top=10, labels=True, bias=False, masked=0.0, grad=False, pad=0),
        # a classifier of the nodes' blocks trained by its log probabilities with a term
        # for the entropy: few classes, many rows
        dict(name="policy_blocks", kind="answer", n=100_003, classes=1000, dim=128, type="bf16",
             top=0, labels=True, bias=True, masked=0.0, grad=True, pad=0),
        # the same over nodes, wide rows in 32 bits, ragged sizes, nodes taken out
        dict(name="policy_nodes", kind="answer", n=3001, classes=50_021, dim=256, type="f32",
             top=0, labels=True, bias=True, masked=0.02, grad=True, pad=32),
        # the optimiser's clipped step on a small head: four tensors, latency
        dict(name="clip_head", kind="clip", sizes="32,32,320,10", params="f32", grads="f32",
             step=True),
        # the same on a vocabulary table and a head
        dict(name="clip_table", kind="clip", sizes="128000000,1000000,128,128", params="f32",
             grads="f32", step=True),
        # the norm alone over many uneven tensors in half width
        dict(name="norm_many", kind="clip", sizes="400x100000", params="bf16", grads="bf16",
             step=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["rms", "rms", "answer", "answer", "answer", "clip"])
    if kind == "rms":
        q8 = rng.random() < 0.3
        dim = rng.choice([4 * _log(rng, 4, 256), _log(rng, 9, 1500)])
        return dict(kind=kind, n=_log(rng, 1, min(1_000_000, 45_000_000 // dim)), dim=dim,
                    type=rng.choice(["f32", "bf16"]), residual=rng.random() < 0.6, q8=q8,
                    grad=not q8 and rng.random() < 0.6, pad=rng.choice([0, 0, 64, 3]))
    if kind == "answer":
        dim = 4 * _log(rng, 4, 96)
        classes = _log(rng, 10, 1_000_000)
        kind_of = rng.choice(["f32", "bf16", "bf16", "q8"])
        grad = kind_of != "q8" and rng.random() < 0.4
        # no more products, and no more logits, than the largest listed case
        most = 4_000_000_000 * 128 // max(dim, 128) // (6 if kind_of == "f32" else 1)
        top = max(1, min(131_072, most // classes // (3 if grad else 1)))
        few = not grad and rng.random() < 0.4
        n = _log(rng, min(256, top) if grad else 1, min(64, top) if few else top)
        return dict(kind=kind, n=n, classes=classes, dim=dim, type=kind_of,
                    top=0 if grad else min(classes, rng.choice([0, 1, 3, 10, 20])),
                    labels=grad or rng.random() < 0.7, bias=rng.random() < 0.5, masked=0.0,
                    grad=grad, pad=rng.choice([0, 0, 32, 4]))
    count = rng.randint(1, 12)
    sizes = [_log(rng, 1, 40_000_000 // count) for _ in range(count)]
    params = rng.choice(["f32", "f32", "bf16"])
    return dict(kind=kind, sizes=",".join(str(s) for s in sizes), params=params,
                grads=rng.choice([params, "f32"]), step=rng.random() < 0.6)


def _sizes(case):
    """Elements of each tensor: a list, or COUNTxSIZE for uneven ones about SIZE."""
    if "x" not in case["sizes"]:
        return [int(t) for t in case["sizes"].split(",")]
    count, size = (int(t) for t in case["sizes"].split("x"))
    return [size * (1 + k % 7) // 4 + k for k in range(count)]


# --------------------------------------------------------------------------- #
# Inputs
# --------------------------------------------------------------------------- #
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rows(n, dim, pad, dtype, g, scale=1.0):
    """n rows of a buffer with `pad` more columns."""
    t = torch.randn((n, dim + pad), device=DEV, generator=g)
    return t.mul_(scale).to(dtype)[:, :dim]


def _table8(x):
    """Rows in 8 bits: codes (e4m3) and a power of two for each 32 columns, as 127 + its
    exponent: the smallest under which nothing is above e4m3's largest, 448."""
    n, dim = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -dim % BLOCK)).view(n, -1, BLOCK)
    m, e = torch.frexp(b.abs().amax(2))            # m 2^e, m in [1/2, 1)
    e = (e - 9 + (m > 0.875)).clamp(LEAST, 127)    # 448 = 0.875 2^9
    codes = torch.ldexp(b, -e[:, :, None]).view(n, -1)[:, :dim].to(torch.float8_e4m3fn)
    return codes.contiguous(), (e + 127).to(torch.uint8)


def _values8(codes, scales):
    """What rows in 8 bits stand for, in 32 bits."""
    e = torch.repeat_interleave(scales.int() - 127, BLOCK, 1)[:, :codes.shape[1]]
    return torch.ldexp(codes.float(), e)


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "rms":
        dt, n, dim, pad = TYPES[case["type"]], case["n"], case["dim"], case["pad"]
        s = dict(x=_rows(n, dim, pad, dt, g, 0.7), residual=None,
                 gamma=1 + 0.1 * torch.randn(dim, device=DEV, generator=g))
        if case["residual"]:  # what earlier layers added up
            s["residual"] = _rows(n, dim, pad, dt, g, 1.5)
        if case["grad"]:
            s["dy"] = _rows(n, dim, pad, dt, g)
            if case["residual"]:
                s["dtotal"] = _rows(n, dim, pad, dt, g)
        return s
    if case["kind"] == "answer":
        n, classes, dim, pad = case["n"], case["classes"], case["dim"], case["pad"]
        dt = TYPES.get(case["type"], torch.bfloat16)
        w = _rows(classes, dim, pad, dt, g, 1.5 / math.sqrt(dim))
        labels = torch.randint(0, classes, (n,), device=DEV, generator=g)
        # normalised rows that lean towards their class's row
        h = torch.randn((n, dim + pad), device=DEV, generator=g)
        h[:, :dim] += torch.rand((n, 1), device=DEV, generator=g) * 3 * w[labels].float()
        s = dict(h=h.to(dt)[:, :dim], w=w, labels=None, bias=None)
        if case["type"] == "q8":
            s["w"], s["scales"] = _table8(w)
        if case["labels"]:
            s["labels"] = labels.to(torch.int32)
        if case["bias"]:
            s["bias"] = 0.3 * torch.randn(classes, device=DEV, generator=g)
        if case["masked"]:
            s["bias"][torch.rand(classes, device=DEV, generator=g) < case["masked"]] = -math.inf
        if case["grad"]:  # advantages, of both signs, and the entropy's weight
            s["dlogp"] = torch.randn(n, device=DEV, generator=g) / n
            s["dentropy"] = torch.full((n,), 0.01 / n, device=DEV)
        return s
    s = dict(params=[], grads=[], m=[], v=[])
    for size in _sizes(case):
        # gradients whose scale differs from row to row of 128, as those of rare and of
        # frequent nodes do, and moments that fit them once they are clipped
        rows = torch.exp(2 * torch.randn(-(-size // 128), device=DEV, generator=g))
        rows = (1e-3 * rows).repeat_interleave(128)[:size]
        s["grads"].append((torch.randn(size, device=DEV, generator=g) * rows)
                          .to(TYPES[case["grads"]]))
        if case["step"]:
            p = 0.1 * torch.randn(size, device=DEV, generator=g)
            s["params"].append(p.to(TYPES[case["params"]]))
            s["m"].append(2e-3 * torch.randn(size, device=DEV, generator=g) * rows)
            v = torch.randn(size, device=DEV, generator=g).abs_() * rows * 1e-2
            s["v"].append(v.mul_(v))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    s["steps"] = 10  # that the optimiser's moments have seen
    if own:
        import paper_2307_14490_amd as P
        s["P"] = P
        if case["kind"] == "answer":
            s["op"] = P.LogProbs(case["n"], case["classes"], case["dim"], dtype=case["type"],
                                 top=case["top"], grad=case["grad"])
            if case["type"] == "q8":
                s["w"] = P.Q8Rows(s["w"], s["scales"])
        if case["kind"] == "clip" and case["step"]:
            s["op"] = P.AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=EPS,
                              weight_decay=DECAY)
            s["op"].load(s["m"], s["v"], s["steps"])
            s["m"] = s["v"] = None
    return s


# --------------------------------------------------------------------------- #
# One pass
# --------------------------------------------------------------------------- #
def run(s):
    kind = s["case"]["kind"]
    if kind == "rms":
        return _rms_own(s) if own else _rms_plain(s)
    if kind == "answer":
        return _answer_own(s) if own else _answer_plain(s)
    return _clip_own(s) if own else _clip_plain(s)


def _rms_own(s):
    P, case = s["P"], s["case"]
    y, total, rstd = P.rms_norm(s["x"], s["gamma"], residual=s["residual"], eps=EPS_NORM,
                                q8=case["q8"])
    # values of 8 bits are read back: a code times a power of two is one in 16 bits
    out = dict(y=P.q8_values(y, dtype="bf16") if case["q8"] else y, rstd=rstd)
    if case["residual"]:
        out["total"] = total
    if case["grad"]:
        out["dx"], out["dgamma"] = P.rms_norm_backward(s["dy"], total, s["gamma"], rstd,
                                                       dtotal=s.get("dtotal"))
    return out


def _rms_plain(s):
    case, dt = s["case"], s["x"].dtype
    total = s["x"]
    if case["residual"]:
        total = (s["x"].float() + s["residual"].float()).to(dt)
    t = total.float()
    rstd = 1 / torch.sqrt((t * t).mean(1) + EPS_NORM)
    z = t * rstd[:, None]
    y = z * s["gamma"]
    out = dict(y=_values8(*_table8(y)).to(torch.bfloat16) if case["q8"] else y.to(dt), rstd=rstd)
    if case["residual"]:
        out["total"] = total
    if case["grad"]:
        dy = s["dy"].float()
        a = dy * s["gamma"]
        dx = (a - z * (a * z).mean(1, keepdim=True)) * rstd[:, None]
        if case["residual"]:
            dx += s["dtotal"].float()
        out.update(dx=dx.to(dt), dgamma=(dy * z).sum(0))
    return out


def _answer_own(s):
    op, case = s["op"], s["case"]
    a = op.log_probs(s["h"], s["w"], labels=s["labels"], bias=s["bias"])
    out = dict(entropy=a.entropy, lse=a.lse)
    if case["labels"]:
        out["logp"] = a.logp
    if case["top"]:
        out.update(ids=a.ids, top_logp=a.top_logp)
    if case["grad"]:
        out["dh"], out["dw"], out["db"] = op.grad(s["h"], s["w"], a, labels=s["labels"],
                                                  dlogp=s["dlogp"], dentropy=s["dentropy"],
                                                  bias=s["bias"])
    return out


def _answer_plain(s):
    case, h = s["case"], s["h"].float()
    w = _values8(s["w"], s["scales"]) if case["type"] == "q8" else s["w"].float()
    x = h @ w.t()
    if s["bias"] is not None:
        x += s["bias"]
    best = None
    if case["top"]:  # more than are wanted, in 32 bits, and their order in 64
        more = torch.topk(x, min(case["classes"], case["top"] + 8), dim=1).indices
        best = _order(s, h, w, more)[:2]
    y = None if s["labels"] is None else s["labels"].long()
    at = None if y is None else x.gather(1, y[:, None])[:, 0]
    top = x.amax(1, keepdim=True)
    x = x.sub_(top).clamp_(min=-1e30)
    p = torch.exp(x)
    total = p.sum(1)
    logs = torch.log(total)
    lse = top[:, 0] + logs
    out = dict(entropy=logs - (p * x).sum(1) / total, lse=lse)
    if y is not None:
        out["logp"] = at - lse
    if best is not None:
        out.update(ids=best[0], top_logp=(best[1] - lse.double()[:, None]).float())
    if case["grad"]:
        # of sum dlogp logp + dentropy entropy: p / total is the probability, x - logs its log
        x -= logs[:, None]
        p /= total[:, None]
        x += out["entropy"][:, None]
        dlogp = s["dlogp"] * (at > -math.inf)  # the others' log probability is constant
        p *= -dlogp[:, None] - s["dentropy"][:, None] * x
        p[torch.arange(len(y), device=y.device), y] += dlogp
        out.update(dh=(p @ w).to(s["h"].dtype), dw=(p.t() @ h).to(s["w"].dtype), db=p.sum(0))
    return out


def _order(s, h, w, ids):
    """The `top` best of the classes `ids` of each row by their logits in 64 bits, the
    lowest first among equals."""
    ids = ids.sort(1).values
    x = (w[ids].double() * h[:, None, :].double()).sum(2)
    if s["bias"] is not None:
        x += s["bias"].double()[ids]
    x, at = torch.sort(x, dim=1, descending=True, stable=True)
    k = s["case"]["top"]
    return ids.gather(1, at)[:, :k].to(torch.int32), x[:, :k]


def _clip_own(s):
    if not s["case"]["step"]:
        return dict(norm=s["P"].grad_norm(s["grads"]))
    op = s["op"]
    norm = op.step(s["grads"], max_norm=MAX_NORM)
    m, v = op.values()
    return dict(norm=norm, params=s["params"], m=m, v=v)


def _clip_plain(s):
    squares = [g.double().square().sum() for g in s["grads"]]
    norm = torch.sqrt(torch.stack(squares).sum()).float().view(1)
    if not s["case"]["step"]:
        return dict(norm=norm)
    s["steps"] += 1
    factor = torch.clamp(MAX_NORM / norm, max=1.0)
    rate = LR / (1 - BETA1 ** s["steps"])
    fix = 1 / math.sqrt(1 - BETA2 ** s["steps"])
    for k, p in enumerate(s["params"]):
        g = s["grads"][k].float() * factor
        s["m"][k] = s["m"][k] * BETA1 + g * (1 - BETA1)
        s["v"][k] = s["v"][k] * BETA2 + (g * g) * (1 - BETA2)
        step = (s["m"][k] * rate) / (torch.sqrt(s["v"][k]) * fix + EPS)
        p.copy_(p.float() * (1 - LR * DECAY) - step)
    return dict(norm=norm, params=s["params"], m=s["m"], v=s["v"])


# --------------------------------------------------------------------------- #
# Work and exact values
# --------------------------------------------------------------------------- #
def work(case):
    if case["kind"] == "clip":
        n = sum(_sizes(case))
        p, g = (2 if case[k] == "bf16" else 4 for k in ("params", "grads"))
        if not case["step"]:
            return dict(bytes=n * g, flops=2 * n)
        # parameter and moments read and written; the gradient is read for the norm
        # and again, for every element's step needs the norm
        return dict(bytes=n * (2 * p + 2 * g + 16), flops=18 * n)
    n, dim = case["n"], case["dim"]
    if case["kind"] == "rms":
        e = 2 if case["type"] == "bf16" else 4
        arrays = 1 + (2 if case["residual"] else 0)  # x; residual, total
        b, f = arrays * n * dim * e + 4 * n + 4 * dim, 5 * n * dim
        # in 8 bits: codes written, and read back as values of 16 bits
        b += n * dim * 4 + 2 * n * -(-dim // BLOCK) if case["q8"] else n * dim * e
        if case["grad"]:
            # total is read again: the backward pass is another call
            b += (4 if case["residual"] else 3) * n * dim * e + 4 * n + 8 * dim
            f += 10 * n * dim
        return dict(bytes=b, flops=f)
    classes, e = case["classes"], 4 if case["type"] == "f32" else 2
    table = classes * dim * e if case["type"] != "q8" else classes * (dim + -(-dim // BLOCK))
    b = n * dim * e + table + 8 * n + (8 * n if case["labels"] else 0) \
        + (4 * classes if case["bias"] else 0) + 8 * n * case["top"]
    f = 2 * n * classes * dim
    if case["grad"]:
        b, f = b + 8 * n + n * dim * e + classes * dim * e + 4 * classes, 3 * f
    return dict(bytes=b, flops=f)


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rms": _rms_exact, "answer": _answer_exact, "clip": _clip_exact}[case["kind"]](case, s)


def _rms_exact(case, s):
    x, gamma, dim = s["x"].double(), s["gamma"].double(), case["dim"]
    if case["residual"]:  # the sum is kept in the rows' type, and that is what is normalised
        sums = x + s["residual"].double()
        x = sums.to(s["x"].dtype).double()
    rstd = ((x * x).sum(1) / dim + EPS_NORM).rsqrt()
    y = x * (rstd[:, None] * gamma)
    if case["q8"]:
        y = _nearest8(y)
    out = dict(y=y, rstd=rstd)
    if case["residual"]:
        out["total"] = x
    if case["grad"]:
        # (I - z z' / dim) applied to the gradient of z
        z, dy = x * rstd[:, None], s["dy"].double()
        along = (dy * gamma * z).sum(1, keepdim=True) / dim
        dx = rstd[:, None] * (dy * gamma - z * along)
        out["dx"] = dx + s["dtotal"].double() if case["residual"] else dx
        out["dgamma"] = torch.mv((dy * z).t().contiguous(), torch.ones_like(rstd))
    return out


def _nearest8(y):
    """The nearest values that 8 bits under a scale for each 32 columns hold: 3 bits
    behind the leading one, down to 2^-9 of the scale, ties to even."""
    n, dim = y.shape
    b = torch.nn.functional.pad(y, (0, -dim % BLOCK)).view(n, -1, BLOCK)
    most = b.abs().amax(2, keepdim=True).clamp(min=1e-300)
    scale = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp(LEAST, 127))
    b = b / scale
    unit = torch.exp2(torch.floor(torch.log2(b.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(b / unit) * unit * scale).view(n, -1)[:, :dim]


def _answer_exact(case, s):
    """In passes over pieces of the vocabulary, with a running maximum and sums."""
    h = s["h"].double()
    n, classes = case["n"], case["classes"]
    w = _values8(s["w"], s["scales"]) if case["type"] == "q8" else s["w"]
    piece = max(1024, min(classes, 400_000_000 // n))
    bias = torch.zeros(classes, device=DEV) if s["bias"] is None else s["bias"]
    top = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
    total, first = torch.zeros_like(top), torch.zeros_like(top)
    ids = torch.zeros((n, 0), dtype=torch.long, device=DEV)
    best = torch.zeros((n, 0), dtype=torch.float64, device=DEV)
    pieces = [(a, min(classes, a + piece)) for a in range(0, classes, piece)]

    def logits(a, b):
        return torch.addmm(bias[a:b].double(), h, w[a:b].double().t())

    for a, b in pieces:
        x = logits(a, b)
        if case["top"]:
            v, k = torch.topk(x, min(case["top"], b - a), dim=1)
            best, ids = torch.cat([best, v], 1), torch.cat([ids, k + a], 1)
        new = torch.maximum(top, x.amax(1))
        keep = torch.exp(top - new)
        # first: sum of exp(x) x, both about the maximum
        first = torch.where(keep > 0, (first + total * (top - new)) * keep, torch.zeros_like(first))
        x = (x - new[:, None]).clamp_(min=-1e300)
        e = torch.exp(x)
        total = total * keep + e.sum(1)
        first += x.mul_(e).sum(1)
        top = new
        del x, e
    lse = top + torch.log(total)
    entropy = torch.log(total) - first / total
    out = dict(entropy=entropy, lse=lse)
    if case["top"]:
        v, k = torch.topk(best, case["top"], dim=1)
        out.update(ids=None, top_logp=v - lse[:, None])
    if not case["labels"]:
        return out
    y = s["labels"].long()
    at = (h * w[y].double()).sum(1) + bias[y].double()
    out["logp"] = at - lse
    if case["grad"]:
        dl, de = s["dlogp"].double() * (at > -math.inf), s["dentropy"].double()
        dh = torch.zeros_like(h)
        dw = torch.empty((classes, case["dim"]), dtype=torch.float64, device=DEV)
        db = torch.empty(classes, dtype=torch.float64, device=DEV)
        for a, b in pieces:
            logp = (logits(a, b) - lse[:, None]).clamp_(min=-1e300)
            g = torch.exp(logp) * (-dl[:, None] - de[:, None] * (logp + entropy[:, None]))
            here = (y >= a) & (y < b)
            g[here.nonzero()[:, 0], y[here] - a] += dl[here]
            dh += g @ w[a:b].double()
            dw[a:b] = g.t() @ h
            db[a:b] = g.sum(0)
            del logp, g
        out.update(dh=dh, dw=dw, db=db)
    return out


def _clip_exact(case, s):
    square = sum(float((g.double() ** 2).sum()) for g in s["grads"])
    norm = math.sqrt(square)
    out = dict(norm=torch.tensor([norm], dtype=torch.float64, device=DEV))
    if not case["step"]:
        return out
    t = 11
    out.update(params=[], m=[], v=[])
    for p, g, m, v in zip(s["params"], s["grads"], s["m"], s["v"]):
        g = g.double() * min(1.0, MAX_NORM / norm)
        m = BETA1 * m.double() + (1 - BETA1) * g
        v = BETA2 * v.double() + (1 - BETA2) * g.square()
        unbiased = v / (1 - BETA2 ** t)
        out["params"].append(p.double() - LR * (m / (1 - BETA1 ** t) / (unbiased.sqrt() + EPS)
                                                + DECAY * p.double()))
        out["m"].append(m)
        out["v"].append(v)
    return out
