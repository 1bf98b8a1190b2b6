"""What normalises, answers and clips on streams, in graphs and together in a head: the
same bits as one call after the other.  Streams are kept busy with other work, so that
what is not ordered would come too early."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402
from test_gpu_head_streams import _need_gpu, busy  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def inputs(dtype, n=300, classes=700, dim=64, seed=8):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    new = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x, r, w = (t.to(kind) for t in (new(n, dim), new(n, dim), new(classes, dim) * 0.2))
    lab = torch.randint(0, classes, (n,), device="cuda", generator=g).to(torch.int32)
    out = dict(x=x, r=r, w=w, lab=lab, adv=new(n), bias=new(classes), gamma=1 + 0.1 * new(dim))
    torch.cuda.synchronize()
    return out


def same(a, b):
    for u, v in zip(a, b):
        assert (u is None and v is None) or torch.equal(u, v)


@pytest.mark.parametrize("dtype,states,norm", [("f32", "f32", "rms"), ("bf16", "q8", "rms"),
                                               ("bf16", "f32", "layer")])
def test_head_takes_turns_between_streams(dtype, states, norm):
    k = inputs(dtype)
    say(f"head that answers on two streams, {dtype}, moments {states}, {norm} norm")

    def train(streams):
        busy()
        head = P.SoftmaxHead(700, 64, 300, dtype=dtype, lr=1e-2, states=states, seed=2, norm=norm,
                             max_norm=0.5, top=3)
        got = []
        for s in streams:
            busy(s)
            got += list(head.step(k["x"], k["lab"], stream=s))
            got.append(head.norm_before)
            a, dx = head.policy_step(k["x"], k["lab"], k["adv"], 0.05, stream=s)
            got += [*a, dx, *head.answers(k["x"], stream=s)[1:]]
        torch.cuda.synchronize()
        head.check()
        return got + list(head.opt.params)

    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    same(train([None] * 4), train([a, b, None, a]))


def together(k, op, opt, small):
    """A training step and an answer, as they follow each other."""
    y, total, rstd = P.rms_norm(k["x"], k["gamma"], k["r"])
    a = op.log_probs(y, k["w"], k["lab"], k["bias"])
    dlogp = k["adv"] * -0.01
    dy, dw, db = op.grad(y, k["w"], a, k["lab"], dlogp, dlogp, k["bias"])
    dx, dgamma = P.rms_norm_backward(dy, total, k["gamma"], rstd, k["r"])
    norm = opt.step([dgamma, dw, db], max_norm=0.01)
    other = P.clip_grads([dw, db], 0.005)
    q, _, _ = P.rms_norm(k["w"], k["gamma"], q8=True)
    s = small.log_probs(k["x"][:20].to(torch.bfloat16), q)
    return [*a, dx, dgamma, norm, other, dw, db, P.q8_values(q), *s[1:], *opt.params,
            P.grad_norm([dx, dgamma])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_run_of_all_replays(dtype):
    """Captured once, replayed between eager work and synchronisations: each replay is
    what the same calls give eagerly."""
    k = inputs(dtype)
    say(f"captured run, {dtype}")

    def make():
        ps = [k["gamma"].clone(), k["w"].clone(), k["bias"].clone()]
        return (P.LogProbs(300, 700, 64, dtype=dtype, top=4, grad=True),
                P.AdamW(ps, lr=1e-2, betas=(0.0, 0.0)),
                P.LogProbs(20, 700, 64, dtype="q8", top=5))

    op, opt, small = make()
    ref_op, ref_opt, ref_small = make()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        together(k, op, opt, small)  # as before any capture
        together(k, ref_op, ref_opt, ref_small)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = together(k, op, opt, small)
    data = [inputs(dtype, seed=20 + i) for i in range(4)]
    for i, d in enumerate(data):
        for name in ("x", "r", "lab", "adv"):
            k[name].copy_(d[name])
        torch.ones(1000, device="cuda").sum()  # eager work between the replays
        if i % 2:
            torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        kept = [None if t is None else t.clone() for t in got]
        # betas of 0: no bias correction is recorded that another step would have
        want = together(k, ref_op, ref_opt, ref_small)
        torch.cuda.synchronize()
        same(kept, want)
    for o in (op, opt, small, ref_op, ref_opt, ref_small):
        o.check()


def test_two_graphs_share_an_operator():
    """One operator in two graphs whose replays take turns."""
    k = inputs("bf16")
    op = P.LogProbs(300, 700, 64, dtype="bf16", top=4, grad=True)
    op.log_probs(k["x"], k["w"])
    torch.cuda.synchronize()
    graphs = []
    for rows in (300, 40):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, rows, op.log_probs(k["x"][:rows], k["w"], bias=k["bias"])))
    for seed in (31, 32):
        k["x"].copy_(inputs("bf16", seed=seed)["x"])
        for g, rows, got in graphs + graphs[::-1]:
            g.replay()
            kept = [t.clone() for t in got if t is not None]
            want = op.log_probs(k["x"][:rows], k["w"], bias=k["bias"])
            same(kept, [t for t in want if t is not None])


@pytest.mark.parametrize("given", [True, False])
def test_workspace_of_a_dropped_operator_is_not_given_away_early(given):
    k = inputs("f32")
    side = torch.cuda.Stream()
    op = P.LogProbs(300, 700, 64, top=4)
    size = op.ws_bytes
    op.log_probs(k["x"], k["w"])
    torch.cuda.synchronize()
    busy(side)
    if given:
        op.log_probs(k["x"], k["w"], stream=side)
    else:
        with torch.cuda.stream(side):
            op.log_probs(k["x"], k["w"])
    del op
    after = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert bool((after == 77).all())


def test_norms_and_clipping_on_two_streams_at_once():
    """The calls without memory of their own keep nothing between them."""
    k = inputs("f32", n=5000)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    gs = {s: [torch.full((100_003,), v, device="cuda"), torch.full((77,), v, device="cuda")]
          for s, v in ((a, 2.0), (b, 3.0))}
    want = {s: [g.clone() for g in gs[s]] for s in gs}
    for s in gs:
        P.clip_grads(want[s], 1.0)
    y = P.rms_norm(k["x"], k["gamma"], k["r"])
    torch.cuda.synchronize()
    busy(a), busy(b)
    got = {}
    for s in (a, b):
        with torch.cuda.stream(s):
            P.clip_grads(gs[s], 1.0)
            got[s] = P.rms_norm(k["x"], k["gamma"], k["r"])
    torch.cuda.synchronize()
    for s in (a, b):
        same(gs[s], want[s])
        same(got[s], y)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_head_of_each_norm_learns_and_its_gradient_is_the_difference(norm):
    """step's dx against differences of the mean loss; answers against the loss; a policy
    of advantages 1 is the step of the loss."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(40, 16, device="cuda", generator=g)
    lab = torch.randint(0, 7, (40,), device="cuda", generator=g).to(torch.int32)
    make = lambda **kw: P.SoftmaxHead(7, 16, 40, norm=norm, lr=1e-2, seed=1, **kw)  # noqa: E731
    head, other = make(top=7), make(top=7)
    mean = lambda x: head.loss(x, lab).double().mean().item()  # noqa: E731
    a = head.answers(x, lab)
    assert (a.logp + head.loss(x, lab)).abs().max().item() < 1e-5
    p = a.top_logp.double().exp()
    assert (p.sum(1) - 1).abs().max().item() < 1e-5  # all seven classes
    assert (a.entropy + (p * a.top_logp).sum(1)).abs().max().item() < 1e-5
    grads = []
    for i, j in ((0, 0), (17, 5), (39, 15)):
        e = torch.zeros_like(x)
        e[i, j] = 0.03
        # a step of 0.03: differences of order 0.03^2 and of the losses' rounding / 0.06
        grads.append((i, j, (mean(x + e) - mean(x - e)) / 0.06))
    loss, dx = head.step(x, lab)
    assert abs(loss.item() + a.logp.double().mean().item()) < 1e-6
    for i, j, d in grads:
        assert abs(dx[i, j].item() - d) < 2e-4
    b, dx2 = other.policy_step(x, lab, torch.ones(40, device="cuda"))
    assert (dx - dx2).abs().max().item() < 1e-6
    for u, v in zip(head.opt.params, other.opt.params):
        assert (u - v).abs().max().item() < 1e-4
    head.check(), other.check()
