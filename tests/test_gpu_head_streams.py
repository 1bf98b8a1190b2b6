"""The softmax head on more than one stream: the same bits as on one.  The streams are
kept busy with other work, so that what is not ordered would come too early."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def busy(stream=None):
    """Some milliseconds of work on a stream."""
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        a = torch.ones((2048, 2048), device="cuda")
        for _ in range(20):
            a = a @ a * 1e-4


def head_case(dtype, n=300, classes=700, dim=64):
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(n, dim, device="cuda", generator=g)
    lab = torch.randint(0, classes, (n,), device="cuda", generator=g).to(torch.int32)
    torch.cuda.synchronize()
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32), lab


@pytest.mark.parametrize("dtype,states", [("f32", "f32"), ("bf16", "q8")])
def test_head_takes_turns_between_streams(dtype, states):
    x, lab = head_case(dtype)
    torch.cuda.synchronize()
    say(f"head on two streams, {dtype}, moments {states}")

    def train(streams):
        busy()
        head = P.SoftmaxHead(700, 64, 300, dtype=dtype, lr=1e-2, states=states, seed=2)
        got = []
        for s in streams:
            busy(s)
            got.append(head.step(x, lab, stream=s))
        torch.cuda.synchronize()
        head.check()
        return [t for pair in got for t in pair] + list(head.opt.params)

    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    want = train([None] * 6)
    for u, v in zip(want, train([a, b, None, a, None, b])):
        assert torch.equal(u, v)


@pytest.mark.parametrize("given", [True, False])
def test_workspace_of_a_dropped_operator_is_not_given_away_early(given):
    """The operator goes while its call waits on a busy stream: tensors made after it
    keep their values."""
    x, lab = head_case("f32")
    w = torch.randn(700, 64, device="cuda")
    side = torch.cuda.Stream()
    op = P.SoftmaxLoss(300, 700, 64)
    size = op.ws_bytes
    op.loss(x, w, lab)
    torch.cuda.synchronize()
    busy(side)
    if given:
        op.loss(x, w, lab, stream=side)
    else:
        with torch.cuda.stream(side):
            op.loss(x, w, lab)
    del op
    after = torch.full((size + 256,), 77, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert bool((after == 77).all())


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_moments_are_those_of_the_last_step(states):
    p, g = torch.zeros(5000, device="cuda"), torch.randn(5000, device="cuda")
    want = P.AdamW([p], states=states)
    want.step([g])
    m, v = want.values()
    opt = P.AdamW([p.clone()], states=states)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    opt.step([g], stream=side)
    m2, v2 = opt.values()
    m2, v2 = m2[0].clone(), v2[0].clone()
    torch.cuda.synchronize()
    assert torch.equal(m2, m[0]) and torch.equal(v2, v[0])


def test_an_error_on_another_stream_is_reported_once():
    x, lab = head_case("f32")
    w = torch.randn(700, 64, device="cuda")
    op, side = P.SoftmaxLoss(300, 700, 64), torch.cuda.Stream()
    bad = lab.clone()
    bad[5] = 700
    torch.cuda.synchronize()
    for _ in range(3):
        busy(side)
        op.loss(x, w, bad, stream=side)
        busy()
        with pytest.raises(P.HugeError):
            op.check()
        op.loss(x, w, lab, stream=side)
        op.check()
        op.loss(x, w, bad, stream=side)
        with pytest.raises(P.HugeError):
            op.check()


def test_capture_after_work_on_the_current_stream():
    """Recorded on a stream that the operator has not seen, replayed between the
    program's own calls of it."""
    x, lab = head_case("bf16")
    w = (torch.randn(700, 64, device="cuda") * 0.2).bfloat16()
    op = P.SoftmaxLoss(300, 700, 64, dtype="bf16")

    def both():
        loss, lse = op.loss(x, w, lab)
        return (loss, *op.grad(x, w, lab, lse))

    want = [t.clone() for t in both()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(3):
        for t in held:
            t.fill_(0)
        graph.replay()
        for u, v in zip(want, held):
            assert torch.equal(u, v)
        for u, v in zip(want, both()):
            assert torch.equal(u, v)
    op.check()
