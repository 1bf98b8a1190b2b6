"""The softmax head on more than one stream, without a GPU: what its classes launch is
ordered, on whatever stream they are called (stream_order records and checks it)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from stream_order import Order, Race  # noqa: E402


@pytest.fixture
def order(monkeypatch):
    o = Order(monkeypatch)
    o.seen = [o.stream(), o.stream()]
    return o


def batch(order, stream):
    """Rows and labels made on the stream that the head is to use."""
    with order.on(stream):
        return torch.randn(6, 8), torch.zeros(6, dtype=torch.int32)


def test_the_record_finds_a_missing_wait(order):
    a, b = order.seen
    with order.on(a):
        t = torch.zeros(4)
    with order.on(b):
        with pytest.raises(Race):
            t + 1
        b.wait_stream(a)
        t + 1
    with order.on(a), pytest.raises(Race):
        t.zero_()  # b still reads
    b.synchronize()
    with order.on(a):
        t.zero_()
    assert order.owned_elsewhere(t) == {b.cuda_stream}
    t.record_stream(b)
    assert not order.owned_elsewhere(t)


def test_head_steps_on_a_stream_of_the_callers(order):
    """Its parameters were filled on the constructor's stream; the mean loss that a step
    returns is formed on the step's stream."""
    a, _ = order.seen
    head = P.SoftmaxHead(5, 8, 6)
    x, lab = batch(order, a)
    for _ in range(2):
        loss, dx = head.step(x, lab, stream=a)
        with order.on(a):
            loss + 1, dx + 1
    assert head.loss(x, lab, stream=a).shape == (6,)


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_head_takes_turns_between_streams(order, states):
    a, b = order.seen
    head = P.SoftmaxHead(5, 8, 6, states=states)
    data = {s: batch(order, s) for s in (a, b, order.default)}
    for s in (a, b, order.default, a, order.default, b):
        loss, _ = head.step(*data[s], stream=s)
        with order.on(s):
            loss + 1
        with order.on(s):  # ... and as the current stream
            head.step(*data[s])
    for s in (order.default, a):  # the parameters of the last step
        head.loss(*data[s], stream=s)
        with order.on(s):
            head.gamma + 1


@pytest.mark.parametrize("given", [True, False])
def test_memory_of_the_operators_is_kept_for_every_stream(order, given):
    """Workspace, status word, moments and parameters, whether the stream is an argument
    or the current one: dropped, they are given to others only behind its work."""
    a, b = order.seen
    head = P.SoftmaxHead(5, 8, 6)
    for s in (a, b):
        x, lab = batch(order, s)
        if given:
            head.step(x, lab, stream=s)
        else:
            with order.on(s):
                head.step(x, lab)
    own = [head.op._ws, head.op.status, head.opt.states, head.opt.status, head.total,
           *head.opt.params]
    assert len(own) == 9
    assert not order.owned_elsewhere(*own)


def test_arguments_are_kept_for_the_stream_that_is_given(order):
    a, _ = order.seen
    x, lab = batch(order, order.default)
    head = P.SoftmaxHead(5, 8, 6)
    a.wait_stream(order.default)
    head.step(x, lab, stream=a)
    assert not order.owned_elsewhere(x, lab)


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_moments_are_those_of_the_last_step(order, states):
    """values() on one stream after a step on another, and a step after values()."""
    a, b = order.seen
    with order.on(a):
        opt = P.AdamW([torch.zeros(300)], states=states)
        grad = torch.ones(300)
    opt.step([grad], stream=a)
    for s in (b, None):
        m, v = opt.values(stream=s)
        with order.on(s or order.default):
            m[0] + v[0]
    opt.step([grad], stream=a)


def test_a_reported_error_is_cleared_before_the_next_call(order):
    """check() on one stream between two calls on another."""
    a, _ = order.seen
    op = P.SoftmaxLoss(6, 5, 8)
    x, lab = batch(order, a)
    w, _ = batch(order, a)
    w = w[:5]
    with order.on(a):
        op.loss(x, w, lab)
        op.status.fill_(-2)  # as a kernel would
    with pytest.raises(P.HugeError):
        op.check()
    op.loss(x, w, lab, stream=a)
    op.check()


def test_capture_on_a_stream_of_its_own(order):
    """A call recorded into a graph waits for no work outside of it, and for the other
    streams of the same graph."""
    a, b = order.seen
    op = P.SoftmaxLoss(6, 5, 8)
    x, lab = batch(order, order.default)
    w = batch(order, order.default)[0][:5]
    op.loss(x, w, lab)
    order.default.synchronize()  # as before any capture
    a.capturing = True
    op.loss(x, w, lab, stream=a)
    b.capturing = True  # forked from a
    op.loss(x, w, lab, stream=b)
    op.loss(x, w, lab, stream=a)
    a.capturing = b.capturing = False
    op.loss(x, w, lab)
    op.check()


def test_parameters_that_share_memory_are_refused(order):
    """One launch updates all: elements listed twice would be read and written by two
    workgroups at once."""
    t = torch.zeros(300)
    for params in ([t, t], [t[:200], t[199:]], [t[100:101], torch.zeros(5), t]):
        with pytest.raises(ValueError):
            P.AdamW(params)
    P.AdamW([t[:200], t[200:], torch.zeros(0), torch.zeros(0)])


def test_a_stream_of_another_device_is_refused(order):
    """Before anything is launched or allocated there."""
    far = order.stream()
    order.seen.append(far)
    far.device = torch.device("cuda", 1)
    x, lab = batch(order, order.default)
    g = torch.ones(8)
    head = P.SoftmaxHead(5, 8, 6)
    opt = P.AdamW([torch.zeros(6, 8)])
    for call in (lambda: P.layer_norm(x, g, g, stream=far), lambda: head.loss(x, lab, stream=far),
                 lambda: head.step(x, lab, stream=far), lambda: opt.step([x], stream=far),
                 lambda: opt.values(stream=far), lambda: head.op.loss(x, x[:5], lab, stream=far)):
        with pytest.raises(ValueError):
            call()
    assert not far.clock and opt.steps == 0
