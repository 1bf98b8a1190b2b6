"""What normalises, answers and clips on more than one stream, without a GPU: launches are
recorded and checked as in test_head_streams."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
import stream_order  # noqa: E402


class Order(stream_order.Order):
    """With the C calls of this module's operators."""

    def __init__(self, monkeypatch):
        super().__init__(monkeypatch)
        monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)

    @staticmethod
    def _huge_rms_norm(x, ldx, res, ldr, n, dim, code, g, eps, total, ldt, y, ldy, codes, ldc,
                       scales, lds, rstd, s):
        return (x, res, g), (total, y, codes, scales, rstd), s

    @staticmethod
    def _huge_rms_norm_backward(dy, ldy, total, ldt, dt, lddt, n, dim, code, g, rstd, dx, ldx, dg,
                                ws, size, s):
        return (dy, total, dt, g, rstd), (dx, dg, ws), s

    @staticmethod
    def _huge_quantise_rows(x, ldx, n, dim, code, codes, ldc, scales, lds, s):
        return (x,), (codes, scales), s

    @staticmethod
    def _huge_dequantise_rows(codes, ldc, scales, lds, n, dim, y, ldy, code, s):
        return (codes, scales), (y,), s

    @staticmethod
    def _huge_log_probs(c, h, ldh, n, w, ldw, scales, lds, bias, labels, logp, entropy, lse, ids,
                        best, status, ws, size, s):
        return (h, w, scales, bias, labels), (logp, entropy, lse, ids, best, status, ws), s

    @staticmethod
    def _huge_log_probs_grad(c, h, ldh, n, w, ldw, bias, labels, lse, entropy, dl, de, dh, dw, db,
                             status, ws, size, s):
        return (h, w, bias, labels, lse, entropy, dl, de), (dh, dw, db, status, ws), s

    @staticmethod
    def _huge_grad_norm(ts, count, norm, ws, size, s):
        return [ts[k].d_grad for k in range(count)], (norm, ws), s

    @staticmethod
    def _huge_clip_grads(ts, count, most, norm, ws, size, s):
        return (), [ts[k].d_grad for k in range(count)] + [norm, ws], s

    @staticmethod
    def _huge_adamw_step_clipped(c, ts, count, most, norm, status, ws, size, s):
        return [t.d_grad for t in ts], \
            [p for t in ts for p in (t.d_param, t.d_state)] + [norm, status, ws], s


@pytest.fixture
def order(monkeypatch):
    o = Order(monkeypatch)
    o.seen = [o.stream(), o.stream()]
    return o


def batch(order, stream):
    with order.on(stream):
        return torch.randn(6, 8), torch.zeros(6, dtype=torch.int32), torch.ones(6)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_head_answers_and_trains_on_streams_in_turn(order, norm):
    a, b = order.seen
    head = P.SoftmaxHead(5, 8, 6, norm=norm, max_norm=1.0, top=2)
    data = {s: batch(order, s) for s in (a, b, order.default)}
    for s in (a, b, order.default, a, order.default, b):
        x, lab, adv = data[s]
        loss, dx = head.step(x, lab, stream=s)
        found = head.answers(x, lab, stream=s)
        before, dx2 = head.policy_step(x, lab, adv, 0.1, stream=s)
        with order.on(s):  # ready there, and as the current stream
            for t in (loss, dx, dx2, *found, *before, head.norm_before):
                t + 1
            head.policy_step(x, lab, adv)
            head.answers(x)
    for s in (order.default, a):  # the parameters of the last step
        head.loss(*data[s][:2], stream=s)
        with order.on(s):
            head.gamma + 1


@pytest.mark.parametrize("given", [True, False])
def test_memory_is_kept_for_every_stream(order, given):
    a, b = order.seen
    head = P.SoftmaxHead(5, 8, 6, norm="rms", max_norm=1.0, top=2)
    for s in (a, b):
        x, lab, adv = batch(order, s)
        if given:
            head.policy_step(x, lab, adv, stream=s)
        else:
            with order.on(s):
                head.policy_step(x, lab, adv)
    own = [head.answering._ws, head.answering.status, head.opt.states, head.opt._norm_ws,
           head.opt.status, *head.opt.params]
    assert len(own) == 8
    assert not order.owned_elsewhere(*own)


def test_arguments_are_kept_for_the_stream_that_is_given(order):
    a, _ = order.seen
    x, lab, adv = batch(order, order.default)
    g = torch.ones(8)
    res, grads = torch.randn(6, 8), [torch.ones(5), torch.ones(3)]
    op = P.LogProbs(6, 6, 8, top=2, grad=True)
    eight = P.LogProbs(6, 6, 8, dtype="q8", top=2)
    half = torch.zeros(6, 8, dtype=torch.bfloat16)
    a.wait_stream(order.default)
    _, total, rstd = P.rms_norm(x, g, res, stream=a)
    P.rms_norm_backward(x, total, g, rstd, res, stream=a)
    q = P.q8_rows(x, stream=a)
    P.q8_values(q, stream=a)
    found = op.log_probs(x, res, lab, stream=a)
    op.grad(x, res, found, lab, adv, adv, stream=a)
    eight.log_probs(half, q, stream=a)
    P.grad_norm(grads, stream=a)
    P.clip_grads(grads, 1.0, stream=a)
    assert not order.owned_elsewhere(x, lab, adv, g, res, total, rstd, half, *q, *grads, *found[:3])


def test_calls_without_memory_of_their_own_do_not_wait(order):
    """Two streams at once: each has its own workspace."""
    for s in order.seen:
        x, _, _ = batch(order, s)
        with order.on(s):
            g = torch.ones(8)
            y, total, rstd = P.rms_norm(x, g, x)
            P.rms_norm_backward(x, total, g, rstd)
            P.clip_grads([y], 1.0)
            P.grad_norm([y, total])


def test_capture_on_a_stream_of_its_own(order):
    a, b = order.seen
    head = P.SoftmaxHead(5, 8, 6, norm="rms", max_norm=1.0, top=2)
    x, lab, adv = batch(order, order.default)
    head.policy_step(x, lab, adv)
    order.default.synchronize()  # as before any capture
    a.capturing = True
    head.policy_step(x, lab, adv, stream=a)
    b.capturing = True  # forked from a
    head.answers(x, stream=b)
    a.capturing = b.capturing = False
    head.answers(x)
    head.check()


def test_a_stream_of_another_device_is_refused(order):
    """Before anything is launched or allocated there."""
    far = order.stream()
    order.seen.append(far)
    far.device = torch.device("cuda", 1)
    x, lab, adv = batch(order, order.default)
    g = torch.ones(8)
    op = P.LogProbs(6, 6, 8, grad=True)
    found = op.log_probs(x, x, lab)
    opt = P.AdamW([torch.zeros(6, 8)])
    q = P.q8_rows(x)
    for call in (lambda: P.rms_norm(x, g, stream=far), lambda: op.log_probs(x, x, stream=far),
                 lambda: op.grad(x, x, found, lab, adv, stream=far),
                 lambda: opt.step([x], max_norm=1.0, stream=far),
                 lambda: P.grad_norm([x], stream=far), lambda: P.clip_grads([x], 1.0, stream=far),
                 lambda: P.q8_rows(x, stream=far), lambda: P.q8_values(q, stream=far)):
        with pytest.raises(ValueError):
            call()
    assert not far.clock and opt.steps == 0


def test_gradients_that_share_memory_are_not_clipped(order):
    """In place, an element listed twice would be scaled twice; their norm is no harm."""
    t = torch.zeros(300)
    for grads in ([t, t], [t[:200], t[199:]]):
        with pytest.raises(ValueError):
            P.clip_grads(grads, 1.0)
        P.grad_norm(grads)


def test_heads_refuse(order):
    for kw in (dict(norm="batch"), dict(max_norm=0.0), dict(max_norm=float("nan"))):
        with pytest.raises(ValueError):
            P.SoftmaxHead(5, 8, 6, **kw)
    head = P.SoftmaxHead(5, 8, 6)
    x, lab, adv = batch(order, order.default)
    for call in (lambda: head.answers(x), lambda: head.policy_step(x, lab, adv)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.SoftmaxHead(5, 8, 6, top=2).policy_step(x, lab, torch.ones(5))
    opt = P.AdamW([torch.zeros(5)])
    for most in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError):
            opt.step([torch.zeros(5)], max_norm=most)


def test_arguments_that_do_not_fit_are_refused(order):
    x, lab, adv = batch(order, order.default)
    g, half = torch.ones(8), torch.zeros(6, 8, dtype=torch.bfloat16)
    op, eight = P.LogProbs(6, 6, 8, grad=True), P.LogProbs(6, 6, 8, dtype="q8")
    found, q = op.log_probs(x, x, lab), P.q8_rows(x)
    for call in (lambda: P.rms_norm(x, None), lambda: P.rms_norm(x, g, half),
                 lambda: P.rms_norm_backward(half, x, g, adv), lambda: op.log_probs(half, x),
                 lambda: op.log_probs(x, half), lambda: op.grad(x, x, found, dlogp=adv),
                 lambda: eight.log_probs(half, half), lambda: eight.log_probs(x, q),
                 lambda: eight.log_probs(half, (x, q.scales)), lambda: eight.grad(half, q, found),
                 lambda: P.q8_values((half, q.scales)), lambda: P.q8_rows(lab.view(2, 3))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: P.rms_norm(x, torch.ones(7)), lambda: P.rms_norm(x, g, x[:5]),
                 lambda: P.rms_norm_backward(x, x, g, adv[:5]),
                 lambda: P.rms_norm_backward(x[:5], x, g, adv),
                 lambda: P.rms_norm_backward(x, x, g, adv, x[:5]),
                 lambda: op.log_probs(x, x[:5]), lambda: op.log_probs(x, x, lab[:5]),
                 lambda: op.log_probs(x, x, bias=torch.ones(5)),
                 lambda: op.grad(x, x, found, lab, adv[:5]),
                 lambda: eight.log_probs(half, P.Q8Rows(q.codes, q.scales[:5])),
                 lambda: eight.log_probs(half, P.Q8Rows(q.codes[:5], q.scales[:5]))):
        with pytest.raises(ValueError):
            call()
