"""What the softmax head's classes launch, in which order: torch's streams and the C
calls replaced by a record of them, on the CPU.

Every call reads and writes memory on one stream.  Each stream has a vector clock
(what it is known to run after); a wait joins two of them, a synchronisation joins the
host's.  An access that is not known to run after the last write of its memory, or a
write that is not known to run after the reads before it, is a Race.  Also kept: the
stream that an allocation belongs to and those that it was recorded on
(Tensor.record_stream), and which streams are being captured into a graph.
"""
import bisect

import torch

import paper_2307_14490_amd as P
from paper_2307_14490_amd import head


class Race(AssertionError):
    pass


class Stream:
    def __init__(self, order, ptr):
        self.order, self.cuda_stream, self.clock, self.capturing = order, ptr, {}, False
        self.device = torch.device("cuda", 0)

    def wait_stream(self, other):
        if self.capturing and not other.capturing:
            raise RuntimeError("a captured stream waits for work that is not captured")
        _join(self.clock, other.clock)

    def synchronize(self):
        if self.capturing:
            raise RuntimeError("a captured stream is synchronised")
        _join(self.order.host, self.clock)


def _join(a, b):
    for k, t in b.items():
        a[k] = max(a.get(k, 0), t)


class Tensor(torch.Tensor):
    """A tensor on the CPU that says it is on the GPU, whose operations are recorded."""
    order = None
    is_cuda = property(lambda t: True)
    device = property(lambda t: torch.device("cuda", 0))

    def record_stream(self, stream):
        self.order.memory(self.data_ptr()).recorded.add(stream.cuda_stream)

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        out = super().__torch_function__(func, types, args, kwargs or {})
        cls.order.torch_call(func.__name__, args, out)
        return out


class Memory:
    def __init__(self, base, size, stream):
        self.base, self.size, self.stream = base, size, stream
        self.recorded, self.used = set(), set()
        self.write, self.reads = None, []


class Order:
    """Use as a context; `streams` are extra streams."""

    def __init__(self, monkeypatch):
        self.host, self.tensors, self.bases, self.memories = {}, [], [], {}
        self.default = Stream(self, 0)
        self.current = [self.default]
        self.made = 0
        self.lib = P.load()
        Tensor.order = self
        set_ = monkeypatch.setattr
        for name in ("empty", "zeros", "ones", "randn", "full"):
            set_(torch, name, self._factory(getattr(torch, name)))
        real = torch.Generator
        set_(torch, "Generator", lambda device=None: real())
        set_(torch.cuda, "current_device", lambda: 0)
        set_(torch.cuda, "current_stream", lambda device=None: self.current[-1])
        set_(torch.cuda, "is_current_stream_capturing", lambda: self.current[-1].capturing)
        set_(torch.cuda, "stream", self.on)
        set_(head, "_current", lambda device: self.current[-1].cuda_stream)
        set_(head, "load", lambda: self)

    # -- streams ---------------------------------------------------------------
    def stream(self):
        self.made += 1
        return Stream(self, 1000 + self.made)

    def on(self, stream):
        order = self

        class On:
            def __enter__(self):
                order.current.append(stream)

            def __exit__(self, *error):
                order.current.pop()
        return On()

    def _by_ptr(self, ptr):
        return next(s for s in [self.default, *self.current, *self.seen] if s.cuda_stream == ptr)

    seen = ()  # streams that calls name by their pointer

    # -- memory ----------------------------------------------------------------
    def _factory(self, real):
        def make(*a, device=None, generator=None, **kw):
            if generator is not None:
                kw["generator"] = generator
            t = real(*a, **kw).as_subclass(Tensor)
            self.new(t, written=real.__name__ != "empty")
            return t
        return make

    def new(self, t, written):
        self.tensors.append(t)  # addresses are not given out again
        size = t.untyped_storage().nbytes()
        base = t.untyped_storage().data_ptr()
        if size:
            bisect.insort(self.bases, base)
            self.memories[base] = Memory(base, size, self.current[-1].cuda_stream)
            if written:
                self.access(self.current[-1], base, True, "its first values")

    def memory(self, ptr):
        at = bisect.bisect_right(self.bases, ptr) - 1
        m = self.memories[self.bases[at]] if at >= 0 else None
        assert m is not None and ptr < m.base + max(m.size, 1), "not an allocation"
        return m

    def access(self, stream, ptr, write, what=""):
        if not ptr:
            return
        m = self.memory(ptr)
        m.used.add(stream.cuda_stream)
        _join(stream.clock, self.host)
        key = stream.cuda_stream
        stream.clock[key] = stream.clock.get(key, 0) + 1
        before = [m.write] if m.write else []
        if write:
            before += m.reads
        for k, t, by in before:
            if stream.clock.get(k, 0) < t:
                raise Race(f"{what} on stream {key} is not behind {by} on stream {k}")
        now = (key, stream.clock[key], what)
        if write:
            m.write, m.reads = now, []
        else:
            m.reads.append(now)

    def torch_call(self, name, args, out):
        stream = self.current[-1]
        given = [a for a in args if isinstance(a, Tensor)]
        if name == "item":
            self.access(stream, given[0].data_ptr(), False, name)
            stream.synchronize()
        elif name == "__setitem__" or (name.endswith("_") and not name.endswith("__")):
            for a in given[1:]:
                self.access(stream, a.data_ptr(), False, name)
            self.access(stream, given[0].data_ptr(), True, name)
        elif isinstance(out, Tensor) and out.numel():
            base = out.untyped_storage().data_ptr()
            if all(a.untyped_storage().data_ptr() != base for a in given):
                for a in given:
                    self.access(stream, a.data_ptr(), False, name)
                self.new(out, written=True)

    def owned_elsewhere(self, *tensors):
        """Streams that use the memory of these tensors, though it neither belongs to
        them nor is recorded on them."""
        out = set()
        for t in tensors:
            m = self.memory(t.data_ptr())
            out |= m.used - m.recorded - {m.stream}
        return out

    # -- the C calls -----------------------------------------------------------
    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.lib, name)
        if not name.startswith("huge_"):
            raise AttributeError(name)

        def call(*a):
            reads, writes, ptr = getattr(self, "_" + name)(*a)
            stream = self._by_ptr(ptr)
            for p in reads:
                self.access(stream, p, False, name)
            for p in writes:
                self.access(stream, p, True, name)
            return 0
        return call

    @staticmethod
    def _huge_layer_norm(x, ldx, n, dim, code, g, b, eps, y, ldy, mean, rstd, s):
        return (x, g, b), (y, mean, rstd), s

    @staticmethod
    def _huge_layer_norm_backward(dy, ldy, x, ldx, n, dim, code, g, mean, rstd, dx, ld, dg, db, ws,
                                  size, s):
        return (dy, x, g, mean, rstd), (dx, dg, db, ws), s

    @staticmethod
    def _huge_softmax_loss(c, h, ldh, n, w, ldw, bias, labels, weights, loss, lse, total, status,
                           ws, size, s):
        return (h, w, bias, labels, weights), (loss, lse, total, status, ws), s

    @staticmethod
    def _huge_softmax_grad(c, h, ldh, n, w, ldw, bias, labels, weights, lse, scale, dh, dw, db,
                           status, ws, size, s):
        return (h, w, bias, labels, weights, lse), (dh, dw, db, status, ws), s

    @staticmethod
    def _huge_adamw_step(c, ts, count, status, s):
        return [t.d_grad for t in ts], [p for t in ts for p in (t.d_param, t.d_state)] + [status], s

    @staticmethod
    def _huge_adamw_get_state(ts, count, kind, m, v, s):
        return [t.d_state for t in ts], [m[0], v[0]], s

    @staticmethod
    def _huge_adamw_set_state(ts, count, kind, m, v, s):
        return [p for q in (m, v) for p in q[:count]], [t.d_state for t in ts], s
