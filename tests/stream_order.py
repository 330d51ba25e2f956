"""Which accesses of the torch layer's buffers are ordered, without a GPU.

``watch(monkeypatch)`` replaces torch's streams by ones that only keep clocks, and the library's calls by ones that only
note the buffers they take. Every torch operation and every library call then is an access on the stream that is current
(or whose handle the call got), with the storages that it reads and writes, and ``races()`` lists the pairs of accesses
of one storage, at least one of them a write, of which neither is ordered before the other. Tensors are small ones on
the CPU.
"""

import contextlib
import ctypes

import torch
from torch.utils._python_dispatch import TorchDispatchMode
from torch.utils._pytree import tree_leaves

import paper_2609_08131_gb300.api as api

# of each library call: the position of its stream, and of the arguments that it writes
CALLS = {
    "jacap_append": (12, (7, 8, 9, 10, 11)),
    "jacap_append_path": (15, (10, 11, 12, 13, 14)),
    "jacap_attend": (9, (5, 6, 7)),
    "jacap_evict_weights": (14, (1, 2, 6, 7, 8, 9, 11, 12)),
    "jacap_rotate": (9, (7, 8)),
    "jacap_score_stats": (9, (6, 7)),
    "jacap_select_compact_inplace": (11, (3, 4, 5, 6, 7, 9)),
    "jacap_select_weights": (16, (6, 7, 10, 11, 12, 13, 14)),
    "jacap_stats_update": (5, (3, 4)),
    "jacap_weigh": (9, (4, 6, 7)),
}


class Stream:
    def __init__(self, order, name, handle):
        self.order, self.name, self.cuda_stream, self.device = order, name, handle, torch.device("cpu")
        self.clock = {}  # per stream: how many of its accesses come before what is next here

    def wait_stream(self, other):
        for name, n in other.clock.items():
            self.clock[name] = max(self.clock.get(name, 0), n)

    def __eq__(self, other):
        return isinstance(other, Stream) and self.cuda_stream == other.cuda_stream

    def __hash__(self):
        return self.cuda_stream


class Event:
    def __init__(self, stream):
        self.stream = Stream(stream.order, stream.name, stream.cuda_stream)
        self.stream.clock = dict(stream.clock)

    def wait(self):
        self.stream.order.current.wait_stream(self.stream)


class Order(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.main, self.side = Stream(self, "current", 1), Stream(self, "side", 2)
        self.current, self.capturing = self.main, False
        self.other, self.device = Stream(self, "other device's", 3), None  # (None: the tensors')
        self.accesses = []  # (what, stream's name, its number there, clock, reads, writes, captured, arguments)
        self.held = {}      # address -> (end, storage's tensor): kept, so that no address comes back

    # ---- accesses
    def note(self, what, stream, reads, writes, args=()):
        number = stream.clock.get(stream.name, 0)
        stream.clock[stream.name] = number + 1
        self.accesses.append((what, stream.name, number, dict(stream.clock), frozenset(reads), frozenset(writes),
                              self.capturing, args))

    def storage(self, t):
        at = t.untyped_storage().data_ptr()
        if at:
            self.held[at] = (at + t.untyped_storage().nbytes(), t)
        return at

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        reads = {self.storage(t) for t in tree_leaves((args, kwargs)) if isinstance(t, torch.Tensor)}
        results = {self.storage(t) for t in tree_leaves(out) if isinstance(t, torch.Tensor)}
        name = func.overloadpacket.__name__
        if not func._schema.is_mutable and results & reads:
            return out  # a view
        if "empty" in name:
            return out  # an allocation
        self.note(name, self.current, reads, {self.storage(args[0])} if func._schema.is_mutable else results)
        return out

    def buffer(self, pointer):
        for at, (end, _) in self.held.items():
            if at <= pointer < end:
                return at
        return None

    def library(self, name):
        place, written = CALLS[name]

        def pointers(x, written=False):
            if isinstance(x, ctypes.Structure):
                for field, kind in x._fields_:
                    if kind is ctypes.c_void_p and not (written and field == "x"):
                        yield getattr(x, field) or 0
            elif isinstance(x, ctypes.c_void_p):
                yield x.value or 0
            elif isinstance(x, int) and not isinstance(x, bool):
                yield x

        def call(*args):
            assert self.device is None, f"{name} with another device current"
            handle = args[place].value if isinstance(args[place], ctypes.c_void_p) else args[place]
            stream = self.main if handle == self.main.cuda_stream else self.side
            assert handle == stream.cuda_stream, name
            reads, writes = set(), set()
            for i, x in enumerate(args):
                reads |= {self.buffer(p) for p in pointers(x) if p > 1 << 16} - {None}
                if i in written:
                    writes |= {self.buffer(p) for p in pointers(x, True) if p > 1 << 16} - {None}
            self.note(name, stream, reads, writes, args)
            return api.JACAP_OK

        return call

    # ---- what is not ordered
    def races(self):
        out = []
        for j, (what, stream, _, clock, reads, writes, _, _) in enumerate(self.accesses):
            for other, on, earlier, _, r, w, _, _ in self.accesses[:j]:
                if on != stream and clock.get(on, 0) <= earlier and (w & (reads | writes) or writes & r):
                    out.append(f"{other} on the {on} stream, {what} on the {stream} one")
        return out

    def calls(self, name):
        return [a for a in self.accesses if a[0] == name]


@contextlib.contextmanager
def watch(monkeypatch):
    order = Order()

    @contextlib.contextmanager
    def on(stream):
        before, order.current = order.current, stream
        yield
        order.current = before

    @contextlib.contextmanager
    def device(d):
        before, order.device = order.device, None
        yield
        order.device = before

    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_stream",
                  lambda d=None: order.current if order.device is None or d is not None else order.other)
        m.setattr(torch.cuda, "current_device", lambda: order.device)
        m.setattr(torch.cuda, "device", device)
        m.setattr(torch.cuda, "stream", on)
        m.setattr(torch.cuda, "is_current_stream_capturing", lambda: order.capturing)
        m.setattr(torch._C, "_cuda_getDevice", lambda: order.device, raising=False)
        m.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: order.current.cuda_stream, raising=False)
        m.setattr(api, "_made", lambda device: Event(order.current), raising=False)
        for name in CALLS:
            m.setattr(api, name, order.library(name))
        with order:
            yield order
