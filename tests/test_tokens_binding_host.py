"""The tensor-level binding of the token operators on the CPU: tensors without a device and a library that only looks at what
it is called with.  Calls of several threads at a time, what they may share and what not."""
import threading

import pytest

torch = pytest.importorskip("torch")

import paper_2609_31938_b200 as ccv  # noqa: E402
from paper_2609_31938_b200 import tokens as tk  # noqa: E402


class Library:
    """Entry points whose calls meet at `gate` (all threads are inside one at that time) and note what they then find."""

    def __init__(self, threads=1):
        self.gate, self.seen, self.lock, self.inside = threading.Barrier(threads, timeout=20), [], threading.Lock(), 0

    def note(self, *what):
        self.gate.wait()
        with self.lock:
            self.seen.append((threading.current_thread().name, *what))
        self.gate.wait()
        return ccv.OK

    def ccv3d_kv_append(self, cache, batch, k, v, rot, q, q_out, heads, dt, status, stream):
        return self.note(batch, k.data, rot)

    def ccv3d_kv_attend(self, cache, batch, q, out, lse, heads, dt, scale, frame, window, ws, n, status, stream):
        return self.note(batch, q.data, ws)


@pytest.fixture
def binding(monkeypatch):
    """`tokens` on tensors of the CPU (their device number is -1)."""
    monkeypatch.setattr(tk, "_device", lambda: -1)
    monkeypatch.setattr(tk, "_stream", lambda dev: 7)
    monkeypatch.setattr(tk, "_capturing", lambda: False)
    monkeypatch.setattr(tk, "_synchronize", lambda dev: None, raising=False)
    monkeypatch.setattr(tk, "ccv3d_kv_attend_workspace", lambda *a: (ccv.OK, 512))

    def use(library):
        monkeypatch.setattr(tk, "lib", library)
        return library
    return use


def cache():
    return tk.PagedCache(torch.zeros(4, 2, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 2))


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def batch(n):
    return tk.TokenBatch(ints(0, n), ints(n), ints(0, 1)[None], n)


def together(*calls):
    threads = [threading.Thread(target=f, name=str(i)) for i, f in enumerate(calls)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()


def test_threads_share_a_rotation_and_a_batch(binding):
    """Two caches of a model, one rotation, one batch object: each call has its own positions and number of rows."""
    lib = binding(Library(2))
    rotary, shared = tk.Rotary(torch.ones(8, 32), torch.zeros(8, 32)), batch(9)
    k = [torch.zeros(n, 2, 64) for n in (5, 3)]
    pos = [torch.zeros(n, 1, dtype=torch.int32) for n in (5, 3)]
    caches = [cache(), cache()]
    together(*[lambda i=i: caches[i].append(k[i], k[i], shared, rotary, pos[i]) for i in (0, 1)])
    assert len(lib.seen) == 2
    for name, b, at, rot in lib.seen:
        i = int(name)
        assert at == k[i].data_ptr()
        assert rot.positions == pos[i].data_ptr() and rot.cos_table == rotary.cos.data_ptr()
        assert (b.tokens, b.max_new, b.new_start) == (5 - 2 * i, 9, shared.new_start.data_ptr())


def test_structs_of_a_batch_are_kept_but_not_without_end(binding):
    binding(Library())
    b = batch(9)
    first = b.c(5)
    assert b.c(5) is first and first.tokens == 5
    for n in range(1000):
        assert b.c(n).tokens == n
    assert len(b._c) <= 64 and first.tokens == 5


def test_threads_on_one_stream_do_not_use_one_scratch_at_a_time(binding):
    """An attend call is two launches that scratch connects: no other call may be given it in between."""
    class Slow(Library):
        busy, clashes, calls = set(), 0, 0

        def ccv3d_kv_attend(self, cache, batch, q, out, lse, heads, dt, scale, frame, window, ws, n, status, stream):
            with self.lock:
                self.clashes += ws in self.busy
                self.busy.add(ws)
                self.calls += 1
            threading.Event().wait(0.01)                 # between the launches
            with self.lock:
                self.busy.discard(ws)
            return ccv.OK

    lib = binding(Slow())
    c, b = cache(), batch(2)
    together(*[lambda: [c.attend(torch.zeros(2, 4, 64), b) for _ in range(8)] for _ in range(4)])
    assert lib.calls == 32 and lib.clashes == 0


def test_status_waits_for_every_stream(binding, monkeypatch):
    """Reports that arrive only once the device was waited for are read, and nothing is left for the next reading."""
    binding(Library())
    c, late = cache(), [4, 0]
    monkeypatch.setattr(tk, "_synchronize", lambda dev: c._status.bitwise_or_(late.pop(0) if late else 0), raising=False)
    c._status[0] = 1
    assert c.status() == 5
    assert c.status() == 0


def test_status_does_not_come_between_a_call_and_its_report(binding):
    """A call under way, in append or attend, is waited for: its report is neither missed nor wiped away."""
    class Reporting(Library):
        def ccv3d_kv_append(self, *a):
            return self.report(1)

        def ccv3d_kv_attend(self, *a):
            return self.report(2)

        def report(self, bit):
            entered.set()
            threading.Event().wait(0.1)
            c._status.bitwise_or_(bit)
            return ccv.OK

    binding(Reporting())
    c, b, x = cache(), batch(2), torch.zeros(2, 2, 64)
    for bit, call in ((1, lambda: c.append(x, x, b)), (2, lambda: c.attend(x, b))):
        entered = threading.Event()
        t = threading.Thread(target=call)
        t.start()
        assert entered.wait(20)
        assert c.status() == bit
        t.join()
        assert c.status() == 0


def test_numbers_past_32_bits_are_refused(binding):
    """They would arrive as other numbers: a window of 2^32 as 0."""
    binding(Library())
    c, b, x = cache(), batch(2), torch.zeros(2, 4, 64)
    for kw in (dict(window=1 << 32), dict(window=1 << 31), dict(frame=1 << 32), dict(frame=(1 << 32) + 1), dict(window=-(1 << 32))):
        with pytest.raises(ValueError):
            c.attend(x, b, **kw)
    assert c.attend(x, b, frame=(1 << 31) - 1, window=(1 << 31) - 1).shape == x.shape
    for n in (1 << 31, (1 << 32) + 1):
        with pytest.raises(ValueError):
            tk.TokenBatch(ints(0, 2), ints(2), ints(0, 1)[None], n)
    with pytest.raises(ValueError):
        tk.gated_norm(torch.zeros(2, 4), rows_per_group=1 << 32)
    with pytest.raises(ValueError):
        tk.gated_norm(torch.zeros(1, 4).expand((1 << 32) + 2, 4), want_h=False, out_r=torch.zeros(1, 4).expand((1 << 32) + 2, 4))
