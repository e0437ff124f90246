"""The binding of the products, decaying states and group norms on the CPU: tensors without a device and a library that only looks at
what it is called with."""
import threading

import pytest

torch = pytest.importorskip("torch")

import paper_2609_31938_b200 as ccv  # noqa: E402
from paper_2609_31938_b200 import tokens as tk  # noqa: E402


def test_status_words_refuse_what_is_none():
    assert ccv.lib.ccv3d_linear_status_word(None) == ccv.ERR_INVALID_ARG
    assert ccv.ccv3d_take_status(None)[0] == ccv.ERR_INVALID_ARG
    assert ccv.ccv3d_take_status(6)[0] == ccv.ERR_ALIGNMENT


class Reporting:
    """Calls that report a while after they were made."""

    def __init__(self, word):
        self.word, self.entered = word, threading.Event()

    def late(self, *a):
        self.entered.set()
        threading.Event().wait(0.1)
        self.word[0] |= 8
        return ccv.OK

    ccv3d_linear = ccv3d_decay_attend = late


@pytest.fixture
def binding(monkeypatch):
    """`tokens` on tensors of the CPU (their device number is -1)."""
    monkeypatch.setattr(tk, "_device", lambda: -1)
    monkeypatch.setattr(tk, "_stream", lambda dev: 7)
    monkeypatch.setattr(tk, "_capturing", lambda: False)
    monkeypatch.setattr(tk, "_synchronize", lambda dev: None)
    monkeypatch.setattr(tk, "_scratch", lambda *a: (None, None, 0))

    def use(library):
        monkeypatch.setattr(tk, "lib", library)
        return library
    return use


def meanwhile(lib, call, status):
    """What `status` says while a call is under way in another thread, and once more after it."""
    t = threading.Thread(target=call)
    t.start()
    assert lib.entered.wait(20)
    during = status()
    t.join()
    return during, status()


def test_status_does_not_come_between_a_call_on_states_and_its_report(binding):
    memory = tk.DecayMemory(torch.zeros(2, 2, 64, 64))
    lib = binding(Reporting(memory._status))
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    batch, x = tk.StreamBatch(ints(0, 3), ints(0), 3), torch.zeros(3, 2, 64)
    assert meanwhile(lib, lambda: memory.attend(x, x, x, torch.zeros(3, 2), batch), memory.status) == (8, 0)


def test_status_does_not_come_between_a_product_and_its_report(binding, monkeypatch):
    word = [0]
    lib = binding(Reporting(word))

    def take(at):
        bits, word[0] = word[0], 0
        return ccv.OK, bits
    monkeypatch.setattr(tk, "_words", {-1: 4096})
    monkeypatch.setattr(tk, "ccv3d_take_status", take)
    assert meanwhile(lib, lambda: tk.linear(torch.zeros(3, 64), torch.zeros(5, 64)), tk.status) == (8, 0)
