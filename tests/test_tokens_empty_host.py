"""Calls without work: a batch of no sequences, as one of no tokens."""
import pytest

import paper_2609_31938_b200 as ccv
from test_tokens_host import append, attend, batch, cache


@pytest.mark.parametrize("b", [
    dict(batch=0, tokens=0), dict(batch=0, tokens=0, max_new=0, max_pages=0, new_start=None, total=None, page_table=None)])
def test_no_sequences(b):
    assert append(b=batch(**b)) == ccv.OK
    assert attend(b=batch(**b)) == ccv.OK
    assert attend(b=batch(**b), ws=None, n=0) == ccv.OK
    assert ccv.ccv3d_kv_attend_workspace(cache(), batch(**b), 2, ccv.BF16) == (ccv.OK, 0)


def test_rows_without_a_sequence_are_refused():
    assert append(b=batch(batch=0, tokens=1)) == ccv.ERR_INVALID_ARG
    assert attend(b=batch(batch=0, tokens=1)) == ccv.ERR_INVALID_ARG
    assert attend(b=batch(batch=-1, tokens=0)) == ccv.ERR_INVALID_ARG
    assert attend(b=batch(batch=1, tokens=0, total=None)) == ccv.ERR_INVALID_ARG
    assert attend(b=batch(batch=0, tokens=0), c=cache(codes=None)) == ccv.ERR_INVALID_ARG
    assert attend(b=batch(batch=0, tokens=0), hq=3) == ccv.ERR_INVALID_ARG


def test_no_sequences_through_the_binding(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2609_31938_b200 import tokens as tk
    monkeypatch.setattr(tk, "_device", lambda: -1)
    monkeypatch.setattr(tk, "_stream", lambda dev: 0)
    monkeypatch.setattr(tk, "_capturing", lambda: False)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c = tk.PagedCache(torch.zeros(4, 2, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 2))
    b = tk.TokenBatch(ints(1), ints(0), ints(0, 5), 0)
    x = torch.zeros(0, 2, 64)
    assert c.append(x, x, b, q=x).shape == (0, 2, 64)
    out, lse = c.attend(torch.zeros(0, 4, 64), b, want_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
