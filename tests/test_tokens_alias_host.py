"""Overlaps that the token operators' C entry points turn down before a device is touched: outputs on inputs, in place or not."""
import pytest

import paper_2609_31938_b200 as ccv
from test_tokens_host import K, append, attend, batch, heads, rotary

WIDE = 1024            # elements between tokens of a fused projection; heads of 64, BF16


def fused(head, hs=64):
    """Heads from `head` on of a projection at 6 K."""
    return heads(6 * K + 2 * 64 * head, ts=WIDE, hs=hs)


@pytest.mark.parametrize("k,v,q", [
    (0, 12, 0),                                   # q, q_out and k are one tensor
    (12, 0, 0),                                   # v in the place of k
    (3, 12, 0),                                   # q's last head on k's first
    (12, 3, 0),
    (11, 12, 12),                                 # k's last head on q's first
])
def test_queries_in_place_on_keys_or_values(k, v, q):
    assert append(k=fused(k), v=fused(v), q=fused(q), qo=fused(q), hq=4) == ccv.ERR_ALIAS


def test_queries_in_place_on_keys_of_one_token():
    one = batch(tokens=1, max_new=1)
    assert append(b=one, k=fused(2), v=fused(12), q=fused(0), qo=fused(0), hq=4) == ccv.ERR_ALIAS
    assert append(b=one, k=fused(0), v=fused(12), q=fused(1), qo=fused(1), hq=4) == ccv.ERR_ALIAS


def test_heads_with_room_between_them():
    """Heads 128 apart: q on the even places, k on the odd ones but for its last head's half."""
    q = heads(6 * K, ts=WIDE, hs=128)
    assert append(k=heads(6 * K + 2 * 160, ts=WIDE, hs=128), v=heads(5 * K), q=q, qo=q, hq=4) == ccv.ERR_ALIAS
    assert append(k=heads(6 * K + 2 * 96, ts=WIDE, hs=64), v=heads(5 * K), q=q, qo=q, hq=2) == ccv.ERR_ALIAS


def test_keys_that_reach_over_the_next_tokens_queries():
    k = heads(6 * K + 2 * (WIDE - 64), ts=WIDE)   # its second head is the next token's first query head
    assert append(k=k, v=heads(5 * K), q=fused(0), qo=fused(0), hq=4) == ccv.ERR_ALIAS
    assert append(k=heads(6 * K + 2 * 512, ts=WIDE + 64), v=heads(5 * K), q=fused(0), qo=fused(0), hq=4) == ccv.ERR_ALIAS     # unlike strides


@pytest.mark.parametrize("at", [K, K + 64, K + 128 + 8])
def test_outputs_on_the_batch_arrays(at):
    at = at // 16 * 16
    assert append(q=heads(6 * K), qo=heads(at)) == ccv.ERR_ALIAS
    assert attend(o=heads(at)) == ccv.ERR_ALIAS
    assert attend(lse=at) == ccv.ERR_ALIAS


@pytest.mark.parametrize("at", [2 * K, 3 * K, K + 256])
def test_rotated_queries_on_the_rotation(at):
    assert append(rot=rotary(), q=heads(6 * K), qo=heads(at)) == ccv.ERR_ALIAS
