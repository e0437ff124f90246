"""Which batches ccv3d_kv_attend takes, by the workspace call (nothing is launched; without a device it gets as far as that)."""
import pytest

import paper_2609_31938_b200 as ccv
from test_tokens_host import batch, cache

TAKEN = (ccv.OK, ccv.ERR_CUDA, ccv.ERR_ARCH)


def ask(kv_heads, q_heads, dtype=ccv.BF16, pages=4096, page_tokens=64, **b):
    return ccv.ccv3d_kv_attend_workspace(cache(pages=pages, kv_heads=kv_heads, page_tokens=page_tokens), batch(**b), q_heads, dtype)[0]


@pytest.mark.parametrize("dtype", [ccv.BF16, ccv.F32])
@pytest.mark.parametrize("b", [
    dict(batch=64, tokens=8192 + 63, max_new=8192, max_pages=2048),          # a prompt beside 63 single tokens, tables for 131072 tokens
    dict(batch=256, tokens=2048 + 255, max_new=2048, max_pages=2048),        # a piece of a prompt beside 255
    dict(batch=512, tokens=512, max_new=1, max_pages=2048),
    dict(batch=1, tokens=131072, max_new=131072, max_pages=2048),            # one prompt that fills its table
    dict(batch=4096, tokens=4096 * 4, max_new=4, max_pages=512),
    dict(batch=2, tokens=100, max_new=0x7FFFFFFF, max_pages=2048),           # no bound known
])
def test_ordinary_batches_are_taken(b, dtype):
    assert ask(8, 32, dtype, **b) in TAKEN


def test_both_sides_of_the_limit():
    """2e9 units: (tokens * g / r + batch) * kv_heads * (max_pages * page_tokens / 128 + 1)."""
    def units(tokens, n, width, kv, g, r):
        return (tokens * g // r + n) * kv * (width * 64 // 128 + 1)
    a = dict(batch=65536, tokens=65536, max_new=64, max_pages=7629)          # tiles of 256 rows
    assert units(65536, 65536, 7629, 8, 1, 256) > 2e9 > units(65536, 65536, 7590, 8, 1, 256)
    assert ask(8, 8, **a) == ccv.ERR_UNSUPPORTED
    assert ask(8, 8, **dict(a, max_pages=7590)) in TAKEN
    a = dict(batch=1, tokens=4, max_new=4, max_pages=(1 << 25) - 5)          # 32-bit token numbers
    assert ask(8, 8, **a) in TAKEN
    assert ask(8, 8, **dict(a, max_pages=1 << 25)) == ccv.ERR_UNSUPPORTED
    assert ask(8, 8, pages=1 << 22, **dict(a, max_pages=8)) == ccv.ERR_UNSUPPORTED      # rows of the pool
