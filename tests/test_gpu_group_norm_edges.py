"""Group norms where their forms and their launches meet, against 64 bits (tolerances: ``test_gpu_group_norm.close``) or bit by bit."""
import pytest
import torch

import _operators_ref as ref
from test_gpu_group_norm import close, inputs

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("s,p,c", [(5, 40_000, 128), (3, 200_000, 72), (7, 9, 8200)])
def test_samples_in_place_over_several_turns(s, p, c, dtype):
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, sc, sh = inputs(s, p, c, dtype, seed=6)
    want = tk.group_norm(x, 4, w, b, scale=sc, shift=sh, activation="silu")
    for i in range(s):                                                    # a sample by itself has the same bits
        assert torch.equal(tk.group_norm(x[i:i + 1], 4, w, b, scale=sc[i:i + 1], shift=sh[i:i + 1], activation="silu"), want[i:i + 1])
    close(want[-1:], *ref.group_norm(x[-1:], 4, w, b, sc[-1:], sh[-1:], 1e-6, "silu"))
    pixels_first = x.transpose(0, 1).contiguous().transpose(0, 1)         # the samples of a pixel side by side
    for z in (x, pixels_first):
        for _ in range(2):
            y = z.clone(memory_format=torch.preserve_format)
            assert tk.group_norm(y, 4, w, b, scale=sc, shift=sh, activation="silu", out=y) is y and torch.equal(y, want)


@pytest.mark.parametrize("p", [1, 9, 3520, 40_000])
@pytest.mark.parametrize("value", [3.0, 1000.0, -2.0 ** 20])
def test_bf16_groups_of_one_large_value(value, p):
    """What is left of the mean's rounding, 2^-18 of the value at most, is multiplied by 1 / sqrt(eps); the mean times the factor is rounded once more
    (2^-24), and so is the sum with the bias."""
    from paper_2609_31938_b200 import tokens as tk
    x, w, b, _, _ = inputs(2, p, 64, BF, seed=7)
    x[1, :, 16:32] = value
    y = tk.group_norm(x, 4, w, b, eps=1e-4)
    want, err = ref.group_norm(x, 4, w, b, None, None, 1e-4, "none")
    close(y, want, err + 2.0 ** -22 * abs(value) * 100 * w.double().abs())
