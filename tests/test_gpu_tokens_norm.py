"""Gated norms of many rows at widths of every form of the kernel that walks over stretches of rows (threads to a row, elements of
an access, accesses of a thread), at the ends of what each takes.  Bounds as in test_gated_norm_of_many_rows."""
import pytest

from test_gpu_tokens import BF16, F32, test_gated_norm_of_many_rows as check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

WIDTHS = [4, 128, 132, 256, 260, 320, 384, 388, 512, 768, 772, 1024, 1028, 1540, 1600, 2044, 2048, 2052, 2500, 3068, 3076, 4092, 4100, 8192,
          3, 77, 129, 383, 641, 1279, 1283, 1999, 2051, 2777, 3075, 4095, 4097]


@pytest.mark.parametrize("ch", WIDTHS)
@pytest.mark.parametrize("res,act,wd,md,post,pre,parts", [
    (F32, BF16, F32, F32, "rms", "layer", "ywbgs"),
    (BF16, BF16, BF16, BF16, "layer", "rms", "ywgs"),
])
def test_gated_norm_at_every_width(ch, res, act, wd, md, post, pre, parts):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    check(331, ch, 3, res, act, wd, md, post, pre, parts)
