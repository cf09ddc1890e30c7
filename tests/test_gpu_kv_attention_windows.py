"""Windows that no position reaches: the same as none, up to the largest number that the argument takes."""
import pytest
import torch

from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, Batch
from tests.test_gpu_kv_attention_rows import FEW, MANY

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [([200, 1], [150, 700], 2, 4, None, 64), ([1, 1], [700, 3], 2, 4, None, 128),
                                                  ([200], [150], 1, 2, None, 256), FEW + (64,), MANY + (128,), FEW + (256,)])
def test_windows_of_any_size(new, ctx, H, Hq, pages, D):
    print("window", new, ctx, D, flush=True)
    b = Batch(new, ctx, H, D, 91, max_pages=pages)
    b.fill()
    pages_d, table, qs, ln = b.dev()
    Q = torch.randn(b.T, Hq, D, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    none = B.kv_pages_attention(Q, pages_d, table, qs, ln, H)
    for window in (2 ** 63 - 1, 2 ** 62 + 5, 2 ** 40, 2 ** 31, 2 ** 31 - 1, 2 ** 20):
        for sinks in (0, 3, 2 ** 62):
            assert torch.equal(B.kv_pages_attention(Q, pages_d, table, qs, ln, H, window=window, sinks=sinks), none), (window, sinks)
