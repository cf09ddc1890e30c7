"""Every form of the attention of few rows against the oracle: tiles of 4, 8 and 16 rows, heads up to 64, 128 and 256 channels, rows that
are loaded whole or channel by channel, both kinds of queries, one workgroup along the keys or several."""
import pytest

from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, F32, Batch
from tests.test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx", [333, 1500])
@pytest.mark.parametrize("q_bits", [16, 4])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (40, BF16), (128, BF16), (128, F32), (100, BF16), (256, BF16), (200, BF16), (256, F32)])
@pytest.mark.parametrize("new", [1, 2, 5])                          # with four query heads to a key / value head: 4, 8 and more rows
def test_forms(new, D, dtype, q_bits, ctx):
    print("form", new, ctx, D, dtype, q_bits, flush=True)
    b = Batch([new], [ctx], 2, D, 121)
    b.fill()
    assert (B.lib().kv_pages_attention_workspace_bytes(b.T, 1, 8, 2, D, b.max_pages) > 0) == (ctx > 1000)
    run(b, 8, q_dtype=dtype, rope=True, q_bits=q_bits)
    run(b, 8, q_dtype=dtype, q_bits=q_bits, window=300, sinks=5)
