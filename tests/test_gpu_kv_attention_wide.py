"""Attention with heads of more than 128 channels and many rows: windows, places and pages that are not there, scales of any size; and
float32 queries of many rows, of all widths."""
import pytest

from tests import test_gpu_kv_attention_rows as R
from tests.attention_util import F32
from tests.test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu
SETS = [s for s in R.SETS if s[5] > 128]


@pytest.mark.parametrize("window,sinks", [(1, 0), (130, 3), (256, 200)])
@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", SETS)
def test_windows(new, ctx, H, Hq, pages, D, window, sinks):
    R.test_windows(new, ctx, H, Hq, pages, D, window, sinks)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", SETS)
def test_pages_and_rows_that_are_not_there(new, ctx, H, Hq, pages, D):
    R.test_pages_and_rows_that_are_not_there(new, ctx, H, Hq, pages, D)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", SETS)
def test_value_scales_of_any_size(new, ctx, H, Hq, pages, D):
    R.test_value_scales_of_any_size(new, ctx, H, Hq, pages, D)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", SETS)
def test_masked_places_may_hold_anything(new, ctx, H, Hq, pages, D):
    R.test_masked_places_may_hold_anything(new, ctx, H, Hq, pages, D)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", R.SETS)
def test_float32_queries(new, ctx, H, Hq, pages, D):
    run(R.batch(new, ctx, H, Hq, pages, D, 37), Hq, q_dtype=F32, rope=True)
