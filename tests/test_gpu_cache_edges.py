"""The operators on a paged KV cache where tables, masks and values are at an edge; the tolerances are those of
test_gpu_cache.py."""
import numpy as np
import pytest

from tests import cache_reference as ref
from tests.gpu_util import say
from tests.test_gpu_cache import check_attend, run_attend

pytestmark = pytest.mark.gpu

NEVER = 1 << 30


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,kv_heads,group,lens,rows,seeing", [
    (64, 1, 1, [320, 192], 192, 128), (64, 2, 4, [64, 64], 64, 32), (128, 1, 1, [500, 256], 256, 128), (256, 1, 1, [512, 160], 160, 128),
    (128, 8, 4, [1024] * 4, 256, 64)])
def test_row_tiles_of_padding_alone(dtype, dim, kv_heads, group, lens, rows, seeing):
    """Rows that see nothing fill whole row tiles, in tables that end with the last sequence's last page."""
    say("case padding", dtype, dim, kv_heads, group, lens, rows)
    start = [max(0, n - rows + i - 40) if i < seeing else NEVER for n in lens for i in range(rows)]
    c = ref.Case(dim, lens, [rows] * len(lens), kv_heads=kv_heads, group=group, dim=dim, dtype=dtype, row_start=start)
    c.table = c.table[:, : -(-max(lens) // c.page)].contiguous()  # no spare page
    out, lse = run_attend(c)
    check_attend(c, out, lse)
    seen = np.tile(np.arange(rows) < seeing, len(lens))
    assert np.isneginf(lse.cpu().numpy()[~seen]).all() and (out.cpu()[~seen] == 0).all() and lse.cpu()[seen].isfinite().all()
