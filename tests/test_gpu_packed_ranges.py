"""GPU tests of the packing calls with page ranges outside the table's rows."""
import pytest
import torch

from paper_2505_13544_amd import binding as B
from tests.test_gpu_packed import context, stream

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("pages_each", [1, 2, 3, 1 << 30])
def test_ranges_outside_the_rows(back, pages_each):
    # both ends count as the nearest place that a row has: sequence 1 has pages 2 and 3 in its range, sequence 3 all four, the others none
    big, small, ps, r, mp = (1 << 31) - 1, -(1 << 31), 16, 64, 4
    first, end = [big, 2, small, small, 5, big - 1], [big, big, small, 4, 3, 2]
    n = len(first) * mp
    ctx, _ = context(r=r, max_batch=len(first), max_slots=mp * ps, page_slots=ps, n_pages=n)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = torch.arange(n, dtype=torch.int32, device=DEV).view(-1, mp)
    pool_c, pool_kr = torch.ones(n, ps, r, dtype=torch.bfloat16, device=DEV), torch.ones(n, ps, 32, dtype=torch.bfloat16, device=DEV)
    pk = B.PackedCache(torch.zeros(n, 1, 2, 16, 16, dtype=torch.uint8, device=DEV), torch.full((n, 1, 2, 16), 77, dtype=torch.uint8, device=DEV),
                       torch.zeros(n, 1, 4, 16, 8, dtype=torch.bfloat16, device=DEV), table)
    go = ctx.pages_unpack if back else ctx.pages_pack
    go(pool_c, pool_kr, table, pk, ints(first), ints(end), len(first), pages_each, stream())
    torch.cuda.synchronize()
    moved = [6, 7, 12, 13, 14, 15]
    where = (pool_kr == 0).flatten(1).all(1) if back else (pk.tensors["keys"] == 1).flatten(1).all(1)
    some = (pool_kr == 0).flatten(1).any(1) if back else (pk.tensors["scales"] != 77).flatten(1).any(1)
    assert where.nonzero().flatten().tolist() == moved and some.nonzero().flatten().tolist() == moved
    rest = [i for i in range(n) if i not in moved]
    assert bool((pool_c[rest] == 1).all()) and bool((pk.tensors["codes"][rest] == 0).all())
