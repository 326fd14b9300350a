"""New tokens in a paged cache on the GPU, where tables are shorter than what a request holds: against the plain models of
oracle/paged_step.py, with the tolerances that tests/test_gpu_paged_step.py derives."""
import math

import pytest
import torch

from oracle import paged_step as O
from paper_2510_20878_amd import binding as B
from tests.test_gpu_paged_step import E, MORE, Pool

pytestmark = pytest.mark.gpu


def rows_are_right(p, out, lse, table, held, start, there, layer=0):
    """Every new row against the rows of its request that it sees and that are there (there(r, i): whether request r's row i is)."""
    torch.cuda.synchronize()
    seen, scale = p.pool.cpu().permute(p.order)[:, layer], p.D ** -0.5
    out, lse, q = out.cpu().double(), lse.cpu().double(), p.q[layer].cpu().double()
    for r in range(p.R):
        n = start[r + 1] - start[r]
        for row in range(start[r], start[r + 1]):
            keep = [i for i in range(held[r] - n + row - start[r] + 1) if there(r, i)]
            if not keep:
                assert (out[row] == 0).all() and (lse[row] == -math.inf).all(), (r, row)
                continue
            kv = torch.stack([seen[table[r][i // p.P], :, :, i % p.P] for i in keep], 2).double()
            o, z, spread, size = O.attend(q[row:row + 1], kv[0], kv[1], scale)
            x = 2.0 ** -15 * (1 + size) * MORE
            tol = MORE * (E * (spread + 2 * o.abs()) + 2 * x[..., None] * spread) + 1e-30
            err = (out[row] - o[0]).abs()
            assert bool((err <= tol[0]).all()), f"request {r}, row {row}: off by {(err / tol[0]).nan_to_num(math.inf).max():.3g} of the allowed"
            assert bool(((lse[row] - z[0]).abs() <= x[0]).all()), (r, row)


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [1, 3, 30, 2], [0, 4, 5, 70]])  # tiles of 16 rows alone; of 16 and of 128
@pytest.mark.parametrize("P,layout,columns", [(16, "page_major", 3), (12, "tile_major", 5), (64, "tile_major", 1), (7, "page_major", 2)])
def test_rows_beyond_the_caches_table_are_as_if_not_there(P, layout, columns, new):
    p = Pool(1, 2, 128, P, [200, 20, 333, 0], new, layout, n_q_heads=8, seed=P)
    p.books()
    table, held, _, _, start, _, _, _ = p.books_are_right()
    p.fill()
    p.append(0)
    short = p.d_table[:, :columns].contiguous()
    p.cache = B.paged_cache(p.pool, short, P, p.n_pages, layout, 1, 2, 128, bad_pages=p.bad, n_table=columns)
    print(f"attend_paged: pages of {P}, {columns} of them in the table, {new} new rows", flush=True)
    out, lse = p.attend(0)
    rows_are_right(p, out, lse, table, held, start, lambda r, i: i < columns * P)
    assert p.bad.item() > 0
