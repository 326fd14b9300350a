"""New tokens in a paged cache on the GPU, in the forms that only some sizes take (the plan's words say which was taken) and where
tables and pages are not what they should be: against the plain models of oracle/paged_step.py, with the tolerances that
tests/test_gpu_paged_step.py derives."""
import math
import random

import pytest
import torch

from oracle import paged_step as O
from paper_2510_20878_amd import binding as B
from tests.test_gpu_paged_step import E, MORE, Pool, _prior

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


def plan_words(p):
    """(workgroups with work, units of a run (0: whole tiles), tokens of a unit, whether the cache is read past) of the step's plan."""
    torch.cuda.synchronize()
    return p.plan[24:40].view(torch.int32).tolist()


def lengths(n, lo, hi, seed):
    return [random.Random(seed + i).randint(lo, hi) for i in range(n)]


@pytest.mark.parametrize("H,G,D,P,held,new", [
    (8, 2, 64, 16, lengths(220, 0, 400, 1), [1] * 220), (8, 2, 64, 12, lengths(220, 0, 400, 2), [1] * 220),   # tiles of 16 rows alone
    (8, 4, 64, 16, lengths(230, 0, 200, 3), [4] * 100 + [40, 70, 33, 40] + [4] * 126),                       # most tiles of 16
    (8, 4, 128, 16, [100] * 30, [90] * 30), (8, 4, 96, 12, [100] * 30, [90] * 30),                            # of 128
    (4, 4, 64, 48, [50, 20] * 30, [80] * 60),
])
@pytest.mark.parametrize("with_prior", [False, True])
def test_attend_a_workgroup_for_each_tile(H, G, D, P, held, new, with_prior):
    p = Pool(1, H, D, P, held, new, n_q_heads=H * G, seed=P)
    p.books()
    n_wgs, run, _, _ = plan_words(p)
    rows = [n * G for n in new]
    large = 16 if p.n_rows * G <= 16 * len(held) else 128
    assert run == 0 and n_wgs == sum(-(-n // (16 if n <= 16 else large)) for n in rows)
    p.fill()
    p.append(0)
    print(f"attend_paged: {H} x {G} heads of {D}, pages of {P}, {n_wgs} tiles", flush=True)
    prior = _prior(p, 3) if with_prior else None
    out, lse = p.attend(0, prior=prior)
    p.attention_is_right(0, out, lse, prior=prior)


def fill_layer(p, layer):
    """Pool.fill() of one layer, on the device; the others are never read."""
    g = torch.Generator(device="cuda").manual_seed(layer)
    p.pool = torch.full(p.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    seen = p.pool.permute(p.order)
    for r, t in enumerate(p.held):
        for i in range(-(-t // p.P)):
            m = min(p.P, t - i * p.P)
            seen[p.table[r][i], layer, :, :, :m] = torch.randn((2, p.H, m, p.D), generator=g, device="cuda").bfloat16()
    p.q, p.k, p.v = (torch.randn((p.n_rows, h, p.D), generator=g, device="cuda").bfloat16().expand(p.L, -1, -1, -1)
                     for h in (p.Hq, p.H, p.H))
    p.cache = B.paged_cache(p.pool, p.d_table, p.P, p.n_pages, p.layout, p.L, p.H, p.D, bad_pages=p.bad, n_table=p.d_table.shape[1])


@pytest.mark.parametrize("L,H,G,D", [(40, 8, 4, 128), (70, 8, 2, 96), (80, 8, 4, 64)])
@pytest.mark.parametrize("P,layout", [(16, "page_major"), (12, "tile_major")])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 40, 2]])
def test_attend_past_the_last_level_cache(L, H, G, D, P, layout, new):
    """All layers' keys and values are more than that cache holds."""
    p = Pool(L, H, D, P, [1500, 900, 30], new, layout, n_q_heads=H * G, seed=L)
    p.books()
    assert plan_words(p)[3] == 1
    fill_layer(p, L - 1)
    p.append(L - 1)
    print(f"attend_paged: {L} layers, {H} x {G} heads of {D}, pages of {P}, {new} new rows", flush=True)
    out, lse = p.attend(L - 1)
    p.attention_is_right(L - 1, out, lse)
    assert p.bad.item() == 0


@pytest.mark.parametrize("G,D,P", [(8, 64, 16), (1, 128, 16), (16, 96, 12), (3, 64, 100)])
def test_attend_more_pieces_than_are_joined_at_once(G, D, P):
    p = Pool(2, 1, D, P, [40000, 100, 33000], [1, 1, 1], n_q_heads=G, seed=G)
    p.books()
    run, unit = plan_words(p)[1:3]
    assert run and 40001 // unit // run > 64
    p.fill()
    for layer in (0, 1, 0):
        p.append(layer)
        print(f"attend_paged: {G} heads of {D} on one, pages of {P}, layer {layer}", flush=True)
        prior = _prior(p, layer) if layer else None
        out, lse = p.attend(layer, prior=prior)
        p.attention_is_right(layer, out, lse, prior=prior)


@pytest.mark.parametrize("P,columns,tokens", [(64, 2 ** 20 + 1, 128), (12, 5600000, 128), (16, 2 ** 24, 256)])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 0, 90]])
def test_attend_tables_of_many_columns(P, columns, tokens, new):
    """Tables so wide that a unit of the plan is more than 64 tokens."""
    p = Pool(1, 1, 64, P, [9000, 300, 3], new, n_q_heads=4, seed=P)
    wide = torch.full((3, columns), -1, dtype=torch.int32, device="cuda")
    wide[:, :p.n_table] = p.d_table
    p.d_table = wide
    p.books()
    assert plan_words(p)[2] == tokens
    fill_layer(p, 0)
    p.append(0)
    print(f"attend_paged: {columns} columns of pages of {P}, {new} new rows", flush=True)
    out, lse = p.attend(0)
    p.attention_is_right(0, out, lse)
    assert p.bad.item() == 0


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("P", [16, 12, 48, 5])
def test_bad_pages_of_large_tiles_are_as_if_not_there(P, D):
    """Page ids out of range at a request's start, between its pages and at its end; page 0, which is read instead, is NaN."""
    new = [40, 50, 33]
    p = Pool(1, 1, D, P, [150, 700, 0], new, n_q_heads=4, seed=7, n_pages=1000)
    p.books()
    table, held, _, _, start, _, _, _ = p.books_are_right()
    assert all(0 not in t for t in table)
    p.fill()
    p.append(0)
    torch.cuda.synchronize()
    gone = {(0, 0): -1, (0, 3): p.n_pages, (1, 1): 2 ** 31 - 1, (1, 2): p.n_pages + 1, (1, -(-held[1] // P) - 1): -1, (2, 0): -2 ** 31}
    for (r, col), page in gone.items():
        p.d_table[r, col] = page
    print(f"attend_paged: pages of {P}, heads of {D}", flush=True)
    out, lse = p.attend(0)
    rows_are_right(p, out, lse, table, held, start, lambda r, i: (r, i // P) not in gone)
    assert p.bad.item() > 0


@pytest.mark.parametrize("layout,P,D,G", [("page_major", 16, 128, 4), ("tile_major", 64, 96, 2), ("page_major", 12, 64, 7)])
def test_documents_loaded_into_the_pages_then_a_question(layout, P, D, G):
    """Pages for the documents come from page_step, load_chunks_paged writes them there, the question's rows are appended
    and attend to both: one cache, as if all had been appended."""
    L, H, T = 2, 2, [100, 64, 37]
    p = Pool(L, H, D, P, [0, 0], [sum(T), T[1]], layout, spare=40, n_q_heads=H * G, seed=17, n_table=300 // P + 3, n_rows=sum(T) + T[1])
    p.books()
    w = p.books_are_right()
    p.fill()
    ctx_docs = B.Context(L, H, D, 128, group_int8=0, group_int4=0)
    slot = ctx_docs.chunk_bytes(B.PREC_16, 128) + 255 & ~255
    ctx_docs.register_slab(B.TIER_HBM, B.PREC_16, torch.empty(slot * len(T), dtype=torch.uint8, device="cuda"))
    docs = [torch.randn((L, 2, H, t, D), generator=p.g).bfloat16().cuda() for t in T]
    for i, t in enumerate(T):
        ctx_docs.pool_insert(i, B.PREC_16, t, None, B.TIER_HBM)
        ctx_docs.quantize_chunk(docs[i], t, B.PREC_16, 0, ctx_docs.pool_slot(i, B.TIER_HBM)[0])
    for r, ids in enumerate(([0, 1, 2], [1])):
        own = B.paged_cache(p.pool, p.d_table[r].contiguous(), P, p.n_pages, layout, L, H, D, bad_pages=p.bad)
        ctx_docs.load_chunks_paged(ids, own)
    torch.cuda.synchronize()
    # the question and the first token of the answer
    p.table, p.held, p.free, p.n_free = w[0], w[1], w[2], w[3]
    for new in ([30, 3], [1, 1]):
        p.new = new
        p.d_new.copy_(torch.tensor(new))
        p.books()
        w = p.books_are_right()
        for layer in range(L):
            p.append(layer)
            out, lse = p.attend(layer)
            p.attention_is_right(layer, out, lse)
        p.table, p.held, p.free, p.n_free = w[0], w[1], w[2], w[3]
    # what the attention was compared with is the documents, in the order in which they were asked for
    seen = p.pool.cpu().permute(p.order)
    for r, ids in enumerate(([0, 1, 2], [1])):
        want = torch.cat([docs[i].cpu() for i in ids], 3)
        got = torch.stack([seen[p.table[r][i // P], :, :, :, i % P] for i in range(want.shape[3])], 3)
        assert torch.equal(got, want)
    assert p.bad.item() == 0
