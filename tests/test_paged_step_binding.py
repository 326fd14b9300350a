"""Tensors that the binding's calls for new tokens in a paged cache refuse, before an address reaches a kernel: no GPU."""
import pytest
import torch

from paper_2510_20878_amd import binding as B
from tests.test_paged_step_host import D, H, cache, ctx_of, rows, step


@pytest.mark.parametrize("dtype", [torch.float16, torch.uint16])
def test_rows_of_other_16_bit_types_are_refused(dtype):
    """The kernels read BF16: a float16 tensor's words mean other numbers."""
    c = ctx_of()
    s, pg = step(c), cache()
    good = lambda heads: torch.zeros(40, heads, D, dtype=torch.bfloat16)
    bad = lambda heads: torch.zeros(40, heads, D, dtype=dtype)
    c.append_paged(good(H).view(torch.int16), good(H), s, pg, 0)
    c.attend_paged(good(16), s, pg, 0, 1.0, good(16).view(torch.int16))
    for call in (lambda: c.append_paged(bad(H), good(H), s, pg, 0), lambda: c.append_paged(good(H), bad(H), s, pg, 0),
                 lambda: c.attend_paged(bad(16), s, pg, 0, 1.0, good(16)), lambda: c.attend_paged(good(16), s, pg, 0, 1.0, bad(16))):
        with pytest.raises(ValueError, match="bfloat16"):
            call()


def test_tensors_in_host_memory_are_refused():
    """Their addresses would fault a kernel.  (The context below stays dry where it counts: none is launched.)"""
    c = ctx_of()
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)
    bf = lambda heads: torch.zeros(40, heads, D, dtype=torch.bfloat16)
    plan = torch.zeros(c.step_plan_bytes(5, 40, 16) + 256, dtype=torch.uint8)
    plan = plan[-plan.data_ptr() % 256:]
    there_s, there_pg, there_t = step(c), cache(), B.PageTables(*[1 << 20] * 6, 5, 8, 100, 16)
    host_s = B.paged_step(i32(6), i32(40), 16, plan=plan)
    host_t = B.page_tables(i32(5, 8), i32(5), i32(100), i32(1), 16)
    pool = torch.zeros(1 << 16, dtype=torch.bfloat16)
    host_pg = B.paged_cache(pool[-(pool.data_ptr() // 2) % 8:], i32(40), 16, 4, "page_major", 3, H, D, n_table=8)
    table = B.paged_cache(1 << 20, i32(40), 16, 4, "page_major", 3, H, D, n_table=8)
    here = 1 << 20
    calls = [lambda: c.page_step(host_t, here, there_s), lambda: c.page_step(there_t, i32(5), there_s),
             lambda: c.page_step(there_t, here, host_s), lambda: c.append_paged(bf(H), rows(), there_s, there_pg, 0),
             lambda: c.append_paged(rows(), bf(H), there_s, there_pg, 0), lambda: c.append_paged(rows(), rows(), host_s, there_pg, 0),
             lambda: c.append_paged(rows(), rows(), there_s, host_pg, 0),
             lambda: c.attend_paged(bf(16), there_s, there_pg, 0, 1.0, rows(16)),
             lambda: c.attend_paged(rows(16), there_s, there_pg, 0, 1.0, bf(16)),
             lambda: c.attend_paged(rows(16), host_s, there_pg, 0, 1.0, rows(16)),
             lambda: c.attend_paged(rows(16), there_s, table, 0, 1.0, rows(16)),
             lambda: c.attend_paged(rows(16), there_s, there_pg, 0, 1.0, rows(16), lse=torch.zeros(40, 16)),
             lambda: c.attend_paged(rows(16), there_s, there_pg, 0, 1.0, rows(16), prior_lse=torch.zeros(40, 16), prior_out=here),
             lambda: c.attend_paged(rows(16), there_s, there_pg, 0, 1.0, rows(16), prior_out=torch.zeros(40, 16, D), prior_lse=here)]
    for call in calls:  # a dry context takes them all
        call()
    c._dry = False
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="on the device"):
            call()
            pytest.fail(f"call {i}")
    c.page_step(there_t, here, there_s)
    c.append_paged(rows(), rows(), there_s, there_pg, 0)
    c.attend_paged(rows(16), there_s, there_pg, 0, 1.0, rows(16), lse=here, prior_out=here, prior_lse=here)


def test_page_tables_of_fewer_entries_than_the_requests_read_are_refused():
    """Without n_table a cache is one request's, of all entries: request r's would begin r times the whole table behind its start."""
    c = ctx_of()
    s, table = step(c), torch.zeros(5, 8, dtype=torch.int32)
    pg = lambda t, **kw: B.paged_cache(1 << 20, t, 16, 100, "page_major", 3, H, D, **kw)
    c.attend_paged(rows(16), s, pg(table, n_table=8), 0, 1.0, rows(16))
    c.attend_paged(rows(16), s, pg(table[:, :6].contiguous(), n_table=6), 0, 1.0, rows(16))
    c.attend_paged(rows(16), s, pg(1 << 20, n_table=8), 0, 1.0, rows(16))  # an address is taken at its word
    c.attend_paged(rows(16), s, pg(table[:, :6], n_table=8), 0, 1.0, rows(16))
    for cache_ in (pg(table), pg(table, n_table=9), pg(table[:4], n_table=8), pg(table[:, :6], n_table=6), pg(table[:4, :6], n_table=8),
                   pg(table.T, n_table=5), pg(table.flatten()[::2], n_table=4)):
        with pytest.raises(ValueError, match="n_table"):
            c.attend_paged(rows(16), s, cache_, 0, 1.0, rows(16))
    one = step(c, n_requests=1)
    c.attend_paged(rows(16), one, pg(table[0]), 0, 1.0, rows(16))


def test_scales_beyond_the_range_are_refused():
    """As attend_packed refuses them: times log2 e they leave binary32, and every score is infinite or no number."""
    c = ctx_of()
    s, pg = step(c), cache()
    c.attend_paged(rows(16), s, pg, 0, 9e29, rows(16))
    for scale in (1e30, 3.4e38, float("inf"), float("nan"), -float("inf")):
        with pytest.raises(B.HaRagError) as e:
            c.attend_paged(rows(16), s, pg, 0, scale, rows(16))
        assert e.value.code == B.EINVAL, scale


def test_plans_that_hold_fewer_bytes_than_they_count_are_refused():
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)
    plan = torch.zeros(1 << 16, dtype=torch.uint8)
    assert B.paged_step(i32(6), i32(40), 16, plan=plan.view(torch.int64)).plan_bytes == 1 << 16
    for bad in (plan[:1].expand(1 << 16), plan[::2]):
        with pytest.raises(ValueError, match="plan"):
            B.paged_step(i32(6), i32(40), 16, plan=bad)
