"""Tensors that the binding's calls for new tokens in a paged cache refuse, before an address reaches a kernel: no GPU."""
import pytest
import torch

from paper_2510_20878_amd import binding as B
from tests.test_paged_step_host import D, H, cache, ctx_of, step


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
