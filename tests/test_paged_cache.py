"""PagedCache's own refusals (CPU)."""
import ctypes

import pytest

from paper_2509_21354_amd import binding as kb


@pytest.mark.parametrize("L,B,H,most", [(32, 64, 32, 1024), (1, 3, 5, (1 << 26) // 15)])
def test_queries_that_the_attention_does_not_take(L, B, H, most):
    """L B H Tq <= 2^26: a cache for more is refused when it is made, and not when it is read; the limit is the library's."""
    sh, pg = kb.make_shape(L=L, B=B, H=H, H_kv=1, d=64, T=0, T_cap=1, C=1, N_cap=0, W=0, d_sum=1, d_g=1, dtype=kb.BF16), kb.make_pages(16, 1, 1)
    with pytest.raises(kb.KvevError, match="attends to no more") as e:
        kb.PagedCache(sh, 16, 1, 1, most + 1, device="cpu")
    assert e.value.status == kb.ERR_INVALID_ARG
    with pytest.raises(kb.KvevError):
        kb.PagedCache(sh, 16, 1, 1, -1, device="cpu")
    kb.PagedCache(sh, 16, 1, 1, most, device="cpu")
    r = ctypes.byref(ctypes.c_int())
    form = kb.lib().kvev_debug_page_form
    assert form(ctypes.byref(sh), ctypes.byref(pg), most, r, r, r) == kb.OK and form(ctypes.byref(sh), ctypes.byref(pg), most + 1, r, r, r) == kb.ERR_INVALID_ARG
