"""Paged-cache calls at the limits of their index arithmetic: what is past them is refused before anything is launched (the addresses here belong to nobody)."""
import ctypes as C

import pytest

from paper_2410_13344_b200 import binding
from test_paged_refusals import AT, PagedAttnArgs, PageSelectArgs

@pytest.fixture(scope="module", autouse=True)
def argument_types():
    L = binding.lib()
    L.cerb_paged_attention_scratch_bytes.argtypes = [C.c_int32] * 8 + [C.POINTER(C.c_size_t)]
    L.cerb_paged_attention.argtypes = [C.POINTER(PagedAttnArgs), C.c_void_p]
    L.cerb_page_select.argtypes = [C.POINTER(PageSelectArgs), C.c_void_p]


def attention(**kw):
    a = dict(dtype=binding.BF16, B=1, n_heads=8, n_kv_heads=2, head_dim=64, max_pages=8, n_pool_pages=8, q=AT, q_row_stride=512, q_head_stride=64, k_pool=AT, v_pool=AT,
             page_table=AT, len=AT, sel=AT, n_sel=AT, max_sel=4, out=AT, lse=AT, scale=1.0, max_len=100, window=0, scratch=AT, scratch_bytes=1 << 40)
    a.update(kw)
    return binding.lib().cerb_paged_attention(C.byref(PagedAttnArgs(**a)), None)


def select(**kw):
    a = dict(dtype=binding.BF16, B=1, n_heads=8, n_kv_heads=2, head_dim=64, max_pages=8, n_pool_pages=8, q=AT, q_row_stride=512, q_head_stride=64, k_min=AT, k_max=AT,
             page_table=AT, len=AT, max_sel=4, n_first=1, n_last=1, max_len=100, sel=AT, n_sel=AT, scratch=AT, scratch_bytes=1 << 40)
    a.update(kw)
    return binding.lib().cerb_page_select(C.byref(PageSelectArgs(**a)), None)


def test_lists_longer_than_a_billion_entries():
    """A list's index is an int that steps by up to 32 x 64 (attention) or 1024 (selection) past its last entry."""
    nb = C.c_size_t(0)
    for K in ((1 << 30) + 1, 2 ** 31 - 1024, 2 ** 31 - 1):
        assert attention(max_sel=K) == binding.E_SHAPE and select(max_sel=K) == binding.E_SHAPE
        assert binding.lib().cerb_paged_attention_scratch_bytes(binding.BF16, 1, 8, 2, 64, 100, 0, K, C.byref(nb)) == binding.E_SHAPE
    for K in (1, 1 << 30):
        assert binding.lib().cerb_paged_attention_scratch_bytes(binding.BF16, 1, 8, 2, 64, 100, 0, K, C.byref(nb)) == binding.OK
