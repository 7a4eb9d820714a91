"""Paged-cache calls that the library and its binding refuse, all of them before anything is launched (the addresses here belong to nobody)."""
import ctypes as C

import pytest
import torch

from paper_2410_13344_b200 import binding

AT = 1 << 20


class Pages(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("max_pages", C.c_int32), ("free_cap", C.c_int32),
        ("len", C.c_void_p), ("page_table", C.c_void_p), ("free_pages", C.c_void_p), ("n_free", C.c_void_p),
    ]


class KvAppendArgs(C.Structure):
    _fields_ = [
        ("dtype", C.c_int32), ("T", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("k_row_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_row_stride", C.c_int64), ("v_head_stride", C.c_int64),
        ("slot", C.c_void_p), ("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("k_min", C.c_void_p), ("k_max", C.c_void_p),
        ("n_pool_pages", C.c_int32),
    ]


class PagedAttnArgs(C.Structure):
    _fields_ = [
        ("dtype", C.c_int32), ("B", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("max_pages", C.c_int32), ("n_pool_pages", C.c_int32),
        ("q", C.c_void_p), ("q_row_stride", C.c_int64), ("q_head_stride", C.c_int64), ("k_pool", C.c_void_p), ("v_pool", C.c_void_p),
        ("page_table", C.c_void_p), ("len", C.c_void_p), ("sel", C.c_void_p), ("n_sel", C.c_void_p), ("max_sel", C.c_int32),
        ("out", C.c_void_p), ("lse", C.c_void_p), ("scale", C.c_float), ("max_len", C.c_int32), ("window", C.c_int32),
        ("scratch", C.c_void_p), ("scratch_bytes", C.c_size_t),
    ]


class PageSelectArgs(C.Structure):
    _fields_ = [
        ("dtype", C.c_int32), ("B", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("max_pages", C.c_int32), ("n_pool_pages", C.c_int32),
        ("q", C.c_void_p), ("q_row_stride", C.c_int64), ("q_head_stride", C.c_int64), ("k_min", C.c_void_p), ("k_max", C.c_void_p),
        ("page_table", C.c_void_p), ("len", C.c_void_p), ("max_sel", C.c_int32), ("n_first", C.c_int32), ("n_last", C.c_int32),
        ("max_len", C.c_int32), ("sel", C.c_void_p), ("n_sel", C.c_void_p), ("scratch", C.c_void_p), ("scratch_bytes", C.c_size_t),
    ]


@pytest.fixture(scope="module", autouse=True)
def argument_types():
    L = binding.lib()
    L.cerb_pages_plan.argtypes = [C.POINTER(Pages), C.c_void_p, C.c_int32] + [C.c_void_p] * 6
    L.cerb_pages_trim.argtypes = [C.POINTER(Pages), C.c_void_p, C.c_void_p]
    L.cerb_kv_append.argtypes = [C.POINTER(KvAppendArgs), C.c_void_p]
    L.cerb_paged_attention_scratch_bytes.argtypes = [C.c_int32] * 8 + [C.POINTER(C.c_size_t)]
    L.cerb_paged_attention.argtypes = [C.POINTER(PagedAttnArgs), C.c_void_p]
    L.cerb_page_select_scratch_bytes.argtypes = [C.c_int32] * 7 + [C.POINTER(C.c_size_t)]
    L.cerb_page_select.argtypes = [C.POINTER(PageSelectArgs), C.c_void_p]



def _pages(**kw):
    a = dict(B=4, max_pages=8, free_cap=32, len=AT, page_table=AT, free_pages=AT, n_free=AT)
    a.update(kw)
    return Pages(**a)


def test_pages_refusals():
    L = binding.lib()

    def plan(state, n_new=AT, rows=16, slot=AT, pos=AT, seq=AT, row_off=AT, granted=AT):
        return L.cerb_pages_plan(C.byref(state), n_new, rows, slot, pos, seq, row_off, granted, None)

    for name in ("len", "page_table", "free_pages", "n_free"):
        assert plan(_pages(**{name: None})) == binding.E_ARG
        assert L.cerb_pages_trim(C.byref(_pages(**{name: None})), AT, None) == binding.E_ARG
    for name in ("n_new", "slot", "pos", "seq", "row_off", "granted"):
        assert plan(_pages(), **{name: None}) == binding.E_ARG
    assert plan(_pages(), rows=-1) == binding.E_ARG and plan(_pages(B=-1)) == binding.E_ARG
    assert plan(_pages(max_pages=0)) == binding.E_ARG and plan(_pages(free_cap=-1)) == binding.E_ARG
    assert plan(_pages(B=8193)) == binding.E_SHAPE and plan(_pages(B=8192, max_pages=1 << 18)) == binding.E_SHAPE
    assert plan(_pages(), rows=(1 << 30) + 1) == binding.E_SHAPE
    assert L.cerb_pages_plan(None, AT, 16, AT, AT, AT, AT, AT, None) == binding.E_ARG
    assert L.cerb_pages_trim(C.byref(_pages()), None, None) == binding.E_ARG
    assert L.cerb_pages_trim(C.byref(_pages(B=0)), AT, None) == binding.OK


def test_append_refusals():
    L = binding.lib()

    def call(**kw):
        a = dict(dtype=binding.BF16, T=4, n_kv_heads=2, head_dim=64, k=AT, v=AT, k_row_stride=128, k_head_stride=64, v_row_stride=128, v_head_stride=64,
                 slot=AT, k_pool=AT, v_pool=AT, k_min=AT, k_max=AT, n_pool_pages=8)
        a.update(kw)
        return L.cerb_kv_append(C.byref(KvAppendArgs(**a)), None)

    assert call(T=0) == binding.OK and call(T=0, k=None, v=None, slot=None) == binding.OK
    for name in ("k", "v", "slot", "k_pool", "v_pool", "k_min", "k_max"):
        assert call(**{name: None}) == binding.E_ARG, name
    for name in ("k", "v", "k_pool", "v_pool", "k_min", "k_max"):
        assert call(**{name: AT + 8}) == binding.E_ARG, name
    for name in ("k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride"):
        assert call(**{name: 68}) == binding.E_ARG, name
        assert call(dtype=binding.F32, T=0, **{name: 68}) == binding.OK, name
    assert call(dtype=2) == binding.E_ARG and call(T=-1) == binding.E_ARG
    assert call(head_dim=96) == binding.E_SHAPE and call(n_kv_heads=0) == binding.E_SHAPE
    assert call(n_pool_pages=0) == binding.E_SHAPE and call(n_pool_pages=1 << 27) == binding.E_SHAPE
    assert L.cerb_kv_append(None, None) == binding.E_ARG


def test_attention_refusals():
    L = binding.lib()

    def call(**kw):
        a = dict(dtype=binding.BF16, B=1, n_heads=8, n_kv_heads=2, head_dim=64, max_pages=8, n_pool_pages=8, q=AT, q_row_stride=512, q_head_stride=64,
                 k_pool=AT, v_pool=AT, page_table=AT, len=AT, sel=None, n_sel=None, max_sel=0, out=AT, lse=AT, scale=1.0, max_len=100, window=0,
                 scratch=None, scratch_bytes=0)
        a.update(kw)
        return L.cerb_paged_attention(C.byref(PagedAttnArgs(**a)), None)

    none = dict(B=0, q=None, k_pool=None, v_pool=None, page_table=None, len=None, out=None)
    assert call(**none) == binding.OK
    for name in ("q", "k_pool", "v_pool", "page_table", "len", "out"):
        assert call(**{name: None}) == binding.E_ARG, name
    for name in ("q", "k_pool", "v_pool", "out"):
        assert call(**{name: AT + 8}) == binding.E_ARG, name
    for name in ("q_row_stride", "q_head_stride"):
        assert call(**{name: 68}) == binding.E_ARG, name
    assert call(sel=AT) == binding.E_ARG and call(n_sel=AT) == binding.E_ARG and call(sel=AT, n_sel=AT) == binding.E_ARG
    assert call(sel=AT, n_sel=AT, max_sel=4, **none) == binding.OK
    for bad in (dict(dtype=5), dict(max_pages=0), dict(n_pool_pages=0), dict(max_len=0), dict(window=-1)):
        assert call(**bad) == binding.E_ARG, bad
    for bad in (dict(B=-1), dict(n_heads=7), dict(n_heads=0), dict(n_kv_heads=0), dict(head_dim=80)):
        assert call(**bad) == binding.E_SHAPE, bad
    assert L.cerb_paged_attention(None, None) == binding.E_ARG
    # a cache long enough to be split, without the scratch or with too little of it
    nb = C.c_size_t(0)
    args = (binding.BF16, 1, 8, 2, 64, 100000, 0, 0)
    assert L.cerb_paged_attention_scratch_bytes(*args, C.byref(nb)) == binding.OK and nb.value > 0
    assert call(B=1, max_len=100000) == binding.E_NOMEM
    assert call(B=1, max_len=100000, scratch=AT, scratch_bytes=nb.value - 1) == binding.E_NOMEM
    assert call(B=1, max_len=100000, scratch=AT + 8, scratch_bytes=nb.value) == binding.E_ARG
    assert L.cerb_paged_attention_scratch_bytes(*args, None) == binding.E_ARG
    assert L.cerb_paged_attention_scratch_bytes(binding.BF16, 1, 8, 2, 64, 0, 0, 0, C.byref(nb)) == binding.E_ARG


def test_select_refusals():
    L = binding.lib()

    def call(**kw):
        a = dict(dtype=binding.BF16, B=1, n_heads=8, n_kv_heads=2, head_dim=64, max_pages=8, n_pool_pages=8, q=AT, q_row_stride=512, q_head_stride=64,
                 k_min=AT, k_max=AT, page_table=AT, len=AT, max_sel=4, n_first=1, n_last=1, max_len=100, sel=AT, n_sel=AT, scratch=None, scratch_bytes=0)
        a.update(kw)
        return L.cerb_page_select(C.byref(PageSelectArgs(**a)), None)

    assert call(B=0, q=None, k_min=None, k_max=None, page_table=None, len=None, sel=None, n_sel=None) == binding.OK
    for name in ("q", "k_min", "k_max", "page_table", "len", "sel", "n_sel"):
        assert call(**{name: None}) == binding.E_ARG, name
    for name in ("q", "k_min", "k_max"):
        assert call(**{name: AT + 8}) == binding.E_ARG, name
    for bad in (dict(dtype=5), dict(n_first=-1), dict(n_last=-1), dict(max_sel=0), dict(max_len=0), dict(n_pool_pages=0), dict(q_head_stride=4)):
        assert call(**bad) == binding.E_ARG, bad
    for bad in (dict(n_first=3, n_last=2), dict(max_pages=(1 << 17) + 1), dict(max_pages=0), dict(n_heads=130), dict(n_heads=7), dict(head_dim=256),
                dict(B=1 << 23)):
        assert call(**bad) == binding.E_SHAPE, bad
    assert call(B=1) == binding.E_NOMEM
    assert L.cerb_page_select(None, None) == binding.E_ARG


def test_binding_wants_tensors_of_a_gpu():
    i32 = dict(dtype=torch.int32)
    lens, table, free, n_free = torch.zeros(2, **i32), torch.zeros(2, 4, **i32), torch.zeros(8, **i32), torch.zeros(1, **i32)
    pool, q = torch.zeros(8, 2, 16, 64), torch.zeros(2, 4, 64)
    summary = torch.zeros(8, 2, 64)
    for call in (lambda: binding.pages_plan(lens, lens, table, free, n_free, 4), lambda: binding.pages_trim(lens, lens, table, free, n_free),
                 lambda: binding.kv_append(q[:, :2], q[:, :2], lens, pool, pool), lambda: binding.paged_attention(q, pool, pool, table, lens, 1.0, 32),
                 lambda: binding.page_select(q, summary, summary, table, lens, 2, 32)):
        with pytest.raises(binding.CerbError) as e:
            call()
        assert e.value.code == binding.E_ARG


def test_kernels_that_change_the_cache_release_nothing_early():
    """Tree attention reads lengths, tables and committed keys ahead of its wait for the kernel in front: what writes them may not let it start early."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(binding.__file__), "csrc", "pages.cu")).read()
    text = re.sub(r"//[^\n]*", "", text)
    assert text.count("__global__") == text.count("griddep_wait()") == 4 and "griddep_launch" not in text
