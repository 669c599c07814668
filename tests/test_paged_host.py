"""Calls of the cache in pages that are refused on the host, before anything is enqueued: no GPU is needed, no pointer is followed."""
import ctypes

import pytest
import torch

import paper_2605_03884_amd as qkv
from paper_2605_03884_amd import binding

OK, NULL, SHAPE, CAPACITY, ALIGN = 0, -1, -2, -5, -6
AT = 1 << 20                                       # an address that is aligned and never read


def pages(**changes):
    count = changes.pop("layers", 2)
    tables = (ctypes.c_void_p * 64)(*[AT + 4096 * i for i in range(64)])
    p = binding.Pages(count, 4, 128, 16, 0, 100, 3, 10, ctypes.cast(tables, ctypes.POINTER(ctypes.c_void_p)), ctypes.cast(tables, ctypes.POINTER(ctypes.c_void_p)),
                      4 * 16 * 128, 16 * 128, 128, AT, AT, AT)
    p.keep = tables
    for name, value in changes.items():
        setattr(p, name, value)
    return p


def query(**changes):
    x = binding.PagedQuery(AT, 8 * 128, 128, 3, 0, AT, AT, 0, 0, AT, 1 << 30, AT, 0, 8, 0, 0, 0.1, 0)
    for name, value in changes.items():
        setattr(x, name, value)
    return x


def rows(**changes):
    x = binding.Rows(AT, AT, 3, 0, 128, 512, 0, 0, 1)
    for name, value in changes.items():
        setattr(x, name, value)
    return x


BAD_PAGES = [
    (dict(layers=0), SHAPE), (dict(layers=65), SHAPE), (dict(kv_heads=0), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(page_tokens=0), SHAPE), (dict(page_tokens=24), SHAPE), (dict(page_tokens=1 << 21), SHAPE), (dict(value_type=2), SHAPE), (dict(value_type=-1), SHAPE),
    (dict(pages=0), SHAPE), (dict(rows=0), SHAPE), (dict(rows=65537), SHAPE), (dict(row_pages=0), SHAPE), (dict(row_pages=1 << 27), SHAPE),
    (dict(rows=65536, row_pages=1 << 15), SHAPE), (dict(page_stride=-8), SHAPE), (dict(page_stride=4), SHAPE), (dict(head_stride=1 << 31), SHAPE),
    (dict(token_stride=64), SHAPE), (dict(token_stride=132), SHAPE), (dict(table_dev=0), NULL), (dict(lens_dev=0), NULL), (dict(table_dev=AT + 2), ALIGN),
    (dict(lens_dev=AT + 1), ALIGN), (dict(refs_dev=AT + 2), ALIGN),
]


@pytest.mark.parametrize("changes,code", BAD_PAGES, ids=[str(c) for c, _ in BAD_PAGES])
def test_pools_that_are_refused(changes, code):
    L, p, out = qkv.lib(), pages(**changes), ctypes.c_uint64(0)
    tokens = changes.get("rows", 3)
    assert L.qkv_paged_attend(p, query(tokens=tokens), None) == code
    assert L.qkv_paged_prompt(p, query(starts_dev=AT), None) == code
    assert L.qkv_pages_append(p, rows(tokens=tokens), AT, None) == code
    assert L.qkv_pages_reserve(p, AT, AT, None) == code
    assert L.qkv_pages_fork(p, AT, AT, 1, AT, None) == code
    assert L.qkv_pages_free(p, AT, 1, 0, 0, AT, None) == code
    assert L.qkv_pages_compact(p, AT, AT, 1 << 30, AT, None) == code
    assert L.qkv_paged_attend_workspace(p, 8, ctypes.byref(out)) == code
    assert L.qkv_paged_prompt_workspace(p, 8, 3, ctypes.byref(out)) == code
    assert L.qkv_pages_compact_workspace(p, ctypes.byref(out)) == code


def test_layer_pointers_are_looked_at():
    L, p = qkv.lib(), pages()
    for value, code in ((0, NULL), (AT + 8, ALIGN)):
        p.keep[1] = value
        assert L.qkv_paged_attend(p, query(), None) == code
    p.k_layers = None
    assert L.qkv_paged_attend(p, query(), None) == NULL
    assert L.qkv_paged_attend(None, query(), None) == NULL


BAD_QUERIES = [
    (dict(q_dev=0), NULL), (dict(out_dev=0), NULL), (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(q_heads=6), SHAPE), (dict(q_heads=2), SHAPE),
    (dict(q_heads=4 * 129), SHAPE), (dict(q_token_stride=-8), SHAPE), (dict(q_token_stride=4), SHAPE), (dict(q_head_stride=4), SHAPE), (dict(window=-1), SHAPE),
    (dict(sinks=-1, window=4), SHAPE), (dict(sinks=1), SHAPE), (dict(softmax_scale=float("nan")), SHAPE), (dict(softmax_scale=float("inf")), SHAPE),
    (dict(q_dev=AT + 8), ALIGN), (dict(out_dev=AT + 8), ALIGN), (dict(lse_dev=AT + 2), ALIGN), (dict(status_dev=AT + 2), ALIGN), (dict(workspace_dev=AT + 8), ALIGN),
    (dict(workspace_dev=0), NULL), (dict(workspace_bytes=64), CAPACITY),
]


@pytest.mark.parametrize("changes,code", BAD_QUERIES, ids=[str(c) for c, _ in BAD_QUERIES])
def test_queries_that_are_refused(changes, code):
    assert qkv.lib().qkv_paged_attend(pages(row_pages=1000), query(**changes), None) == code
    assert qkv.lib().qkv_paged_prompt(pages(row_pages=1000), query(starts_dev=AT, **changes), None) == code


def test_what_belongs_to_one_of_the_two_calls():
    L = qkv.lib()
    assert L.qkv_paged_attend(pages(), query(tokens=2), None) == SHAPE
    assert L.qkv_paged_attend(pages(), query(starts_dev=AT), None) == SHAPE
    assert L.qkv_paged_attend(pages(), query(prior_out_dev=AT), None) == NULL
    assert L.qkv_paged_attend(pages(), query(prior_lse_dev=AT), None) == NULL
    assert L.qkv_paged_attend(pages(), query(prior_out_dev=AT + 4, prior_lse_dev=AT), None) == ALIGN
    assert L.qkv_paged_attend(pages(), None, None) == NULL
    assert L.qkv_paged_prompt(pages(), query(), None) == NULL
    assert L.qkv_paged_prompt(pages(), query(starts_dev=AT + 2), None) == ALIGN
    assert L.qkv_paged_prompt(pages(), query(starts_dev=AT, tokens=0), None) == SHAPE
    assert L.qkv_paged_prompt(pages(), query(starts_dev=AT, prior_out_dev=AT, prior_lse_dev=AT), None) == SHAPE
    assert L.qkv_paged_attend(pages(rows=65536, row_pages=32767, page_tokens=4096), query(tokens=65536), None) == SHAPE


BAD_ROWS = [
    (dict(k_dev=0), NULL), (dict(v_dev=0), NULL), (dict(tokens=-1, starts_dev=AT), SHAPE), (dict(tokens=2), SHAPE), (dict(layer_begin=-1), SHAPE), (dict(layer_begin=2), SHAPE),
    (dict(layer_count=0), SHAPE), (dict(layer_count=3), SHAPE), (dict(token_stride=4), SHAPE), (dict(head_stride=-8), SHAPE), (dict(layer_stride=1 << 40), SHAPE),
    (dict(k_dev=AT + 8), ALIGN), (dict(v_dev=AT + 2), ALIGN), (dict(starts_dev=AT + 2), ALIGN),
]


@pytest.mark.parametrize("changes,code", BAD_ROWS, ids=[str(c) for c, _ in BAD_ROWS])
def test_rows_that_are_refused(changes, code):
    assert qkv.lib().qkv_pages_append(pages(), rows(**changes), AT, None) == code


def test_pool_calls_that_are_refused():
    L, p = qkv.lib(), pages()
    assert L.qkv_pages_append(p, None, AT, None) == NULL
    assert L.qkv_pages_append(p, rows(), AT + 2, None) == ALIGN
    none = pages(refs_dev=0)
    assert L.qkv_pages_reserve(none, AT, AT, None) == NULL and L.qkv_pages_free(none, AT, 1, 0, 0, AT, None) == NULL
    assert L.qkv_pages_fork(none, AT, AT, 1, AT, None) == NULL and L.qkv_pages_compact(none, AT, AT, 1 << 30, AT, None) == NULL
    assert L.qkv_pages_reserve(p, AT, None, None) == NULL and L.qkv_pages_reserve(p, AT + 2, AT, None) == ALIGN
    assert L.qkv_pages_fork(p, None, AT, 1, AT, None) == NULL and L.qkv_pages_fork(p, AT, AT, 1, None, None) == NULL
    assert L.qkv_pages_fork(p, AT, AT, 0, AT, None) == SHAPE and L.qkv_pages_fork(p, AT, AT, 4, AT, None) == SHAPE
    assert L.qkv_pages_fork(p, AT, AT + 2, 1, AT, None) == ALIGN
    assert L.qkv_pages_free(p, AT, 0, 0, 0, AT, None) == SHAPE and L.qkv_pages_free(p, AT, 4, 0, 0, AT, None) == SHAPE
    assert L.qkv_pages_free(p, None, 2, 0, 0, AT, None) == SHAPE and L.qkv_pages_free(p, AT, 1, 0, 3, AT, None) == SHAPE
    assert L.qkv_pages_free(p, AT, 1, -1, 0, AT, None) == SHAPE and L.qkv_pages_free(p, AT + 2, 1, 0, 0, AT, None) == ALIGN
    need = ctypes.c_uint64(0)
    assert L.qkv_pages_compact_workspace(p, ctypes.byref(need)) == OK and need.value >= 12 * 100
    assert L.qkv_pages_compact(p, AT, AT, need.value - 1, AT, None) == CAPACITY
    assert L.qkv_pages_compact(p, AT, None, need.value, AT, None) == NULL and L.qkv_pages_compact(p, AT, AT, need.value, None, None) == NULL
    assert L.qkv_pages_compact(p, AT, AT + 8, need.value, AT, None) == ALIGN and L.qkv_pages_compact(p, AT + 2, AT, need.value, AT, None) == ALIGN


def test_workspaces_by_shape():
    need = ctypes.c_uint64(1)
    L = qkv.lib()
    assert L.qkv_paged_attend_workspace(pages(row_pages=8), 8, ctypes.byref(need)) == OK and need.value == 0      # 128 tokens: never split
    assert L.qkv_paged_attend_workspace(pages(row_pages=9), 8, ctypes.byref(need)) == OK and need.value > 0
    assert L.qkv_paged_attend_workspace(pages(), 8, None) == NULL and L.qkv_paged_attend_workspace(pages(), 7, ctypes.byref(need)) == SHAPE
    assert L.qkv_paged_prompt_workspace(pages(), 8, 100000, ctypes.byref(need)) == OK and need.value == 0         # many query tiles: keys are not split
    assert L.qkv_paged_prompt_workspace(pages(row_pages=10000), 8, 20, ctypes.byref(need)) == OK and need.value > 0
    assert L.qkv_paged_prompt_workspace(pages(), 8, 0, ctypes.byref(need)) == SHAPE and L.qkv_paged_prompt_workspace(pages(), 8, 1 << 40, ctypes.byref(need)) == SHAPE


def test_tensors_that_are_refused():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    table, lens = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        qkv.Pages.make([], [], table, lens)
    with pytest.raises(ValueError):
        qkv.Pages.make([k], [k, k], table, lens)
    with pytest.raises(ValueError):
        qkv.Pages.make([k], [k], table, lens)                      # host memory
    with pytest.raises(ValueError):
        qkv.Pages.make([k.float()], [k.float()], table, lens)
