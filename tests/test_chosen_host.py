"""Calls around chosen pages that are refused on the host, before anything is enqueued: no GPU is needed, no pointer is followed."""
import ctypes

import pytest

import paper_2605_03884_amd as qkv
from paper_2605_03884_amd import binding
from test_paged_host import ALIGN, AT, BAD_PAGES, BAD_QUERIES, CAPACITY, NULL, OK, SHAPE, pages, query


def digests(**changes):
    tables = (ctypes.c_void_p * 64)(*[AT + 4096 * i for i in range(64)])
    d = binding.Digests(ctypes.cast(tables, ctypes.POINTER(ctypes.c_void_p)), AT)
    d.keep = tables
    for name, value in changes.items():
        setattr(d, name, value)
    return d


def choose(**changes):
    x = binding.Choose(AT, 8 * 128, 128, 3, 0, AT, AT, 1 << 30, AT, 0, 8, 4, 1, 2, 0)
    for name, value in changes.items():
        setattr(x, name, value)
    return x


def slots(**changes):
    x = binding.Slots(AT, 3, AT, AT, AT, AT)
    for name, value in changes.items():
        setattr(x, name, value)
    return x


@pytest.mark.parametrize("changes,code", BAD_PAGES, ids=[str(c) for c, _ in BAD_PAGES])
def test_pools_that_are_refused(changes, code):
    if "refs_dev" in changes:
        code = ALIGN
    L, p, out = qkv.lib(), pages(**changes), ctypes.c_uint64(0)
    tokens = changes.get("rows", 3)
    assert L.qkv_pages_digest(p, digests(), None, tokens, 0, 1, AT, None) == code
    assert L.qkv_paged_choose(p, digests(), choose(tokens=tokens), None) == code
    assert L.qkv_paged_choose_workspace(p, 3, ctypes.byref(out)) == code
    assert L.qkv_paged_attend_chosen(p, query(tokens=tokens), AT, 0, None) == code
    assert L.qkv_paged_attend_chosen_workspace(p, 8, 0, ctypes.byref(out)) == code
    assert L.qkv_paged_prompt_chosen(p, query(starts_dev=AT), AT, None) == code
    assert L.qkv_paged_prompt_chosen_workspace(p, 8, 3, ctypes.byref(out)) == code
    assert L.qkv_pages_slots(p, slots(), AT, None) == code


@pytest.mark.parametrize("changes,code", BAD_QUERIES, ids=[str(c) for c, _ in BAD_QUERIES])
def test_queries_that_are_refused(changes, code):
    assert qkv.lib().qkv_paged_attend_chosen(pages(row_pages=1000), query(**changes), AT, 0, None) == code
    assert qkv.lib().qkv_paged_prompt_chosen(pages(row_pages=1000), query(starts_dev=AT, **changes), AT, None) == code


def test_what_belongs_to_one_of_the_two_calls():
    L = qkv.lib()
    assert L.qkv_paged_attend_chosen(pages(), query(), None, 0, None) == NULL
    assert L.qkv_paged_attend_chosen(pages(), query(), AT + 2, 0, None) == ALIGN
    assert L.qkv_paged_attend_chosen(pages(), query(), AT, -1, None) == SHAPE
    assert L.qkv_paged_attend_chosen(pages(), query(window=5), AT, 0, None) == SHAPE
    assert L.qkv_paged_attend_chosen(pages(), query(tokens=2), AT, 0, None) == SHAPE
    assert L.qkv_paged_attend_chosen(pages(), query(starts_dev=AT), AT, 0, None) == SHAPE
    assert L.qkv_paged_attend_chosen(pages(), query(prior_out_dev=AT), AT, 0, None) == NULL
    assert L.qkv_paged_attend_chosen(pages(), query(prior_out_dev=AT + 4, prior_lse_dev=AT), AT, 0, None) == ALIGN
    assert L.qkv_paged_attend_chosen(pages(), None, AT, 0, None) == NULL
    assert L.qkv_paged_prompt_chosen(pages(), query(starts_dev=AT), None, None) == NULL
    assert L.qkv_paged_prompt_chosen(pages(), query(), AT, None) == NULL
    assert L.qkv_paged_prompt_chosen(pages(), query(starts_dev=AT), AT + 2, None) == ALIGN
    assert L.qkv_paged_prompt_chosen(pages(), query(starts_dev=AT, window=5), AT, None) == SHAPE
    assert L.qkv_paged_prompt_chosen(pages(), query(starts_dev=AT, tokens=0), AT, None) == SHAPE
    assert L.qkv_paged_prompt_chosen(pages(), query(starts_dev=AT, prior_out_dev=AT, prior_lse_dev=AT), AT, None) == SHAPE


def test_digests_that_are_refused():
    L, p = qkv.lib(), pages()
    for bad, code in ((digests(layers=None), NULL), (digests(exponents_dev=0), NULL), (digests(exponents_dev=AT + 8), ALIGN)):
        assert L.qkv_pages_digest(p, bad, None, 3, 0, 1, AT, None) == code
        assert L.qkv_paged_choose(p, bad, choose(), None) == code
    for value, code in ((0, NULL), (AT + 8, ALIGN)):
        d = digests()
        d.keep[1] = value
        assert L.qkv_pages_digest(p, d, None, 3, 0, 1, AT, None) == code and L.qkv_paged_choose(p, d, choose(), None) == code
    assert L.qkv_pages_digest(p, None, None, 3, 0, 1, AT, None) == NULL
    for starts, tokens, begin, count in ((None, 4, 0, 1), (AT, -1, 0, 1), (AT, 1 << 27, 0, 1), (AT, 5, -1, 1), (AT, 5, 2, 1), (AT, 5, 0, 0), (AT, 5, 0, 3), (AT, 5, 1, 2)):
        assert L.qkv_pages_digest(p, digests(), starts, tokens, begin, count, AT, None) == SHAPE
    assert L.qkv_pages_digest(pages(page_tokens=1), digests(), AT, 1 << 22, 0, 1, AT, None) == SHAPE          # a grid's threads
    assert L.qkv_pages_digest(p, digests(), AT + 2, 5, 0, 1, AT, None) == ALIGN and L.qkv_pages_digest(p, digests(), AT, 5, 0, 1, AT + 2, None) == ALIGN


BAD_CHOICES = [
    (dict(q_dev=0), NULL), (dict(choice_dev=0), NULL), (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(q_heads=6), SHAPE), (dict(q_heads=2), SHAPE),
    (dict(q_heads=4 * 129), SHAPE), (dict(q_token_stride=-8), SHAPE), (dict(q_token_stride=4), SHAPE), (dict(q_head_stride=4), SHAPE), (dict(first=-1), SHAPE),
    (dict(last=0), SHAPE), (dict(most=2), SHAPE), (dict(first=2 ** 30, last=2 ** 30, most=2 ** 31 - 1), SHAPE), (dict(tokens=2), SHAPE),
    (dict(tokens=0, starts_dev=AT), SHAPE), (dict(tokens=1 << 40, starts_dev=AT), SHAPE), (dict(q_dev=AT + 8), ALIGN), (dict(choice_dev=AT + 2), ALIGN),
    (dict(starts_dev=AT + 2), ALIGN), (dict(status_dev=AT + 2), ALIGN), (dict(workspace_dev=AT + 8), ALIGN),
]


@pytest.mark.parametrize("changes,code", BAD_CHOICES, ids=[str(c) for c, _ in BAD_CHOICES])
def test_choices_that_are_refused(changes, code):
    assert qkv.lib().qkv_paged_choose(pages(), digests(), choose(**changes), None) == code


def test_workspaces():
    L, need = qkv.lib(), ctypes.c_uint64(1)
    for p in (pages(), pages(row_pages=100000, page_tokens=1), pages(rows=500, row_pages=2000)):
        sizes = []
        for tokens in (p.rows, p.rows + 1, 700, 5000, 100000):
            assert L.qkv_paged_choose_workspace(p, tokens, ctypes.byref(need)) == OK
            sizes.append(need.value)
        assert sizes == sorted(sizes)
        if need.value:
            assert L.qkv_paged_choose(p, digests(), choose(starts_dev=AT, tokens=100000, workspace_dev=0), None) == NULL
            assert L.qkv_paged_choose(p, digests(), choose(starts_dev=AT, tokens=100000, workspace_bytes=64), None) == CAPACITY
    assert L.qkv_paged_choose_workspace(pages(), 3, None) == NULL and L.qkv_paged_choose_workspace(pages(), 0, ctypes.byref(need)) == SHAPE
    assert L.qkv_paged_choose_workspace(pages(row_pages=1 << 20, page_tokens=1), 3, ctypes.byref(need)) == SHAPE
    assert L.qkv_paged_attend_chosen_workspace(pages(), 8, 0, None) == NULL and L.qkv_paged_attend_chosen_workspace(pages(), 7, 0, ctypes.byref(need)) == SHAPE
    assert L.qkv_paged_attend_chosen_workspace(pages(), 8, -1, ctypes.byref(need)) == SHAPE
    assert L.qkv_paged_attend_chosen_workspace(pages(rows=600), 8, 0, ctypes.byref(need)) == OK and need.value == 0        # as many items as there is room for
    assert L.qkv_paged_attend_chosen_workspace(pages(row_pages=1000), 8, 200, ctypes.byref(need)) == OK and need.value > 0
    assert L.qkv_paged_prompt_chosen_workspace(pages(), 8, 5, None) == NULL and L.qkv_paged_prompt_chosen_workspace(pages(), 8, 0, ctypes.byref(need)) == SHAPE


def test_slots_that_are_refused():
    L, p = qkv.lib(), pages()
    for bad, code in ((dict(starts_dev=0), NULL), (dict(tokens=0), SHAPE), (dict(tokens=1 << 27), SHAPE), (dict(more_dev=AT + 2), ALIGN), (dict(starts_dev=AT + 2), ALIGN),
                      (dict(row_dev=AT + 2), ALIGN), (dict(place_dev=AT + 2), ALIGN), (dict(slot_dev=AT + 4), ALIGN)):
        assert L.qkv_pages_slots(p, slots(**bad), AT, None) == code
    assert L.qkv_pages_slots(p, None, AT, None) == NULL and L.qkv_pages_slots(p, slots(), AT + 2, None) == ALIGN
