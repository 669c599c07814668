"""Workspaces of prompts over pages: one that is enough for a batch is enough for every smaller one.  No GPU is needed."""
import ctypes

import pytest

import paper_2605_03884_amd as qkv
from test_paged_host import AT, CAPACITY, NULL, OK, pages, query

SHAPES = [(32, 8, 128, 131072), (32, 8, 128, 9000), (64, 8, 64, 65536), (16, 2, 256, 40000), (28, 4, 128, 40000), (5, 1, 64, 70000), (128, 1, 128, 33000),
          (20, 1, 128, 1500)]


def pool(kv_heads, dim, room):
    return pages(kv_heads=kv_heads, head_dim=dim, row_pages=room // 16, rows=2, page_stride=kv_heads * 16 * dim, head_stride=16 * dim, token_stride=dim)


def needs(p, q_heads, tokens):
    need = ctypes.c_uint64(1)
    assert qkv.lib().qkv_paged_prompt_workspace(p, q_heads, tokens, ctypes.byref(need)) == OK
    return need.value


def refused(p, q_heads, tokens, space):
    """Whether a call is refused for its workspace.  `starts` out of place are what is looked at last, so no call gets as far as the GPU."""
    x = query(q_heads=q_heads, tokens=tokens, starts_dev=AT + 2, workspace_bytes=space, workspace_dev=AT if space else 0)
    return qkv.lib().qkv_paged_prompt(p, x, None) in (CAPACITY, NULL)


@pytest.mark.parametrize("q_heads,kv_heads,dim,room", SHAPES)
def test_sizes_rise_with_the_batch(q_heads, kv_heads, dim, room):
    p, before = pool(kv_heads, dim, room), 0
    for tokens in [*range(1, 700), *range(700, 14000, 37), 20000, 30000, 100000]:
        now = needs(p, q_heads, tokens)
        assert now >= before, tokens
        before = now
    assert before > 0


@pytest.mark.parametrize("q_heads,kv_heads,dim,room", SHAPES)
def test_what_is_enough_for_a_batch_is_enough_for_smaller_ones(q_heads, kv_heads, dim, room):
    p = pool(kv_heads, dim, room)
    for largest in (1, 61, 600, 2100, 6000, 8192, 20000):
        space = needs(p, q_heads, largest)
        for tokens in {*range(1, min(largest, 400) + 1), *range(1, largest + 1, 53), largest}:
            assert not refused(p, q_heads, tokens, space), (largest, tokens)


def test_no_more_than_some_batch_needs():
    p = pool(8, 128, 131072)
    for largest in (61, 300, 2100):
        space = needs(p, 32, largest)
        assert any(refused(p, 32, tokens, space - 4) for tokens in range(1, largest + 1)), largest
    assert refused(p, 32, 61, 64) and refused(p, 32, 61, 0)
