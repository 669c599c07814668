"""Limits and workspaces of the calls around chosen pages, on the host: nothing is enqueued, no pointer is followed."""
import ctypes

import pytest

import paper_2605_03884_amd as qkv
from test_chosen_host import choose, digests
from test_paged_host import ALIGN, AT, CAPACITY, NULL, OK, SHAPE, pages, query


@pytest.mark.parametrize("head_dim,kv_heads,q_heads", [(64, 1, 64), (64, 8, 64), (128, 1, 64), (128, 8, 32), (256, 2, 16), (256, 1, 128)])
@pytest.mark.parametrize("page_tokens,row_pages", [(16, 100), (16, 2048), (64, 4000)])
def test_a_prompts_workspace_is_enough_for_smaller_batches(head_dim, kv_heads, q_heads, page_tokens, row_pages):
    """Up to more query tiles than are ever cut (four times as many as run at once).  A choice that is not aligned is refused behind the look at the workspace."""
    p = pages(head_dim=head_dim, kv_heads=kv_heads, page_tokens=page_tokens, row_pages=row_pages, token_stride=head_dim, head_stride=head_dim * page_tokens,
              page_stride=head_dim * page_tokens * kv_heads)
    L, need = qkv.lib(), ctypes.c_uint64(0)
    per = 128 // (q_heads // kv_heads)
    most = (3200 // kv_heads + 2) * per
    marks = sorted({max(1, n + d) for n in [1, per, 2 * per] + [most * i // 60 // per * per for i in range(61)] for d in (-1, 0, 1)})
    last, some = 0, False
    for at, tokens in enumerate(marks):
        assert L.qkv_paged_prompt_chosen_workspace(p, q_heads, tokens, ctypes.byref(need)) == OK
        assert need.value >= last
        last = need.value
        for smaller in marks[max(0, at - 12): at + 1] + marks[: at + 1: 9]:
            x = query(starts_dev=AT, tokens=smaller, q_heads=q_heads, workspace_bytes=need.value)
            assert L.qkv_paged_prompt_chosen(p, x, AT + 2, None) == ALIGN, (tokens, smaller)
        x = query(starts_dev=AT, tokens=tokens, q_heads=q_heads, workspace_bytes=0)
        cut = L.qkv_paged_prompt_chosen(p, x, AT + 2, None) == CAPACITY
        some = some or (cut and (tokens + per - 1) // per * kv_heads > 256)
    assert some == (page_tokens * row_pages >= 2 * 4096)             # a few long parts, where tiles are more than CUs


@pytest.mark.parametrize("starts", [0, AT])
def test_as_many_choices_as_a_launch_has_room_for(starts):
    """rows * kv_heads < 2^23, with one token of every row too: the last number that is taken comes as far as the look at the workspace."""
    L, need = qkv.lib(), ctypes.c_uint64(0)
    for rows, kv_heads, code in ((65535, 128, CAPACITY), (65536, 128, SHAPE), (65536, 127, CAPACITY), (65536, 512, SHAPE)):
        p = pages(rows=rows, kv_heads=kv_heads, row_pages=3000, page_tokens=1)
        tokens = 1 if starts else rows
        x = choose(starts_dev=starts, tokens=tokens, q_heads=kv_heads, workspace_bytes=64)
        assert L.qkv_paged_choose(p, digests(), x, None) == code
        assert L.qkv_paged_choose_workspace(p, tokens, ctypes.byref(need)) == (OK if code == CAPACITY else SHAPE)
        assert code == SHAPE or need.value > 0
