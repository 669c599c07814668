"""Attention of single tokens over chosen pages, joined with another result in place, and with queries that are one row for all sequences."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_sets, as_words, draw_choices, expected
from oracle import paged_ref
from paged_case import TYPES, Cache, check_attend
from test_gpu_attend_chosen import run
from test_gpu_choose import Scored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [0, 1])
@pytest.mark.parametrize("q_heads,heads,dim", [(6, 2, 64), (6, 2, 128), (40, 2, 64), (34, 2, 128), (20, 1, 256)])
def test_joined_in_place(most, q_heads, heads, dim):
    """prior_out is out and prior_lse is lse: items in several parts, and whole where a word about how few are chosen says so; to the bit what other memory gives."""
    cache = Cache([400, 0, 90, 17], heads, dim, 16, seed=dim + q_heads)
    choices = draw_choices(cache, cache.lens, heads, 0.3, dim)
    choices[2] = [set()] * heads
    words = as_words(choices, cache.table.shape[1])
    assert (qkv.paged_attend_chosen_workspace(cache.pages, q_heads, most) > 0) == (most == 0)
    gen = torch.Generator().manual_seed(3)
    other, other_lse = torch.randn(4, q_heads, dim, generator=gen), torch.randn(4, q_heads, generator=gen) + 3
    other_lse[1] = -float("inf")
    other_lse[3] = -float("inf")
    q, want, want_lse = run(cache, words, q_heads, dim, 0.1, most=most, prior=(other.cuda(), other_lse.cuda()))
    out, lse = other.cuda(), other_lse.cuda()
    qkv.paged_attend_chosen(cache.pages, words, q.cuda(), 0.1, out, lse, most=most, prior=(out, lse))
    assert np.array_equal(out.double().cpu().numpy(), want) and np.array_equal(lse.double().cpu().numpy(), want_lse)
    alone = expected(cache, q.double().numpy(), range(4), [n - 1 for n in cache.lens], choices, 0.1)
    o, l = paged_ref.joined(alone[0], alone[1], other.double().numpy(), other_lse.double().numpy())
    size = np.maximum(alone[2], np.abs(other.double().numpy()))
    # as where the other result is somewhere else: a handful of half steps more, of both sides' sizes
    check_attend(want, want_lse, (o, l, size, alone[3], np.maximum(alone[4], np.abs(np.where(np.isfinite(l), l, 0)))), dim, 400 + 64)


def test_queries_that_are_one_row():
    """Strides of 0 between sequences and between heads."""
    x = Scored([300, 77, 0, 9], 2, 3, 64, 8, seed=1)
    one = torch.randn(64, generator=torch.Generator().manual_seed(2)).to(TYPES["fp16"])
    x.q = one.expand(4, 6, 64)
    q = one.cuda().expand(4, 6, 64)
    choice = qkv.paged_choose(x.cache.pages, x.digests(), q, 9)
    choices = as_sets(choice, x.cache.table.shape[1])
    assert choices == x.want(9)
    out, lse = torch.full((4, 6, 64), 7.0, device="cuda"), torch.full((4, 6), 7.0, device="cuda")
    qkv.paged_attend_chosen(x.cache.pages, choice, q, 0.2, out, lse)
    want = expected(x.cache, x.q.double().numpy(), range(4), [n - 1 for n in x.cache.lens], choices, 0.2)
    check_attend(out.double().cpu().numpy(), lse.double().cpu().numpy(), want, 64, 300)
