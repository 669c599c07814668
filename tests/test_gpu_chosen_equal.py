"""Attention over chosen pages where all keys are the same and score tens of millions: out is the mean of the values that are seen, lse the score and the log of their number."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_words, ragged
from paged_case import HALF_STEP, TYPES, Cache

pytestmark = pytest.mark.gpu


def the_same_keys(length, dim, size, kind):
    cache = Cache([length], 1, dim, size, kind, seed=dim + size)
    key = (torch.randn(dim, generator=torch.Generator().manual_seed(1)) * 2000).to(TYPES[kind])
    cache.k[:] = key
    cache.gpu()
    return cache, key


def mean(cache, chosen, place):
    _, v = cache.rows()[0]
    some = [t for j in sorted(chosen) for t in range(j * cache.size, (j + 1) * cache.size) if t <= place]
    return v[0, some].mean(0), np.abs(v[0, some]).mean(0), len(some)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("size", [4, 32, 64])
@pytest.mark.parametrize("length", [600, 9000])
def test_prompts(kind, dim, size, length):
    cache, key = the_same_keys(length, dim, size, kind)
    q = (torch.randn(40, 3, dim, generator=torch.Generator().manual_seed(2)) * 2000).to(TYPES[kind])
    width = (length - 1) // size
    choices = [[{0, 2, i % 5, width // 2, width - i % 3}] for i in range(40)]
    out, lse = torch.zeros(40, 3, dim, device="cuda", dtype=q.dtype), torch.zeros(40, 3, device="cuda")
    qkv.paged_prompt_chosen(cache.pages, as_words(choices, cache.table.shape[1]), q.cuda(), ragged(cache, [40])[2], 1.0, out, lse)
    u = HALF_STEP[kind]
    for i in range(40):
        want, size_of, n = mean(cache, choices[i][0], length - 40 + i)
        # weights are the same power of two; sums of n products and of n weights, two steps of the quotient, half a step of the result
        bound = (n + 4) * 2.0 ** -23 * size_of * (1 + u) + u * np.abs(want) + (2.0 ** -25 if kind == "fp16" else 0.0)
        assert (np.abs(out[i].double().cpu().numpy() - want) <= bound).all()
        score, terms = q[i].double() @ key.double(), q[i].double().abs() @ key.double().abs()
        # dim products' sum, the scale's and the product's rounding, the sum with a number that is small beside it
        assert (np.abs(lse[i].double().cpu().numpy() - score.numpy() - np.log(n)) <= (dim + 8) * 2.0 ** -24 * terms.numpy() + 2.0 ** -20).all()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("size", [4, 32])
@pytest.mark.parametrize("most", [0, 1])
def test_single_tokens(kind, dim, size, most):
    cache, key = the_same_keys(700, dim, size, kind)
    q = (torch.randn(1, 3, dim, generator=torch.Generator().manual_seed(2)) * 2000).to(TYPES[kind])
    chosen = {0, 2, 5, 9, 699 // size}
    out, lse = torch.zeros(1, 3, dim, device="cuda"), torch.zeros(1, 3, device="cuda")
    qkv.paged_attend_chosen(cache.pages, as_words([[chosen]], cache.table.shape[1]), q.cuda(), 1.0, out, lse, most=most)
    want, size_of, n = mean(cache, chosen, 699)
    # as above, the result in 32 bits; weights are held to 22 bits
    bound = ((n + 16) * 2.0 ** -23 + 2.0 ** -21) * size_of
    assert (np.abs(out[0].double().cpu().numpy() - want) <= bound).all()
    score, terms = q[0].double() @ key.double(), q[0].double().abs() @ key.double().abs()
    assert (np.abs(lse[0].double().cpu().numpy() - score.numpy() - np.log(n)) <= (dim + 8) * 2.0 ** -24 * terms.numpy() + 2.0 ** -20).all()
