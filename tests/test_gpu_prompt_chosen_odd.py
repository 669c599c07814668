"""Attention of many new tokens over chosen pages, where a value is infinite or no number: the other dimensions are what they are without it, however large the scores."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_words, expected, ragged
from paged_case import HALF_STEP, TYPES, Cache

pytestmark = pytest.mark.gpu

ODD = [3, 10]                                                        # dimensions with an odd value


def run(cache, new, choices, q, scale):
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    qkv.paged_prompt_chosen(cache.pages, as_words(choices, cache.table.shape[1]), q.cuda(), ragged(cache, new)[2], scale, out, lse, status=cache.status)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def put(cache, page, token, dimension, value):
    cache.v[0, cache.table[0, page], 0, token, dimension] = value


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [4, 16, 32, 64])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_keys_that_are_equal_weigh_the_same_whatever_they_score(kind, dim, size, scale):
    """Scores of tens of millions, each of them the same: out is the mean of the values, and a rounding of scores that is not the same twice is a factor of 2^several."""
    cache = Cache([6 * size + 40], 1, dim, size, kind, seed=dim + size)
    page = cache.table[0, 0]
    cache.k[0, page, 0] = (torch.randn(dim, generator=torch.Generator().manual_seed(1)) * 2000).to(TYPES[kind])
    want = cache.v[0, page, 0].double().mean(0).numpy()
    size_of = cache.v[0, page, 0].double().abs().mean(0).numpy()
    put(cache, 0, 1, ODD[0], float("inf"))
    put(cache, 0, size - 1, ODD[1], float("nan"))
    cache.gpu()
    q = (torch.randn(40, 3, dim, generator=torch.Generator().manual_seed(2)) * 2000).to(TYPES[kind])
    out, lse = run(cache, [40], [[{0}]] * 40, q, scale)
    assert np.isposinf(out[:, :, ODD[0]]).all() and np.isnan(out[:, :, ODD[1]]).all() and np.isfinite(lse).all()
    rest = [d for d in range(dim) if d not in ODD]
    # each weight is 2^7, a sum of `size` of them and one of as many products are off by size 2^-24 of the sizes' sum each, the quotient by two steps of
    # 2^-23 and the result by half a step of its type
    u = HALF_STEP[kind]
    bound = ((size + 4) * 2.0 ** -23 * size_of * (1 + u) + u * np.abs(want))[rest] + (2.0 ** -25 if kind == "fp16" else 0.0)
    assert (np.abs(out[:, :, rest] - want[rest]) <= bound).all(), (np.abs(out[:, :, rest] - want[rest]) / bound).max()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [4, 32, 64])
@pytest.mark.parametrize("scale", [0.2, -0.2, 100.0, -3000.0])
@pytest.mark.parametrize("length", [700, 9000])
@pytest.mark.parametrize("absent", [False, True])
def test_the_other_dimensions(kind, size, scale, length, absent):
    """Against the same call without odd values: with keys in one part and in several, some of a workgroup's tokens at the odd pages and some not; `absent`: a page is not there."""
    caches = [Cache([length], 1, 64, size, kind, seed=size) for _ in range(2)]
    n, places, middle = 50, list(range(length - 50, length)), (length // 2) // size
    choices = [[{0, 2, 6, middle, p // size} | ({1} if i % 3 == 0 else set())] for i, p in enumerate(places)]
    lost = {(0, 2)} if absent else set()
    for cache in caches:
        for _, page in lost:
            cache.gtable[0, page] = -1
    put(caches[1], 1, 0, ODD[0], -float("inf"))
    put(caches[1], middle, size - 1, ODD[1], float("nan"))
    caches[1].gv.copy_(caches[1].v)
    q = torch.randn(n, 4, 64, generator=torch.Generator().manual_seed(2)).to(TYPES[kind])
    clean, clean_lse = run(caches[0], [n], choices, q, scale)
    out, lse = run(caches[1], [n], choices, q, scale)
    assert all(int(c.status) == (qkv.STATUS_BAD_PAGE if absent else 0) for c in caches)
    assert np.array_equal(lse, clean_lse)
    sees = np.array([i % 3 == 0 for i in range(n)])
    # a weight may underflow; then an infinite value is still seen
    assert not np.isfinite(out[sees][:, :, ODD[0]]).any() and np.isfinite(out[~sees][:, :, ODD[0]]).all() and np.isnan(out[:, :, ODD[1]]).all()
    same = expected(caches[0], q.double().numpy(), [0] * n, places, choices, scale, lost=lost)
    # both have their weights rounded to the type, at maxima that need not be the same, and where a maximum passes 2^12 on the way scores with it, by 2^-13 of a
    # power of two; sums and quotients in 32 bits; each result is rounded by half a step
    u, keys = HALF_STEP[kind], 6 * size
    bound = (2 * u + 2.0 ** -12 + 2 * (keys + 8) * 2.0 ** -23) * same[2] * (1 + u) + u * (np.abs(clean) + np.abs(np.where(np.isfinite(out), out, 0)))
    bound += (2.0 ** -24 + keys * 2.0 ** -31 * 20) if kind == "fp16" else 0.0
    rest = [d for d in range(64) if d not in ODD]
    assert np.isfinite(out[:, :, rest]).all()
    err = np.abs(out - clean)[:, :, rest]
    assert (err <= bound[:, :, rest]).all(), (err / bound[:, :, rest]).max()


def far_apart(length, size, kind, rows=1):
    """Tokens of the first two pages score lowest by far; the second one holds an infinite value, the last one of the first page something that is no number."""
    cache = Cache([length] * rows, 1, 64, size, kind, seed=size)
    cache.k[..., 0] = 8.0
    for b in range(rows):
        cache.k[0, cache.table[b, :2].long(), :, :, 0] = -8.0
        cache.v[0, cache.table[b, 1], 0, 0, ODD[0]] = -float("inf")
        cache.v[0, cache.table[b, 0], 0, size - 1, ODD[1]] = float("nan")
    cache.gpu()
    return cache


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [4, 32, 64])
@pytest.mark.parametrize("strength", [1.0, 30.0, 1000.0])
def test_an_infinite_value_without_weight(kind, size, strength):
    """Weights of 2^-20 down to nothing: the value's dimension is infinite, whichever part of the keys it is in."""
    length, n = 9000, 40
    cache = far_apart(length, size, kind)
    q = torch.randn(n, 4, 64, generator=torch.Generator().manual_seed(2)).to(TYPES[kind])
    q[:, :, 0] = strength
    choices = [[{1, (length // 2) // size, (length - n + i) // size} | ({0} if i % 2 else set())] for i in range(n)]
    out, lse = run(cache, [n], choices, q, 1.0)
    assert np.isneginf(out[:, :, ODD[0]]).all() and np.isnan(out[1::2, :, ODD[1]]).all() and np.isfinite(out[::2, :, ODD[1]]).all() and np.isfinite(lse).all()
    assert np.isfinite(out[:, :, [d for d in range(64) if d not in ODD]]).all()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [4, 64])
@pytest.mark.parametrize("strength", [1.0, 30.0, 1000.0])
@pytest.mark.parametrize("most", [0, 3])
@pytest.mark.parametrize("prior", [None, 0.0, 1e6])
def test_an_infinite_value_without_weight_and_single_tokens(kind, size, strength, most, prior):
    """The same for one token of a sequence, in parts or whole, alone or joined with what weighs as much or more."""
    rows = 2
    cache = far_apart(2000, size, kind, rows)
    q = torch.randn(rows, 4, 64, generator=torch.Generator().manual_seed(2)).to(TYPES[kind])
    q[:, :, 0] = strength
    some = {1, 1999 // size} | set(range(8, 1999 // size, 2))
    words = as_words([[some], [some | {0}]], cache.table.shape[1])
    out, lse = torch.full((rows, 4, 64), 7.0, device="cuda"), torch.full((rows, 4), 7.0, device="cuda")
    other = None if prior is None else (torch.ones(rows, 4, 64, device="cuda"), torch.full((rows, 4), 8.0 * strength + prior, device="cuda"))
    qkv.paged_attend_chosen(cache.pages, words, q.cuda(), 1.0, out, lse, most=most, prior=other)
    got = out.double().cpu().numpy()
    assert np.isneginf(got[:, :, ODD[0]]).all() and np.isnan(got[1, :, ODD[1]]).all() and np.isfinite(got[0, :, ODD[1]]).all() and bool(torch.isfinite(lse).all())
    assert np.isfinite(got[:, :, [d for d in range(64) if d not in ODD]]).all()
