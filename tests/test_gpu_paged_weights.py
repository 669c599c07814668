"""Attention of single tokens over pages where most weights are next to nothing, and where values are infinite or no number."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from oracle import paged_ref
from paged_case import TYPES, Cache, score_bound

pytestmark = pytest.mark.gpu


def run(cache, q, scale, window=0, sinks=0):
    rows, heads, dim = q.shape
    out, lse = torch.full((rows, heads, dim), 7.0, device="cuda"), torch.full((rows, heads), 7.0, device="cuda")
    qkv.paged_attend(cache.pages, q.cuda(), scale, out, lse, window=window, sinks=sinks, status=cache.status)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def put(cache, row, token, k=None, v=None):
    """Writes a token's row of K or V, the same in all heads."""
    page, place = int(cache.table[row, token // cache.size]), token % cache.size
    if k is not None:
        cache.k[0, page, :, place] = k.to(cache.k.dtype)
    if v is not None:
        cache.v[0, page, :, place] = v.to(cache.v.dtype)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,heads,q_heads,dim,size", [([40, 3], 2, 4, 64, 16), ([3000, 700], 2, 4, 128, 32), ([32768], 1, 2, 64, 64), ([1500], 1, 3, 256, 8)])
@pytest.mark.parametrize("gap", [6, 14, 25, 60])
def test_one_token_outweighs_all_others_and_its_value_is_nothing(kind, lens, heads, q_heads, dim, size, gap):
    """Every other score lies about `gap` below that of one token whose value is 0: the result is what the small weights add up to.  Beside what scores,
    sums and 22 bits of a weight are off by, a weight is held to half of 2^-24 where the largest is 2^15 (fp16; bf16 reaches further down):
    2^-40 of a value for each token."""
    cache = Cache(lens, heads, dim, size, kind, seed=gap, strong=1.0)
    gen = torch.Generator().manual_seed(gap + dim)
    for x in (cache.k, cache.v):
        x[torch.isnan(x) | torch.isinf(x)] = 0.0
    cache.k[..., 0] = -2.0 * gap
    cache.k[..., 1:] *= 0.25
    cache.v.copy_(1.0 + 0.25 * torch.rand(cache.v.shape, generator=gen))
    for b, n in enumerate(lens):
        put(cache, b, n // 3, k=torch.zeros(dim), v=torch.zeros(dim))
    cache.gpu()
    q = torch.randn(len(lens), q_heads, dim, generator=gen).to(TYPES[kind]) * 0.5
    q[..., 0] = 0.5
    got, lse = run(cache, q, 1.0)
    for b, (K, V) in enumerate(cache.rows()):
        out, want_lse, each, terms, top = paged_ref.attend(q[b:b + 1].double().numpy(), K, V, [lens[b] - 1], 1.0)
        s = score_bound(terms, top, dim)
        bound = (2 * s + 6 * 2.0 ** -22 + (lens[b] + 16) * 2.0 ** -24)[..., None] * each + (2.0 ** -40 * lens[b] * np.abs(V).max() if kind == "fp16" else 0.0) + 1e-30
        err = np.abs(got[b:b + 1] - out)
        assert (err <= bound).all(), (err / bound).max()
        assert (np.abs(lse[b] - want_lse[0]) <= s[0] + 2.0 ** -21 + lens[b] * 2.0 ** -24 + 2.0 ** -22 * np.abs(want_lse[0])).all()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,size", [([50, 1], 16), ([5000, 300], 64), ([2600], 4)])
def test_a_score_of_minus_infinity_weighs_nothing(kind, lens, size):
    """All keys but two in a row have a dimension of -inf, all values but theirs are 1: the result is that of the two."""
    cache = Cache(lens, 1, 64, size, kind, seed=size, strong=1.0)
    few = Cache([min(2, n) for n in lens], 1, 64, size, kind, seed=size, strong=1.0)
    gen = torch.Generator().manual_seed(size)
    cache.k[..., 3] = -float("inf")
    cache.v.fill_(1.0)
    for b, n in enumerate(lens):
        for i, token in enumerate(sorted({n // 2, n - 1})):
            k, v = torch.randn(64, generator=gen), torch.randn(64, generator=gen) * 1e-3
            put(cache, b, token, k, v)
            put(few, b, i, k, v)
    cache.gpu()
    few.gpu()
    q = torch.randn(len(lens), 4, 64, generator=gen).abs().to(TYPES[kind]) + 0.25
    got, lse = run(cache, q, 0.3)
    want, want_lse = run(few, q, 0.3)
    # the maximum of a wave's tokens, and with it the rounding of what is taken off, is the two tokens' own where they lie in one tile; a few steps otherwise
    assert np.abs(got - want).max() <= 16 * 2.0 ** -22 * 5e-3 and np.abs(lse - want_lse).max() <= 2.0 ** -18
    for b, (K, V) in enumerate(few.rows()):
        out = paged_ref.attend(q[b:b + 1].double().numpy(), K, V, [K.shape[1] - 1], 0.3)[0]
        assert np.abs(got[b:b + 1] - out).max() <= 32 * 2.0 ** -22 * 5e-3


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("lens,heads,q_heads,dim,size,window", [([70, 9], 1, 2, 64, 16, 0), ([3000, 45, 600], 2, 8, 128, 64, 0), ([3000, 45, 600], 2, 6, 256, 8, 0),
                                                                ([2000, 500], 1, 20, 128, 32, 300), ([6000], 1, 1, 64, 128, 0)])
def test_infinite_values_reach_their_dimension_whatever_they_weigh(kind, lens, heads, q_heads, dim, size, window):
    """inf, -inf and no number in values that are seen make their own dimension the sum of them; in values that are not seen they are nothing, and what
    weighs next to nothing counts too."""
    sinks = 5 if window else 0
    cache = Cache(lens, heads, dim, size, kind, seed=dim, strong=1.0)
    inf, gen = float("inf"), torch.Generator().manual_seed(dim)
    for b, n in enumerate(lens):
        for token, d, x in ((n - 1, 3, inf), (n // 2, 7, -inf), (max(0, n - 40), 7, inf), (2, 11, inf), (n - 2, 12, float("nan")), (n // 3, 15, -inf), (4, 33, -inf)):
            page, place = int(cache.table[b, token // size]), token % size
            cache.v[0, page, :, place, d] = x
        page, place = int(cache.table[b, n // 3 // size]), n // 3 % size
        cache.k[0, page, :, place, 0] = -30000.0                      # weighs nothing at all
    cache.gpu()
    q = torch.randn(len(lens), q_heads, dim, generator=gen).to(TYPES[kind])
    q[..., 0] = 1.0
    got, lse = run(cache, q, dim ** -0.5, window, sinks)
    for b, (K, V) in enumerate(cache.rows()):
        n = lens[b]
        ts = paged_ref.seen(n - 1, n, window, sinks)
        odd = np.where(np.isfinite(V), 0.0, V)[:, ts]
        with np.errstate(invalid="ignore"):
            mark = odd.sum(1).repeat(q_heads // heads, 0)              # 0 where every value is a number
        out, want_lse, each, terms, top = paged_ref.attend(q[b:b + 1].double().numpy(), K, np.where(np.isfinite(V), V, 0.0), [n - 1], dim ** -0.5, window, sinks)
        hit = mark != 0
        assert hit.any() and np.array_equal(got[b][hit], mark[hit], equal_nan=True)
        bound = (2 * score_bound(terms, top, dim) + 6 * 2.0 ** -22 + (n + 16) * 2.0 ** -24)[..., None] * each + 2.0 ** -40 * n * 8
        assert (np.abs(got[b] - out[0])[~hit] <= bound[0][~hit]).all()
        assert np.isfinite(lse[b]).all()
    assert int(cache.status) == 0


@pytest.mark.parametrize("lens,heads", [([5000], 1), ([40, 3000, 900], 2), ([100], 1)])
def test_an_infinite_value_among_tokens_that_all_weigh_nothing(lens, heads):
    """A part of a cut sequence in which every score is -inf: its values that are infinite or no number are seen all the same."""
    cache = Cache(lens, heads, 64, 32, seed=3, strong=1.0)
    for b, n in enumerate(lens):
        for token in range(n // 2 // 32 * 32, n // 2 // 32 * 32 + 32):
            if token < n - 1:
                page, place = int(cache.table[b, token // 32]), token % 32
                cache.k[0, page, :, place, 0] = -float("inf")
                if token % 32 == 5:
                    cache.v[0, page, :, place, 9] = float("inf")
    cache.gpu()
    q = torch.randn(len(lens), heads, 64, generator=torch.Generator().manual_seed(1)).half()
    q[..., 0] = 1.0
    got, lse = run(cache, q, 0.125)
    assert not np.isfinite(got[..., 9]).any() and np.isfinite(lse).all()
    assert np.isfinite(np.delete(got, 9, -1)).all()
