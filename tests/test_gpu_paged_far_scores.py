"""Attention over pages with scores of up to 2^32 that are known exactly: the tokens with the largest score share all the weight.

One dimension of q and K carries whole numbers, so that products of q and K are exact in fp32; two different ones are at least 8 apart, times a scale of 2^8 or more.
The weight of a token is 1 / (how many have the largest score) or nothing, however a score of 2^20 or 2^30 is rounded: equal ones are rounded alike,
or half a step apart where that is 2^-13 at most (a prompt's scores, where a wave begins to round them)."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from paged_case import HALF_STEP, TYPES, Cache

pytestmark = pytest.mark.gpu

SCALES = [2.0 ** 8, 2.0 ** 12, -2.0 ** 13, 2.0 ** 17, -2.0 ** 21]


def place_scores(cache, order, scale, seed):
    """Whole numbers 8 j, j = 0 .. 255, for every token: "rising" by one every 23 tokens, "falling", or in "any" order with ties all over.  Returns j of
    every row's tokens; K holds them with the scale's sign."""
    rng, got = np.random.default_rng(seed), []
    cache.k[torch.isfinite(cache.k)] = 0.0
    for b, n in enumerate(cache.lens):
        t = np.arange(n)
        j = {"rising": np.minimum(255, t // 23), "falling": np.maximum(0, 255 - t // 23), "any": rng.integers(0, 200, n)}[order]
        for i in range(n):
            cache.k[0, cache.table[b, i // cache.size], :, i % cache.size, 0] = float(8 * j[i]) * (1.0 if scale > 0 else -1.0)
        got.append(j)
    cache.gpu()
    return got


def leaders(j, V, places):
    """The mean of V [H, T, D] over the tokens with the largest j up to each place, the mean of its size, the largest j and how many have it."""
    out, size, most, count = [], [], [], []
    for p in places:
        top = j[: p + 1].max()
        who = np.flatnonzero(j[: p + 1] == top)
        out.append(V[:, who].mean(1))
        size.append(np.abs(V[:, who]).mean(1))
        most.append(top)
        count.append(len(who))
    return np.stack(out), np.stack(size), np.array(most, dtype=np.float64), np.array(count, dtype=np.float64)


def check(got, lse, want, q0, scale, q_heads, half_step, length):
    """`half_step`: of the type weights and the result are rounded to (0 for single tokens, whose weights have 22 bits).  lse: the product with the scale, the
    scale with log2 e in it, the maximum taken off, added again and turned into a natural logarithm round once each."""
    out, size, most, count = want
    rep = q_heads // out.shape[1]
    out, size = out.repeat(rep, 1), size.repeat(rep, 1)
    bound = (half_step + 6 * 2.0 ** -22 + (length + 16) * 2.0 ** -24) * size * (1 + half_step) + half_step * np.abs(out) + (2.0 ** -24 if half_step else 0.0)
    assert (np.abs(got - out) <= bound).all(), (np.abs(got - out) / bound).max()
    want_lse = abs(scale) * 8 * most[:, None] * q0 + np.log(count)[:, None]
    assert (np.abs(lse - want_lse) <= 6 * 2.0 ** -24 * np.abs(want_lse) + 2.0 ** -20 + (length + 16) * 2.0 ** -24).all()


def queries(tokens, q_heads, dim, kind):
    """1, 2, 3 or 4 in the dimension that counts, anything in the others, where K is 0."""
    q = torch.randn(tokens, q_heads, dim, generator=torch.Generator().manual_seed(3)).to(TYPES[kind])
    q0 = 1.0 + np.arange(tokens * q_heads).reshape(tokens, q_heads) % 4
    q[..., 0] = torch.from_numpy(q0)
    return q, q0


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("order", ["rising", "falling", "any"])
@pytest.mark.parametrize("lens,heads,q_heads,dim,size", [([90, 1, 33, 120], 2, 8, 128, 16), ([2600, 77, 700], 1, 5, 64, 64), ([1300], 1, 1, 256, 8)])
def test_single_tokens(kind, scale, order, lens, heads, q_heads, dim, size):
    cache = Cache(lens, heads, dim, size, kind, seed=dim)
    j = place_scores(cache, order, scale, dim)
    q, q0 = queries(len(lens), q_heads, dim, kind)
    out, lse = torch.empty(len(lens), q_heads, dim, device="cuda"), torch.empty(len(lens), q_heads, device="cuda")
    qkv.paged_attend(cache.pages, q.cuda(), scale, out, lse)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (_, V) in enumerate(cache.rows()):
        check(out[b:b + 1], lse[b:b + 1], leaders(j[b], V, [lens[b] - 1]), q0[b:b + 1], scale, q_heads, 0.0, lens[b])


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("order", ["rising", "falling", "any"])
@pytest.mark.parametrize("new,old,heads,q_heads,dim,size", [([60, 3, 90], [500, 1, 0], 2, 8, 128, 16), ([5, 70], [3000, 0], 1, 4, 64, 64), ([40], [300], 1, 3, 256, 8),
                                                            ([2100], [0], 1, 32, 128, 64)])
def test_prompts(kind, scale, order, new, old, heads, q_heads, dim, size):
    lens, tokens = [a + b for a, b in zip(new, old)], sum(new)
    cache = Cache(lens, heads, dim, size, kind, seed=dim)
    j = place_scores(cache, order, scale, dim)
    q, q0 = queries(tokens, q_heads, dim, kind)
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    out, lse = torch.empty(tokens, q_heads, dim, dtype=TYPES[kind], device="cuda"), torch.empty(tokens, q_heads, device="cuda")
    qkv.paged_prompt(cache.pages, q.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), scale, out, lse)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, (_, V) in enumerate(cache.rows()):
        pick = list(range(new[b])) if new[b] < 200 else list(range(0, new[b], 61)) + [new[b] - 1]
        mine = [starts[b] + i for i in pick]
        check(out[mine], lse[mine], leaders(j[b], V, [old[b] + i for i in pick]), q0[mine], scale, q_heads, HALF_STEP[kind], lens[b])


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 2.4e38])
def test_the_largest_scales_leave_scores_of_zero_what_they_are(kind, scale):
    """A product of 0 scores 0, whatever the scale: all tokens weigh the same."""
    cache = Cache([90, 700], 1, 64, 16, kind, seed=5)
    q = torch.zeros(2, 2, 64, dtype=TYPES[kind])
    out, lse = torch.empty(2, 2, 64, device="cuda"), torch.empty(2, 2, device="cuda")
    qkv.paged_attend(cache.pages, q.cuda(), scale, out, lse)
    half, half_lse = torch.empty(2, 2, 64, dtype=TYPES[kind], device="cuda"), torch.empty(2, 2, device="cuda")
    qkv.paged_prompt(cache.pages, q.cuda(), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), scale, half, half_lse)
    for b, (_, V) in enumerate(cache.rows()):
        want = (V.mean(1).repeat(2, 0)[None], np.abs(V).mean(1).repeat(2, 0)[None], np.zeros(1), np.array([cache.lens[b]], dtype=np.float64))
        check(out[b:b + 1].double().cpu().numpy(), lse[b:b + 1].double().cpu().numpy(), want, np.zeros((1, 2)), 1.0, 2, 0.0, cache.lens[b])
        check(half[b:b + 1].double().cpu().numpy(), half_lse[b:b + 1].double().cpu().numpy(), want, np.zeros((1, 2)), 1.0, 2, HALF_STEP[kind], cache.lens[b])
