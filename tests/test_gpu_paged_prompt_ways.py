"""Which way a wave of the prompt kernel takes shows in nothing but its roundings: where the same pairs see the same keys, the same bits."""
import pytest
import torch

import paper_2605_03884_amd as qkv
from paged_case import TYPES, Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim,heads,new,window", [(64, 2, 32, 384), (128, 2, 32, 384), (256, 1, 32, 384), (128, 32, 2080, 384)])
def test_a_pair_that_sees_none_of_the_first_keys_changes_nothing_for_the_others(kind, dim, heads, new, window):
    """The last 32 query tokens fill a wave, their window starts with a tile, and (for all pairs but a few, which are left out) the largest score is
    that of the one key of it that all of them see.  Without the last token its place in the wave sees nothing there; the 31 others see what they saw,
    and their running maximum stays what it is from there on, whatever makes it be looked at again.
    Scores lie around -250, where a score that is rounded and one that is not give weights that are apart."""
    cache = Cache([window + 64 + new], heads, dim, 64, kind, seed=dim, strong=1.0)
    first = window + 64 + new - 32 - window + 1                       # the first key that the first of the 32 sees
    length = window + 64 + new - first % 64
    first -= first % 64
    for b, j in ((0, t) for t in range(length)):
        page = cache.table[b, j // 64]
        cache.k[0, page, :, j % 64, 0] = -980.0 if j == first + 31 else -1000.0
    cache.gpu()
    gen = torch.Generator().manual_seed(7)
    q = torch.randn(new, heads, dim, generator=gen).to(TYPES[kind])
    q[..., 0] = 4.0
    q[-1] = 0.0
    base, keys = length - 32, cache.rows()[0][0]
    scores = torch.einsum("nhd,htd->nht", q[new - 32: new - 1].double(), torch.from_numpy(keys))
    place, t = base + torch.arange(31)[:, None, None], torch.arange(keys.shape[1])
    scores = scores.masked_fill((t > place) | (t <= place - window), -float("inf"))
    held = scores.argmax(2) == first + 31
    assert held.double().mean() > 0.9 and base - window + 1 == first
    q = q.cuda()
    got = []
    for n in (new, new - 1):
        cache.glens.fill_(length - (new - n))
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        out, lse = torch.empty(n, heads, dim, dtype=TYPES[kind], device="cuda"), torch.empty(n, heads, device="cuda")
        qkv.paged_prompt(cache.pages, q[:n], starts, 0.0625, out, lse, window=window, status=cache.status)
        got.append((out[new - 32: new - 1].cpu()[held], lse[new - 32: new - 1].cpu()[held]))
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][0], got[1][0])
    assert bool(torch.isfinite(got[0][1]).all()) and int(cache.status) == 0
