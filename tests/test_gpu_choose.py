"""Pages chosen by a score, against the definition in whole numbers: every bit."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_sets, ragged
from oracle import chosen_ref
from paged_case import TYPES, Cache

pytestmark = pytest.mark.gpu


class Scored:
    """A cache with digests of any content and queries, and the definition's choice."""

    def __init__(self, lens, heads, rep, dim, size, kind="fp16", new=None, layers=1, seed=0, spread=2, digests=None, extra_entries=1):
        self.cache = Cache(lens, heads, dim, size, kind, layers=layers, seed=seed, extra_entries=extra_entries)
        gen = torch.Generator().manual_seed(seed + 77)
        pages = self.cache.k.shape[1]
        self.digest = digests if digests is not None else torch.randint(-128, 128, (layers, pages, heads, 2, dim), generator=gen, dtype=torch.int8)
        self.exponents = torch.randint(-spread, spread + 1, (layers, heads, dim), generator=gen, dtype=torch.int8)
        self.rows, self.places, self.starts = (list(range(len(lens))), [n - 1 for n in lens], None) if new is None else ragged(self.cache, new)
        self.tokens, self.heads, self.rep, self.dim, self.size = len(self.rows), heads, rep, dim, size
        self.wide = torch.randn(max(1, self.tokens), (heads * rep + 2) * dim, generator=gen).to(TYPES[kind])
        self.q = self.wide[:, dim: (heads * rep + 1) * dim].view(-1, heads * rep, dim)
        self.gdigest = self.digest.cuda()

    def digests(self):
        return qkv.Digests.make(self.cache.pages, list(self.gdigest), self.exponents.cuda())

    def run(self, most, first=1, last=1, layer=0, choice=None, spare=0):
        heads, rep, dim = self.heads, self.rep, self.dim
        wide = torch.cat([self.wide, self.wide[:1].expand(spare, -1)]).cuda()
        q = wide[:, dim: (heads * rep + 1) * dim].view(-1, heads * rep, dim)
        words = (self.cache.table.shape[1] + 31) // 32
        choice = torch.full((self.tokens + spare, heads, words), 0x55555555, dtype=torch.int32, device="cuda") if choice is None else choice
        qkv.paged_choose(self.cache.pages, self.digests(), q, most, choice, first=first, last=last, layer=layer, starts=self.starts, status=self.cache.status)
        torch.cuda.synchronize()
        if spare:
            assert bool((choice[self.tokens:] == 0x55555555).all())
        return as_sets(choice[: self.tokens], self.cache.table.shape[1])

    def want(self, most, first=1, last=1, layer=0):
        table = self.cache.gtable.cpu().numpy()
        digest = self.gdigest.cpu().numpy()
        return [[chosen_ref.choose(self.q[i, h * self.rep:(h + 1) * self.rep].float().numpy(), self.places[i], self.size, table[self.rows[i]], digest.shape[1],
                                   digest[layer, :, h], self.exponents[layer, h].numpy(), most, first, last) for h in range(self.heads)] for i in range(self.tokens)]

    def check(self, most, first=1, last=1, layer=0, spare=0):
        got = self.run(most, first, last, layer, spare=spare)
        assert got == self.want(most, first, last, layer)
        return got


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("heads,rep,dim", [(4, 1, 128), (2, 4, 128), (1, 5, 64), (2, 7, 64), (1, 20, 128), (2, 2, 256)])
def test_heads_and_types(kind, heads, rep, dim):
    x = Scored([0, 1, 7, 8, 9, 130, 700], heads, rep, dim, 8, kind, layers=2, seed=dim + rep)
    x.check(11, 1, 2, layer=1)
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("most,first,last", [(1, 0, 1), (2, 1, 1), (3, 0, 3), (9, 4, 5), (10, 4, 5), (32, 0, 1), (63, 1, 1), (64, 1, 2), (65, 1, 1), (1000, 1, 1),
                                             (2 ** 31 - 1, 2 ** 30, 2 ** 30 - 1), (40, 0, 40)])
def test_how_many(most, first, last):
    x = Scored([1, 40, 512, 513, 600], 2, 2, 64, 8, seed=most % 1000)
    got = x.check(most, first, last)
    for token, place in zip(got, x.places):
        assert all(len(h) == min(most, place // 8 + 1) for h in token)


@pytest.mark.parametrize("size", [1, 2, 32, 128])
@pytest.mark.parametrize("new", [None, [40, 0, 3, 200, 1, 130]])
def test_page_sizes(size, new):
    x = Scored([500, 0, 3, 333, 64, 130], 2, 3, 64, size, new=new, seed=size)
    x.check(9, 1, 2, spare=0 if new is None else 5)
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("kind,dim", [("fp16", 128), ("bf16", 64), ("fp16", 256)])
def test_prompts(kind, dim):
    """Tokens whose own pages differ within a tile of them, and the first tokens of a sequence."""
    x = Scored([200, 90, 17], 2, 2, dim, 4, kind, new=[200, 1, 17], seed=dim)
    x.check(13, 2, 1)
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("pages", [1023, 1025, 1100, 2049, 5000, 12000])
def test_many_pages(pages):
    x = Scored([pages, pages - 1, 5], 1, 2, 64, 1, seed=pages)
    x.check(100, 3, 4)
    x = Scored([pages + 7], 1, 1, 64, 1, new=[20], seed=pages)
    x.check(1000, 1, 1)


@pytest.mark.parametrize("pages", [700, 1000, 1500, 2000, 3000, 4090, 6000, 8190, 12000, 16300])
@pytest.mark.parametrize("heads,tokens", [(4, 600), (16, 800)])
def test_many_tokens_with_many_pages(pages, heads, tokens):
    """Thousands of choices at a time, some of them against the definition; all of them have as many pages as they should."""
    tokens = min(tokens, pages)
    x = Scored([pages], heads, 1, 64, 1, new=[tokens], seed=pages)
    got = x.run(150, 2, 3)
    assert all(len(one) == min(150, place + 1) for token, place in zip(got, x.places) for one in token)
    some = sorted({0, 1, 15, 16, 63, 64, tokens - 1} | set(range(5, tokens, 61)))
    table, digest = x.cache.gtable.cpu().numpy(), x.gdigest.cpu().numpy()
    for i in some:
        for h in range(0, heads, 3):
            assert got[i][h] == chosen_ref.choose(x.q[i, h:h + 1].float().numpy(), x.places[i], 1, table[0], digest.shape[1], digest[0, :, h],
                                                  x.exponents[0, h].numpy(), 150, 2, 3), (i, h)


def test_more_pages_than_registers_hold():
    x = Scored([17000], 1, 1, 64, 1, seed=1)
    x.check(2000, 1, 1)
    x.check(16900, 1, 1)


@pytest.mark.parametrize("size", [1, 8])
@pytest.mark.parametrize("pages", [70, 500, 1500])
def test_equal_scores(size, pages):
    """All the same, or one of a few: the lowest page first."""
    some = torch.randint(-128, 128, (3, 2, 64), generator=torch.Generator().manual_seed(1), dtype=torch.int8)
    for kinds in (1, 2, 3):
        x = Scored([pages * size, pages * size - 1], 1, 2, 64, size, seed=kinds)
        x.gdigest.copy_(some[torch.arange(x.digest.shape[1]) % kinds].view(1, -1, 1, 2, 64))
        for most in (3, pages // 3, pages - 2, pages - 1):
            x.check(most, 1, 1)


@pytest.mark.parametrize("pages,heads,tokens", [(1000, 16, 800), (1500, 16, 800), (2000, 4, 600), (3000, 4, 600), (6000, 4, 600), (12000, 4, 600)])
def test_equal_scores_of_many_tokens(pages, heads, tokens):
    some = torch.randint(-128, 128, (2, heads, 2, 64), generator=torch.Generator().manual_seed(1), dtype=torch.int8)
    x = Scored([pages], heads, 1, 64, 1, new=[tokens], seed=pages)
    x.gdigest.copy_(some[torch.arange(x.digest.shape[1]) % 2].unsqueeze(0))
    table, digest = x.cache.gtable.cpu().numpy(), x.gdigest.cpu().numpy()
    for most in (pages // 5, pages - tokens // 2):
        got = x.run(most)
        for i in (0, 100, tokens // 2, tokens - 1):
            for h in range(0, heads, 3):
                assert got[i][h] == chosen_ref.choose(x.q[i, h:h + 1].float().numpy(), x.places[i], 1, table[0], digest.shape[1], digest[0, :, h],
                                                      x.exponents[0, h].numpy(), most, 1, 1), (most, i, h)


def test_the_largest_scores():
    """Codes at the ends of their range: scores of plus and minus 127 * 128 * 2 * 256."""
    x = Scored([640], 2, 1, 256, 16, seed=2, spread=0)
    x.q[:] = torch.where(torch.arange(256) % 2 == 0, 1.0, -1.0).to(torch.float16)
    even = torch.arange(256, device="cuda") % 2 == 0
    for page in range(x.digest.shape[1]):
        good = torch.where(even, 127, -128).to(torch.int8)
        x.gdigest[0, page] = good if page % 3 == 0 else -1 - good if page % 3 == 1 else 0
    x.check(17, 1, 1)
    x.check(30, 0, 1)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_queries_of_every_size(kind):
    """Zeros, one value that dwarfs the others, subnormal ones, infinite ones, no numbers, sums that leave 32 bits; steps of every size."""
    x = Scored([300] * 9, 2, 3, 64, 8, kind, seed=4)
    t = TYPES[kind]
    big = torch.finfo(t).max
    x.q[0] = 0
    x.q[1, :, 5] = big
    x.q[2] = (torch.randn(6, 64) * 2.0 ** -20).to(t)
    x.q[3, :, ::7] = float("inf")
    x.q[4, 1, ::5] = float("nan")
    x.q[5] = big
    x.q[6] = -float("inf")
    x.q[7] = float("nan")
    if kind == "bf16":
        x.q[8] = (torch.randn(6, 64) * 2.0 ** -130).to(t)
    x.check(9, 1, 1)
    x.exponents = torch.randint(-128, 128, x.exponents.shape, dtype=torch.int8, generator=torch.Generator().manual_seed(3))
    x.check(9, 1, 1)


def test_pages_that_are_not_there():
    """Entries that name no page are left out, at the front, at the end and in between; nothing is flagged."""
    x = Scored([400, 400, 400, 200], 2, 2, 64, 8, seed=5)
    x.cache.gtable[0, 0] = -1
    x.cache.gtable[1, 49] = -1
    x.cache.gtable[2, 3:45] = x.cache.k.shape[1]
    x.cache.gtable[3, :25] = -1
    got = x.check(12, 1, 2)
    assert got[3] == [set(), set()] and all(0 not in h for h in got[0]) and int(x.cache.status) == 0


def test_prompts_that_may_not_be():
    x = Scored([40, 10], 1, 1, 64, 4, new=[40, 10], seed=6)
    want = x.want(4, 1, 1)
    x.cache.glens[1] = 4                                             # six tokens stand in front of the sequence
    got = x.run(4, 1, 1)
    assert int(x.cache.status) == qkv.STATUS_BAD_ROW
    assert got[:40] == want[:40] and got[40:46] == [[set()]] * 6 and got[46:] == want[40:44]


def test_tiles_in_several_turns():
    """More tokens than the workspace holds scores of at a time."""
    x = Scored([16300 * 4], 8, 1, 64, 4, new=[400], seed=7)
    got = x.run(40, 1, 1)
    some = [0, 63, 64, 255, 256, 399]
    table, digest = x.cache.gtable.cpu().numpy(), x.gdigest.cpu().numpy()
    for i in some:
        for h in (0, 7):
            assert got[i][h] == chosen_ref.choose(x.q[i, h:h + 1].float().numpy(), x.places[i], 4, table[0], digest.shape[1], digest[0, :, h],
                                                  x.exponents[0, h].numpy(), 40, 1, 1)


def test_captured_and_replayed():
    """A captured call follows what lengths, digests and queries are at each replay."""
    x = Scored([300, 77], 2, 2, 64, 8, seed=8)
    q = x.wide.cuda()
    view = q[:, 64: 5 * 64].view(-1, 4, 64)
    digests = x.digests()
    choice = torch.zeros((2, 2, (x.cache.table.shape[1] + 31) // 32), dtype=torch.int32, device="cuda")
    workspace = torch.empty(qkv.paged_choose_workspace(x.cache.pages, 2), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        qkv.paged_choose(x.cache.pages, digests, view, 9, choice, workspace=workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qkv.paged_choose(x.cache.pages, digests, view, 9, choice, workspace=workspace)
    for turn, lens in enumerate([(300, 77), (299, 0), (64, 77)]):
        x.cache.glens.copy_(torch.tensor(lens, dtype=torch.int32))
        x.places = [n - 1 for n in lens]
        x.gdigest.copy_(torch.randint(-128, 128, x.gdigest.shape, dtype=torch.int8, generator=torch.Generator().manual_seed(turn)))
        choice.fill_(-1)
        workspace.fill_(0xAB)
        graph.replay()
        torch.cuda.synchronize()
        assert as_sets(choice, x.cache.table.shape[1]) == x.want(9)
