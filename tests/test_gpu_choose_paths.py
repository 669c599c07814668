"""Pages chosen by a score, against the definition in whole numbers, on the ways that large batches take: tiles of 32 tokens, a token that all waves of a workgroup share
with several blocks of pages to each, many sequences, and scores that go through the workspace.  Some tokens are compared with the definition; all have as many pages as they should."""
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_sets
from oracle import chosen_ref
from test_gpu_choose import Scored

pytestmark = pytest.mark.gpu


def compare(x, got, most, first, last, tokens, heads=None):
    table, digest = x.cache.gtable.cpu().numpy(), x.gdigest.cpu().numpy()
    for token, place in zip(got, x.places):
        assert all(len(h) == min(most, place // x.size + 1) for h in token)
    for i in tokens:
        for h in heads or range(x.heads):
            assert got[i][h] == chosen_ref.choose(x.q[i, h * x.rep:(h + 1) * x.rep].float().numpy(), x.places[i], x.size, table[x.rows[i]], digest.shape[1], digest[0, :, h],
                                                  x.exponents[0, h].numpy(), most, first, last), (i, h)


def few_kinds(x, kinds):
    """Digests that are one of a few, for scores that are equal."""
    some = torch.randint(-128, 128, (kinds, x.heads, 2, x.dim), generator=torch.Generator().manual_seed(1), dtype=torch.int8)
    x.gdigest.copy_(some[torch.arange(x.digest.shape[1]) % kinds].unsqueeze(0))


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("pages", [200, 380])
def test_tiles_of_32_tokens(kind, dim, pages):
    """Up to 384 pages, 32 tokens of a sequence or more, 8192 choices or more; the first tokens of a sequence and ends of tiles among those that are compared."""
    lens = [pages * 4 - 3, pages * 3]
    new = [lens[0] - 20, max(33, 1100 - lens[0])]
    x = Scored(lens, 8, 2, dim, 4, kind, new=new, seed=dim + pages)
    while x.tokens * 8 < 8192:                                       # 200 pages are too few for that many tokens of two sequences
        lens, new = lens + [pages * 4], new + [pages * 2]
        x = Scored(lens, 8, 2, dim, 4, kind, new=new, seed=dim + pages)
    assert x.tokens >= 32 * len(lens) and x.cache.table.shape[1] <= 384
    some = sorted({0, 1, 31, 32, 33, new[0] - 1, new[0], new[0] + 31, new[0] + 32, x.tokens - 1} | set(range(7, x.tokens, 97)))
    compare(x, x.run(23, 2, 3, spare=3), 23, 2, 3, some)
    compare(x, x.run(150, 1, 1), 150, 1, 1, some[::4])
    for kinds in (1, 3):
        few_kinds(x, kinds)
        compare(x, x.run(40, 1, 2), 40, 1, 2, some[::3])
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("pages", [520, 1100, 2040])
@pytest.mark.parametrize("kind,dim", [("fp16", 64), ("bf16", 128), ("fp16", 256)])
def test_single_tokens_of_many_sequences(pages, kind, dim):
    """512 to 2048 pages and 256 (sequence, kv head) pairs or more: a workgroup has several blocks of 64 pages to a wave."""
    lens = [pages, pages - 1, pages - 63, 64 * 8 + 1, 65, 1, 0] + [1 + 37 * i % 500 for i in range(25)]
    x = Scored(lens, 8, 1, dim, 1, kind, seed=pages)
    assert len(lens) * 8 >= 256 and 512 < (x.cache.table.shape[1] + 63) // 64 * 64 <= 2048
    for most, first, last in ((64, 1, 1), (400, 70, 3)):
        compare(x, x.run(most, first, last), most, first, last, range(9), (0, 3, 7))
    for kinds in (1, 2, 3):
        few_kinds(x, kinds)
        for most in (5, pages // 2, pages - 2):
            compare(x, x.run(most), most, 1, 1, range(4), (0, 7))


def test_new_tokens_of_many_sequences():
    """More sequences than a wave has lanes, some of them without new tokens."""
    lens = [3 + 29 * i % 300 for i in range(150)]
    new = [0 if i % 4 == 1 else min(lens[i], 1 + 11 * i % 40) for i in range(150)]
    x = Scored(lens, 2, 2, 64, 8, new=new, seed=1)
    compare(x, x.run(9, 1, 2, spare=4), 9, 1, 2, range(0, x.tokens, 13))
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("bf16", 128), ("fp16", 128), ("bf16", 256), ("fp16", 256)])
@pytest.mark.parametrize("rows", [3, 70])
def test_several_sequences_through_the_workspace(kind, dim, rows):
    """More pages than LDS has room for scores of: tiles of 64 tokens of three sequences, and of 16 of seventy."""
    lens = [1700, 900, 300] + [1 + 7 * i % 60 for i in range(rows - 3)]
    new = [150, 70, 33] + [min(n, 1 + n % 5) for n in lens[3:]]
    x = Scored(lens, 2, 2, dim, 1, kind, new=new, seed=dim + rows)
    assert qkv.paged_choose_workspace(x.cache.pages, x.tokens) > 0
    compare(x, x.run(60, 2, 3, spare=2), 60, 2, 3, sorted({0, 63, 64, 149, 150, 213, 219, 220, 252, x.tokens - 1} | set(range(5, x.tokens, 31))))
    few_kinds(x, 2)
    compare(x, x.run(200), 200, 1, 1, (0, 64, 149, 151, 252))


def call(x, q, choice, workspace, most=60, starts=None):
    qkv.paged_choose(x.cache.pages, x.gpu_digests, q, most, choice, first=2, last=3, starts=starts, workspace=workspace, status=x.cache.status)


def through_the_workspace(seed, single):
    x = Scored([1700, 1650, 4], 2, 2, 64, 1, new=None if single else [100, 30, 4], seed=seed)
    x.gpu_digests = x.digests()
    wide = x.wide.cuda()
    q = wide[:, x.dim: (x.heads * x.rep + 1) * x.dim].view(-1, x.heads * x.rep, x.dim)
    choice = torch.zeros((x.tokens, x.heads, (x.cache.table.shape[1] + 31) // 32), dtype=torch.int32, device="cuda")
    return x, q, choice


@pytest.mark.parametrize("single", [True, False])
def test_the_workspace_of_a_larger_batch(single):
    """What is named for a number of tokens is enough for fewer; what it holds does not matter, and nothing is written behind it."""
    x, q, choice = through_the_workspace(3, single)
    need = qkv.paged_choose_workspace(x.cache.pages, x.tokens)
    with pytest.raises(qkv.QkvError):
        call(x, q, choice, torch.empty(0, dtype=torch.uint8, device="cuda"), starts=x.starts)
    want = None
    for tokens in (x.tokens, 400, 3000):
        size = qkv.paged_choose_workspace(x.cache.pages, tokens)
        assert size >= need > 0
        for fill in (0x00, 0xAB, 0x7F, 0xFF):
            workspace = torch.full((size + 256,), fill, dtype=torch.uint8, device="cuda")
            choice.fill_(-1)
            call(x, q, choice, workspace[:size], starts=x.starts)
            got = as_sets(choice, x.cache.table.shape[1])
            assert bool((workspace[size:] == fill).all())
            if want is None:
                compare(x, got, 60, 2, 3, sorted({0, 1, x.tokens - 1}))
                want = got
            assert got == want
    assert int(x.cache.status) == 0


@pytest.mark.parametrize("single", [True, False])
def test_captured_and_replayed_through_the_workspace(single):
    """Lengths, digests and queries are those at each replay, with eager calls that have a workspace of their own in between."""
    x, q, choice = through_the_workspace(4, single)
    workspace = torch.empty(qkv.paged_choose_workspace(x.cache.pages, x.tokens), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(x, q, choice, workspace, starts=x.starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(x, q, choice, workspace, starts=x.starts)
    for turn, lens in enumerate([(1700, 1650, 4), (900, 1600, 4), (101, 30, 4), (1700, 1650, 4)]):
        x.cache.glens.copy_(torch.tensor(lens, dtype=torch.int32))
        gen = torch.Generator().manual_seed(turn)
        x.gdigest.copy_(torch.randint(-128, 128, x.gdigest.shape, dtype=torch.int8, generator=gen))
        q.copy_(torch.randn(q.shape, generator=gen))
        workspace.fill_(0xAB)
        choice.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        other = torch.full_like(choice, 5)
        call(x, q, other, None, starts=x.starts)
        torch.cuda.synchronize()
        assert torch.equal(other, choice)
        x.places = [n - 1 for n in lens] if single else [lens[b] - n + i for b, n in enumerate([100, 30, 4]) for i in range(n)]
        x.q = q.cpu()
        compare(x, as_sets(choice, x.cache.table.shape[1]), 60, 2, 3, sorted({0, 1, x.tokens - 1}))


@pytest.mark.parametrize("single", [True, False])
def test_two_streams_with_a_workspace_each(single):
    """Two batches at once, over and over; with workspaces that are given and with those that calls take by themselves."""
    made = [through_the_workspace(seed, single) for seed in (5, 6)]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for given in (True, False):
        spaces = [torch.empty(qkv.paged_choose_workspace(x.cache.pages, x.tokens), dtype=torch.uint8, device="cuda") if given else None for x, _, _ in made]
        torch.cuda.synchronize()
        for _ in range(20):
            for (x, q, choice), stream, space in zip(made, streams, spaces):
                with torch.cuda.stream(stream):
                    choice.fill_(-1)
                    call(x, q, choice, space, starts=x.starts)
        torch.cuda.synchronize()
        for x, _, choice in made:
            compare(x, as_sets(choice, x.cache.table.shape[1]), 60, 2, 3, sorted({0, 1, x.tokens - 1}))
