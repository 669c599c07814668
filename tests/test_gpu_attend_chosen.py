"""Attention of single tokens over chosen pages, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_words, draw_choices, expected
from oracle import paged_ref
from paged_case import TYPES, Cache, check_attend

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 31, 32, 33, 129, 500]


def queries(rows, heads, dim, kind, seed=5):
    wide = torch.randn(rows, (heads + 3) * dim, generator=torch.Generator().manual_seed(seed)).to(TYPES[kind])
    return wide, wide[:, dim: (heads + 1) * dim].view(rows, heads, dim)


def run(cache, choices, q_heads, dim, scale, layer=0, most=0, prior=None, with_lse=True, workspace=None, q=None):
    rows = len(cache.lens)
    wide, mine = queries(rows, q_heads, dim, cache.kind)
    gq = wide.cuda()[:, dim: (q_heads + 1) * dim].view(rows, q_heads, dim) if q is None else q.cuda()
    out = torch.full((rows, q_heads, dim), 7.0, device="cuda")
    lse = torch.full((rows, q_heads), 7.0, device="cuda") if with_lse else None
    words = choices if torch.is_tensor(choices) else as_words(choices, cache.table.shape[1])
    qkv.paged_attend_chosen(cache.pages, words, gq, scale, out, lse, layer=layer, most=most, prior=prior, workspace=workspace, status=cache.status)
    torch.cuda.synchronize()
    return (mine if q is None else q), out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()


def check(cache, choices, q_heads, dim, scale, layer=0, most=0, lost=(), with_lse=True):
    places = [n - 1 for n in cache.lens]
    q, out, lse = run(cache, choices, q_heads, dim, scale, layer, most, with_lse=with_lse)
    want = expected(cache, q.double().numpy(), range(len(cache.lens)), places, choices, scale, layer, lost)
    check_attend(out, lse, want, dim, max(cache.lens))


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim", [(4, 4, 128), (8, 2, 128), (5, 1, 64), (14, 2, 64), (34, 2, 64), (20, 1, 128), (4, 2, 256)])
@pytest.mark.parametrize("most", [0, 3])
def test_heads_and_types(kind, q_heads, heads, dim, most):
    """With and without a word about how many are chosen: items in parts and whole."""
    cache = Cache(LENGTHS, heads, dim, 16, kind, layers=2, seed=dim + q_heads)
    choices = draw_choices(cache, LENGTHS, heads, 0.4, q_heads)
    check(cache, choices, q_heads, dim, dim ** -0.5, layer=1, most=most)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 2, 8, 16, 32, 64, 512])
@pytest.mark.parametrize("layout", ["heads", "tokens", "both"])
def test_page_sizes_and_layouts(size, layout):
    cache = Cache([300, 0, 64, 7], 2, 128, size, layout=layout, seed=size)
    check(cache, draw_choices(cache, cache.lens, 2, 0.5, size), 6, 128, 0.07)
    assert int(cache.status) == 0


@pytest.mark.parametrize("share", [0.0, 0.03, 0.9, 1.0])
@pytest.mark.parametrize("size", [4, 64])
def test_none_few_most_and_all(share, size):
    """Rows that see nothing; all pages, which is attention over all of them, and rows of 40 that are not cut."""
    cache = Cache([700, 1, 0, 65, 256] + [90] * 35, 2, 64, size, "bf16", seed=size)
    choices = draw_choices(cache, cache.lens, 2, share, size)
    check(cache, choices, 6, 64, 0.125)
    if share == 1.0:
        q, out, lse = run(cache, choices, 6, 64, 0.125)
        other, other_lse = torch.empty(40, 6, 64, device="cuda"), torch.empty(40, 6, device="cuda")
        qkv.paged_attend(cache.pages, q.cuda(), 0.125, other, other_lse)
        np.testing.assert_allclose(out, other.double().cpu().numpy(), atol=2.0 ** -12)


def test_only_the_own_page():
    cache = Cache([33, 64, 1, 100], 2, 64, 32, seed=1)
    choices = [[{(n - 1) // 32}, {0}] for n in cache.lens]
    check(cache, choices, 4, 64, 0.2)


@pytest.mark.parametrize("size,length", [(1, 9000), (4, 33000), (64, 9000)])
def test_long_lists(size, length):
    """More pages than a list holds, and bits far apart."""
    cache = Cache([length, 3], 1, 64, size, seed=size)
    width = cache.table.shape[1]
    choices = [[set(range(0, width, 3)) | {width - 2}], [{0, 1, 2}]]
    check(cache, choices, 2, 64, 0.2)
    check(cache, [[{0, (length - 1) // size}], [set()]], 2, 64, 0.2, most=2)


def test_many_rows():
    cache = Cache([17 * i % 200 for i in range(300)], 2, 64, 8, seed=2)
    check(cache, draw_choices(cache, cache.lens, 2, 0.3, 1), 4, 64, 0.2, most=8)


@pytest.mark.parametrize("rows", [1, 30])
def test_joined(rows):
    """With what attention over other tokens gave: also where nothing is chosen, and where the other saw nothing."""
    cache = Cache([400, 0, 90][:1] + [50] * (rows - 1) if rows > 1 else [400], 2, 128, 16, seed=rows)
    choices = draw_choices(cache, cache.lens, 2, 0.3, rows)
    if rows > 1:
        choices[2] = [set(), set()]
    gen = torch.Generator().manual_seed(3)
    other, other_lse = torch.randn(rows, 6, 128, generator=gen), torch.randn(rows, 6, generator=gen) + 3
    if rows > 1:
        other_lse[2] = -float("inf")
        other_lse[3] = -float("inf")
    q, out, lse = run(cache, choices, 6, 128, 0.1, prior=(other.cuda(), other_lse.cuda()))
    want = expected(cache, q.double().numpy(), range(rows), [n - 1 for n in cache.lens], choices, 0.1)
    o, l = paged_ref.joined(want[0], want[1], other.double().numpy(), other_lse.double().numpy())
    # the join's two exponentials, their sum and quotients: a handful of half steps, of both sides' sizes
    size = np.maximum(want[2], np.abs(other.double().numpy()))
    check_attend(out, lse, (o, l, size, want[3], np.maximum(want[4], np.abs(np.where(np.isfinite(l), l, 0)))), 128, 400 + 64)


def test_pages_that_are_not_there():
    cache = Cache([200, 200, 64], 2, 64, 16, seed=4)
    choices = [[{0, 1, 5, 9}, {1, 2}], [{3}, {0, 12}], [{0, 2, 3}, {1}]]
    cache.gtable[0, 1] = -1
    cache.gtable[1, 3] = cache.k.shape[1]
    cache.gtable[2, 3] = -7
    cache.gtable[0, 7] = -1                                          # nobody has chosen it
    check(cache, choices, 4, 64, 0.2, lost={(0, 1), (1, 3), (2, 3)})
    assert int(cache.status) == qkv.STATUS_BAD_PAGE
    cache.status.zero_()
    check(cache, [[{0, 5}, {2}], [{1}, {0}], [{0}, {1}]], 4, 64, 0.2)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [8, 32])
def test_what_is_infinite_or_no_number(size):
    """In pages that are not chosen, behind the length and in what has no page it counts for nothing; where it is seen, for its own dimension."""
    cache = Cache([300, 300], 1, 64, size, seed=5)
    last = 299 // size
    choices = [[{0, 2, last}], [{0, 2, last}]]
    for j in (1, 3, 4):
        cache.k[:, cache.table[0, j].long()] = float("nan")
        cache.v[:, cache.table[0, j].long()] = float("inf")
    cache.v[0, cache.table[1, 2], 0, 3, 10] = float("inf")
    cache.v[0, cache.table[1, 0], 0, 1, 11] = -float("inf")
    cache.v[0, cache.table[1, last], 0, 0, 12] = float("nan")
    cache.v[0, cache.table[1, 3], 0, 0, 13] = float("nan")           # not chosen
    cache.v[0, cache.table[1, 0], 0, 0, 14] = float("inf")
    cache.v[0, cache.table[1, 2], 0, 0, 14] = -float("inf")
    cache.gpu()
    q, out, lse = run(cache, choices, 2, 64, 0.2)
    clean = Cache([300, 300], 1, 64, size, seed=5)
    want = expected(clean, q.double().numpy(), [0, 1], [299, 299], choices, 0.2)
    assert np.isposinf(out[1, :, 10]).all() and np.isneginf(out[1, :, 11]).all() and np.isnan(out[1, :, 12]).all() and np.isnan(out[1, :, 14]).all()
    out[1][:, [10, 11, 12, 14]] = want[0][1][:, [10, 11, 12, 14]]
    check_attend(out, lse, want, 64, 300)


@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0, 1e-30])
def test_scales(scale):
    cache = Cache([120, 40], 2, 64, 8, seed=6)
    check(cache, draw_choices(cache, cache.lens, 2, 0.5, 2), 4, 64, scale)


def test_without_lse_and_with_a_workspace_of_its_own():
    cache = Cache([900], 1, 128, 16, seed=7)
    choices = draw_choices(cache, [900], 1, 0.5, 3)
    check(cache, choices, 4, 128, 0.1, with_lse=False)
    need = qkv.paged_attend_chosen_workspace(cache.pages, 4, 20)
    assert need > 0
    workspace = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    a = run(cache, choices, 4, 128, 0.1, most=20, workspace=workspace[:need])
    assert bool((workspace[need:] == 0xFF).all())
    b = run(cache, choices, 4, 128, 0.1, most=20, workspace=workspace[:need])
    assert np.array_equal(a[1], b[1])


def test_captured_and_replayed():
    """A captured call follows lengths, choices and queries as they are at each replay, with eager calls in between."""
    cache = Cache([300, 77], 2, 64, 8, seed=8)
    q = queries(2, 4, 64, "fp16")[1].cuda()
    out, lse = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 4, device="cuda")
    words = as_words(draw_choices(cache, cache.lens, 2, 0.5, 1), cache.table.shape[1])
    workspace = torch.empty(qkv.paged_attend_chosen_workspace(cache.pages, 4), dtype=torch.uint8, device="cuda")
    qkv.paged_attend_chosen(cache.pages, words, q, 0.2, out, lse, workspace=workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qkv.paged_attend_chosen(cache.pages, words, q, 0.2, out, lse, workspace=workspace)
    for turn, lens in enumerate([(300, 77), (17, 0), (256, 50)]):
        cache.glens.copy_(torch.tensor(lens, dtype=torch.int32))
        choices = draw_choices(cache, lens, 2, 0.5, turn)
        words.copy_(as_words(choices, cache.table.shape[1]))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.double().cpu().numpy(), lse.double().cpu().numpy()
        other, other_lse = torch.zeros_like(out), torch.zeros_like(lse)
        qkv.paged_attend_chosen(cache.pages, words, q, 0.2, other, other_lse)
        assert torch.equal(other, out) and torch.equal(other_lse, lse)
        held = cache.lens
        cache.lens = list(lens)
        want = expected(cache, q.double().cpu().numpy(), [0, 1], [n - 1 for n in lens], choices, 0.2)
        check_attend(*got, want, 64, 300)
        cache.lens = held
