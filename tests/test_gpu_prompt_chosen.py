"""Attention of many new tokens over the pages chosen for each, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_words, draw_choices, expected, ragged
from paged_case import TYPES, Cache, check_prompt

pytestmark = pytest.mark.gpu


def queries(tokens, heads, dim, kind, seed=5):
    wide = torch.randn(tokens, (heads + 3) * dim, generator=torch.Generator().manual_seed(seed)).to(TYPES[kind])
    return wide, wide[:, dim: (heads + 1) * dim].view(tokens, heads, dim)


def run(cache, new, choices, q_heads, dim, scale, layer=0, spare=0, workspace=None, with_lse=True):
    rows, places, starts = ragged(cache, new)
    tokens = len(rows)
    wide, q = queries(tokens + spare, q_heads, dim, cache.kind)
    gq = wide.cuda()[:, dim: (q_heads + 1) * dim].view(tokens + spare, q_heads, dim)
    out = torch.full((tokens + spare, q_heads, dim), 7.0, device="cuda", dtype=TYPES[cache.kind])
    lse = torch.full((tokens + spare, q_heads), 7.0, device="cuda") if with_lse else None
    words = as_words(choices + [choices[0]] * spare, cache.table.shape[1])
    qkv.paged_prompt_chosen(cache.pages, words, gq, starts, scale, out, lse, layer=layer, workspace=workspace, status=cache.status)
    torch.cuda.synchronize()
    if spare:
        assert bool((out[tokens:] == 7.0).all()) and (lse is None or bool((lse[tokens:] == 7.0).all()))
    return q[:tokens], out[:tokens].double().cpu().numpy(), None if lse is None else lse[:tokens].double().cpu().numpy()


def check(cache, new, choices, q_heads, dim, scale, layer=0, spare=0, lost=(), some=None, workspace=None, with_lse=True):
    """`some`: which tokens are compared, all by default."""
    rows, places, _ = ragged(cache, new)
    q, out, lse = run(cache, new, choices, q_heads, dim, scale, layer, spare, workspace, with_lse)
    some = list(range(len(rows))) if some is None else some
    want = expected(cache, q[some].double().numpy(), [rows[i] for i in some], [places[i] for i in some], [choices[i] for i in some], scale, layer, lost)
    most = max((float(np.abs(v).max()) for _, v in cache.rows(layer) if v.size), default=0.0)
    check_prompt(out[some], None if lse is None else lse[some], want, dim, max(cache.lens), cache.kind, most)
    return out, lse


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim", [(4, 4, 128), (8, 2, 128), (5, 1, 64), (14, 2, 64), (34, 2, 64), (4, 2, 256), (128, 1, 64)])
def test_heads_and_types(kind, q_heads, heads, dim):
    cache = Cache([70, 0, 133, 33, 1], heads, dim, 16, kind, layers=2, seed=dim + q_heads)
    new = [70, 0, 40, 1, 1]
    rows, places, _ = ragged(cache, new)
    check(cache, new, draw_choices(cache, rows, heads, 0.4, q_heads), q_heads, dim, dim ** -0.5, layer=1, spare=3)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 2, 4, 8, 16, 32, 64, 512])
@pytest.mark.parametrize("layout", ["heads", "tokens", "both"])
def test_page_sizes_and_layouts(size, layout):
    cache = Cache([300, 0, 64, 7], 2, 64, size, layout=layout, seed=size)
    new = [90, 0, 64, 3]
    rows, places, _ = ragged(cache, new)
    check(cache, new, draw_choices(cache, rows, 2, 0.3, size), 6, 64, 0.1)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 2, 4, 8, 16, 32, 64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_large_batches(size, kind):
    """Workgroups of eight waves, which take 64 keys at a time."""
    cache = Cache([700], 1, 128, size, kind, seed=size)
    choices = draw_choices(cache, range(600), 1, 0.1, size)
    q_heads = 110
    assert 600 * q_heads >= 256 * 256
    check(cache, [600], choices, q_heads, 128, 0.09, some=[0, 1, 2, 63, 64, 300, 599])


@pytest.mark.parametrize("share", [0.0, 0.02, 0.9, 1.0])
@pytest.mark.parametrize("size", [4, 64])
def test_none_few_most_and_all(share, size):
    cache = Cache([400, 20], 2, 64, size, "bf16", seed=size)
    new = [100, 20]
    rows, places, _ = ragged(cache, new)
    choices = draw_choices(cache, rows, 2, share, size)
    out, lse = check(cache, new, choices, 6, 64, 0.125)
    if share == 0.0:
        assert (out == 0).all() and np.isneginf(lse).all()


def test_tokens_that_share_nothing():
    """Every token has one page of its own, another one than its neighbours; every third has none."""
    cache = Cache([500], 1, 64, 8, seed=1)
    choices = [[set() if i % 3 == 0 else {(i * 7) % 50}] for i in range(90)]
    check(cache, [90], choices, 4, 64, 0.2)


@pytest.mark.parametrize("size,length", [(1, 8300), (1, 17000), (4, 33000), (64, 9000)])
@pytest.mark.parametrize("new", [3, 70])
def test_long_lists(size, length, new):
    """More pages than a list holds; keys in parts where there are few tokens."""
    cache = Cache([length], 1, 64, size, seed=size)
    width = cache.table.shape[1]
    gen = np.random.default_rng(size)
    choices = [[set(gen.integers(0, width, 40).tolist()) | {0, (length - new + i) // size}] for i in range(new)]
    choices[1] = [set(range(width))]
    choices[2] = [{8191 if size == 1 else 5}]
    assert size != 1 or qkv.paged_prompt_chosen_workspace(cache.pages, 2, new) > 0
    check(cache, [new], choices, 2, 64, 0.2, some=list(range(min(new, 12))))


def test_many_rows():
    lens = [5 + 13 * i % 60 for i in range(150)]
    cache = Cache(lens, 1, 64, 8, seed=2)
    new = [1 + i % 5 for i in range(150)]
    rows, _, _ = ragged(cache, new)
    check(cache, new, draw_choices(cache, rows, 1, 0.4, 1), 4, 64, 0.2)


def test_pages_that_are_not_there():
    cache = Cache([200], 2, 64, 16, seed=4)
    choices = draw_choices(cache, range(50), 2, 0.3, 4)
    for token in choices:
        for h in token:
            h.discard(7)                                             # nobody has chosen it
            h.discard(12)
            h.discard(13)
    lost = {(0, 1), (0, 5)}
    for j in (1, 5, 7):
        cache.gtable[0, j] = -1 if j != 5 else cache.k.shape[1]
    check(cache, [50], choices, 4, 64, 0.2, lost=lost)
    assert int(cache.status) == qkv.STATUS_BAD_PAGE
    cache.status.zero_()
    for token in choices:
        for h in token:
            h -= {1, 5}
    check(cache, [50], choices, 4, 64, 0.2)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [8, 32, 64])
def test_all_tokens_choose_a_page_that_is_not_there(size):
    cache = Cache([400], 1, 64, size, seed=14)
    cache.gtable[0, 1] = -1
    check(cache, [70], [[{0, 1, 2, 3, (330 + i) // size}] for i in range(70)], 4, 64, 0.2, lost={(0, 1)})
    assert int(cache.status) == qkv.STATUS_BAD_PAGE


@pytest.mark.parametrize("size", [4, 32, 64])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_what_is_infinite_or_no_number(size, kind):
    """In pages nobody or another token has chosen, and behind a token's place, it counts for nothing; where it is seen, for its own dimension."""
    cache = Cache([300], 1, 64, size, kind, seed=5)
    clean = Cache([300], 1, 64, size, kind, seed=5)
    places = list(range(260, 300))
    choices = [[{0, 2} if i % 2 else {0, 3}] for i in range(40)]
    for i in range(20, 40):
        choices[i][0].add((260 + i) // size)
    cache.k[:, cache.table[0, 1].long()] = float("nan")
    cache.v[:, cache.table[0, 1].long()] = float("inf")
    cache.v[0, cache.table[0, 3], 0, 1, 10] = float("inf")           # the even ones see it
    cache.v[0, cache.table[0, 2], 0, 2, 11] = float("nan")           # the odd ones do
    cache.v[0, cache.table[0, 290 // size], 0, 290 % size, 12] = -float("inf")
    cache.gpu()
    q, out, lse = run(cache, [40], choices, 2, 64, 0.2)
    want = expected(clean, q.double().numpy(), [0] * 40, places, choices, 0.2)
    for i in range(40):
        sees = {10: i % 2 == 0, 11: i % 2 == 1, 12: i >= 30 and 290 // size in choices[i][0]}
        for d, some in sees.items():
            if some:
                assert (np.isnan(out[i, :, d]) if d == 11 else np.isinf(out[i, :, d]) & (np.sign(out[i, :, d]) == (1 if d == 10 else -1))).all(), (i, d)
                out[i, :, d] = want[0][i, :, d]
    check_prompt(out, lse, want, 64, 300, kind, 20.0)


@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0, 3e4])
def test_scales(scale):
    """Scores beyond 2^12, where a maximum's own rounding counts, among them."""
    cache = Cache([150], 2, 64, 8, seed=6)
    choices = draw_choices(cache, range(60), 2, 0.5, 2)
    if scale == 3e4:
        _, out, lse = run(cache, [60], choices, 4, 64, scale)
        assert np.isfinite(out).all()
    else:
        check(cache, [60], choices, 4, 64, scale)


def test_batches_that_may_not_be():
    cache = Cache([40, 10], 1, 64, 4, seed=7)
    rows, _, _ = ragged(cache, [40, 10])
    choices = draw_choices(cache, rows, 1, 0.6, 1)
    want = run(cache, [40, 10], choices, 2, 64, 0.2)
    cache.glens[1] = 4                                               # six tokens stand in front of the sequence
    got = run(cache, [40, 10], choices, 2, 64, 0.2)
    assert int(cache.status) == qkv.STATUS_BAD_ROW
    assert np.array_equal(got[1][:40], want[1][:40]) and (got[1][40:46] == 0).all() and np.isneginf(got[2][40:46]).all()


def test_the_workspace_for_a_batch_is_enough_for_smaller_ones():
    cache = Cache([5000], 2, 64, 16, seed=8)
    sizes = [qkv.paged_prompt_chosen_workspace(cache.pages, 8, n) for n in range(1, 3000, 7)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    need = qkv.paged_prompt_chosen_workspace(cache.pages, 8, 40)
    workspace = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    choices = draw_choices(cache, range(40), 2, 0.05, 1)
    check(cache, [40], choices, 8, 64, 0.2, workspace=workspace[:need])
    assert bool((workspace[need:] == 0xFF).all())


def test_captured_and_replayed():
    cache = Cache([3000, 77], 2, 64, 16, seed=9)
    new = [30, 10]
    rows, _, starts = ragged(cache, new)
    q = queries(40, 4, 64, "fp16")[1].cuda()
    out, lse = torch.zeros(40, 4, 64, device="cuda", dtype=torch.float16), torch.zeros(40, 4, device="cuda")
    words = as_words(draw_choices(cache, rows, 2, 0.1, 1), cache.table.shape[1])
    workspace = torch.empty(qkv.paged_prompt_chosen_workspace(cache.pages, 4, 40), dtype=torch.uint8, device="cuda")
    assert workspace.numel() > 0
    qkv.paged_prompt_chosen(cache.pages, words, q, starts, 0.2, out, lse, workspace=workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qkv.paged_prompt_chosen(cache.pages, words, q, starts, 0.2, out, lse, workspace=workspace)
    for turn, lens in enumerate([(3000, 77), (30, 10), (2000, 50)]):
        cache.glens.copy_(torch.tensor(lens, dtype=torch.int32))
        words.copy_(as_words(draw_choices(cache, rows, 2, 0.1, turn), cache.table.shape[1]))
        out.fill_(9.0)
        workspace.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        other, other_lse = torch.zeros_like(out), torch.zeros_like(lse)
        qkv.paged_prompt_chosen(cache.pages, words, q, starts, 0.2, other, other_lse)
        torch.cuda.synchronize()
        assert torch.equal(other, out) and torch.equal(other_lse, lse)
