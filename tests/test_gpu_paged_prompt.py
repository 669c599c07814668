"""Attention of many new tokens over pages, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from oracle import paged_ref
from paged_case import TYPES, Cache, check_prompt

pytestmark = pytest.mark.gpu


def run(cache, new, q_heads, dim, scale, layer=0, window=0, sinks=0, behind=3, seed=5, with_lse=True):
    """`behind` tokens of the batch belong to no row."""
    tokens = sum(new) + behind
    starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
    wide = torch.randn(tokens, (q_heads + 2) * dim, generator=torch.Generator().manual_seed(seed)).to(TYPES[cache.kind])
    cut = lambda x: x[:, dim: (q_heads + 1) * dim].view(tokens, q_heads, dim)  # noqa: E731
    out = torch.full((tokens, q_heads, dim), 7.0, dtype=TYPES[cache.kind], device="cuda")
    lse = torch.full((tokens, q_heads), 7.0, device="cuda") if with_lse else None
    qkv.paged_prompt(cache.pages, cut(wide.cuda()), starts.cuda(), scale, out, lse, layer=layer, window=window, sinks=sinks, status=cache.status)
    torch.cuda.synchronize()
    out = out.double().cpu().numpy()
    assert (out[tokens - behind:] == 7.0).all() and (lse is None or (lse[tokens - behind:] == 7.0).all())
    return cut(wide)[: sum(new)], out[: sum(new)], None if lse is None else lse.double().cpu().numpy()[: sum(new)]


def expected(cache, new, q, scale, window=0, sinks=0, absent=None, layer=0):
    parts, at = [], 0
    for b, (K, V) in enumerate(cache.rows(layer)):
        n = cache.lens[b]
        parts.append(paged_ref.attend(q[at:at + new[b]].double().numpy(), K, V, list(range(n - new[b], n)), scale, window, sinks, () if absent is None else absent[b]))
        at += new[b]
    return [np.concatenate(x) for x in zip(*parts)]


def expected_fast(cache, new, q, scale, window=0, sinks=0):
    """expected() with whole matrices of a head at a time (torch, float64, on the CPU): the same definition for sizes that token by token take too long."""
    parts, at = [], 0
    for b, (K, V) in enumerate(cache.rows()):
        n, (H, T, D) = new[b], K.shape
        place, t = torch.arange(T - n, T)[:, None], torch.arange(T)[None]
        seen = (t <= place) & ((t > place - window) | (t < sinks)) if window else t <= place
        x, heads = q[at:at + n].double(), q.shape[1]
        got = [torch.zeros(n, heads, D, dtype=torch.float64), torch.full((n, heads), -float("inf"), dtype=torch.float64), torch.zeros(n, heads, D, dtype=torch.float64),
               torch.zeros(n, heads, dtype=torch.float64), torch.zeros(n, heads, dtype=torch.float64)]
        for h in range(heads if n else 0):
            k, v = (torch.from_numpy(np.ascontiguousarray(y[h // (heads // H)])) for y in (K, V))
            s = (x[:, h] @ k.T) * scale
            p = torch.softmax(s.masked_fill(~seen, -float("inf")), 1)
            got[0][:, h], got[1][:, h], got[2][:, h] = p @ v, torch.logsumexp(s.masked_fill(~seen, -float("inf")), 1), p @ v.abs()
            got[3][:, h] = (abs(scale) * (x[:, h].abs() @ k.abs().T)).masked_fill(~seen, 0).amax(1)
            got[4][:, h] = s.abs().masked_fill(~seen, 0).amax(1)
        parts.append([y.numpy() for y in got])
        at += n
    return [np.concatenate(y) for y in zip(*parts)]


def check(cache, new, got, want, dim):
    q, out, lse = got
    most = max([float(np.abs(V).max()) for _, V in cache.rows() if V.size] + [1.0])
    check_prompt(out, lse, want, dim, max(cache.lens), cache.kind, most)


NEW, OLD = [1, 0, 70, 33, 129], [0, 5, 0, 100, 64]


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim", [(4, 4, 128), (8, 2, 128), (5, 1, 64), (14, 2, 64), (34, 1, 64), (128, 1, 64), (4, 2, 256)])
def test_heads_and_types(kind, q_heads, heads, dim):
    new, old = ([1, 0, 9, 20], [0, 5, 0, 70]) if q_heads > 16 else (NEW, OLD)
    cache = Cache([a + b for a, b in zip(new, old)], heads, dim, 16, kind, layers=2, seed=dim + q_heads)
    got = run(cache, new, q_heads, dim, dim ** -0.5, layer=1)
    check(cache, new, got, expected(cache, new, got[0], dim ** -0.5, layer=1), dim)
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 8, 16, 32, 64, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens", "both"])
def test_page_sizes_and_layouts(size, layout):
    new, lens = [40, 100, 3], [40, 150, 64]
    cache = Cache(lens, 2, 128, size, layout=layout, seed=size)
    got = run(cache, new, 6, 128, 0.07)
    check(cache, new, got, expected(cache, new, got[0], 0.07), 128)
    assert int(cache.status) == 0


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (32, 0), (33, 4), (64, 64), (65, 70), (100, 1000), (130, 3), (5000, 4)])
@pytest.mark.parametrize("size", [8, 64])
def test_windows(window, sinks, size):
    """Pages that no new token sees may be gone: their entries name nothing."""
    new, old = [200, 1, 30], [150, 299, 320]
    cache = Cache([a + b for a, b in zip(new, old)], 1, 64, size, "bf16" if window == 33 else "fp16", seed=window)
    for b, n in enumerate(old):
        for j in range(-(-cache.lens[b] // size)):
            if (j + 1) * size <= n + 1 - window and j * size >= sinks:
                cache.gtable[b, j] = -1
    got = run(cache, new, 3, 64, 0.125, window=window, sinks=sinks)
    check(cache, new, got, expected(cache, new, got[0], 0.125, window, sinks), 64)
    assert int(cache.status) == 0


@pytest.mark.parametrize("new,old,window", [([5], [3000], 0), ([1], [5000], 0), ([20, 3], [2500, 0], 0), ([17], [4000], 900), ([0, 2, 0], [10, 2100, 0], 0)])
def test_few_queries_behind_many_keys(new, old, window):
    cache = Cache([a + b for a, b in zip(new, old)], 1, 64, 16, seed=len(new) + window, extra_entries=4)
    assert qkv.paged_prompt_workspace(cache.pages, 4, sum(new) + 3) > 0
    got = run(cache, new, 4, 64, 0.125, window=window, sinks=2 if window else 0)
    check(cache, new, got, expected(cache, new, got[0], 0.125, window, 2 if window else 0), 64)


@pytest.mark.parametrize("kind,size,window,sinks", [("fp16", 64, 0, 0), ("bf16", 16, 0, 0), ("fp16", 8, 300, 5), ("bf16", 128, 70, 0)])
def test_large_prompts(kind, size, window, sinks):
    """As many (token, head) pairs as give every CU a tile of 256: another kernel than small prompts have."""
    new, old = [1500, 0, 3, 640], [77, 10, 0, 1000]
    cache = Cache([a + b for a, b in zip(new, old)], 4, 128, size, kind, seed=size)
    got = run(cache, new, 32, 128, 0.09, window=window, sinks=sinks)
    check(cache, new, got, expected_fast(cache, new, got[0], 0.09, window, sinks), 128)
    assert int(cache.status) == 0


def test_large_prompts_with_an_entry_that_names_no_page_and_infinite_values():
    cache = Cache([2100], 1, 128, 16, seed=8)
    lost = set(range(1600, 1616))
    cache.v[0, cache.table[0, 125], 0, 3, 100] = float("inf")
    cache.gpu()
    cache.gtable[0, 100] = -1
    q, out, lse = run(cache, [2100], 32, 128, 0.09)
    assert int(cache.status) == qkv.STATUS_BAD_PAGE
    assert np.isposinf(out[2003:, :, 100]).all() and np.isfinite(out[:2003]).all()
    few = [0, 1, 1599, 1600, 1615, 1700, 2002, 2003, 2099]
    K, V = cache.rows()[0]
    V = np.where(np.isfinite(V), V, 0.0)
    want = paged_ref.attend(q[few].double().numpy(), K, V, few, 0.09, absent=lost)
    out = out[few]
    out[7:, :, 100] = want[0][7:, :, 100]
    check_prompt(out, lse[few], want, 128, 2100, "fp16", float(np.abs(V).max()))


@pytest.mark.parametrize("size", [8, 32, 64])
@pytest.mark.parametrize("dim", [64, 256])
def test_page_sizes_of_other_dimensions(size, dim):
    new, lens = [40, 100, 3], [40, 150, 64]
    cache = Cache(lens, 1, dim, size, seed=size)
    got = run(cache, new, 3, dim, 0.07)
    check(cache, new, got, expected(cache, new, got[0], 0.07), dim)


def test_short_and_long_sequences_in_a_wide_table():
    """The host allows parts; only the long sequences have them."""
    new, old = [9, 1, 30, 0, 4], [0, 1100, 3, 6000, 600]
    cache = Cache([a + b for a, b in zip(new, old)], 2, 64, 16, seed=21, extra_entries=3000)
    assert qkv.paged_prompt_workspace(cache.pages, 4, sum(new) + 3) > 0
    got = run(cache, new, 4, 64, 0.125)
    check(cache, new, got, expected(cache, new, got[0], 0.125), 64)


def test_many_rows():
    new = [(i * 7) % 5 for i in range(300)]
    cache = Cache([n + i % 9 for i, n in enumerate(new)], 1, 64, 8, seed=22)
    got = run(cache, new, 2, 64, 0.125)
    check(cache, new, got, expected(cache, new, got[0], 0.125), 64)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 3.0])
def test_scales(scale):
    cache = Cache([90, 33], 1, 64, 16, seed=3)
    got = run(cache, [90, 10], 4, 64, scale)
    check(cache, [90, 10], got, expected(cache, [90, 10], got[0], float(np.float32(scale))), 64)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [3e5, -3e6, 1e8, 1e10])
def test_scores_whose_steps_are_large(kind, scale):
    """fp32 scores of 2^24 and more lie 2 and more apart, and so does a maximum that is rounded: a weight beside it may not overflow."""
    new, old = [60, 3, 90], [500, 1, 0]
    cache = Cache([a + b for a, b in zip(new, old)], 2, 128, 16, kind)
    got = run(cache, new, 8, 128, scale)
    check(cache, new, got, expected(cache, new, got[0], scale), 128)


def test_scores_that_rise_from_key_to_key():
    """The running maximum moves in every tile, by more and by less than what is put up with."""
    cache = Cache([300], 1, 64, 16, seed=5, strong=1.0)
    cache.k[:] = torch.where(torch.isnan(cache.k), cache.k, cache.k * 0.05)
    for t in range(300):
        cache.k[0, cache.table[0, t // 16], 0, t % 16, 0] = t * 0.5
    cache.gpu()
    got = run(cache, [300], 2, 64, 0.3, seed=7)
    check(cache, [300], got, expected(cache, [300], got[0], float(np.float32(0.3))), 64)


@pytest.mark.parametrize("size", [16, 128])
def test_entries_that_name_no_page(size):
    cache = Cache([200, 90], 1, 64, size, seed=1)
    absent = [set(range(size, 2 * size)), set()]
    cache.gtable[0, 1] = -1
    got = run(cache, [60, 90], 4, 64, 0.125)
    check(cache, [60, 90], got, expected(cache, [60, 90], got[0], 0.125, absent=absent), 64)
    assert int(cache.status) == qkv.STATUS_BAD_PAGE


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_infinite_and_missing_numbers_behind_a_query(kind):
    """Values of later tokens do not touch the earlier ones, keys of theirs neither; a query that sees them has them in their own dimensions."""
    cache = Cache([100], 1, 64, 16, kind, seed=4)
    for t, d, x in ((50, 5, "inf"), (50, 6, "nan"), (77, 40, "-inf")):
        cache.v[0, cache.table[0, t // 16], 0, t % 16, d] = float(x)
    cache.gpu()
    q, out, lse = run(cache, [100], 2, 64, 0.125)
    K, V = cache.rows()[0]
    want = [x.copy() for x in paged_ref.attend(q.double().numpy(), K, np.where(np.isfinite(V), V, 0.0), list(range(100)), 0.125)]
    assert np.isposinf(out[50:, :, 5]).all() and np.isnan(out[50:, :, 6]).all() and np.isneginf(out[77:, :, 40]).all()
    for t, d in ((50, 5), (50, 6), (77, 40)):
        out[t:, :, d] = want[0][t:, :, d]
    check_prompt(out, lse, want, 64, 100, kind, float(np.abs(V[np.isfinite(V)]).max()))


def test_a_row_with_more_new_tokens_than_length():
    """Tokens in front of the sequence see nothing; the status word says so."""
    cache = Cache([10, 40], 1, 64, 16, seed=2)
    q, out, lse = run(cache, [15, 40], 2, 64, 0.125)
    assert int(cache.status) == qkv.STATUS_BAD_ROW
    assert (out[:5] == 0).all() and np.isneginf(lse[:5]).all()
    cache.lens = [10, 40]
    want = expected(cache, [10, 40], q[5:], 0.125)
    check_prompt(out[5:], lse[5:], want, 64, 40, "fp16", 20.0)


def test_batches_that_make_no_sense_stay_inside():
    cache = Cache([10, 40], 1, 64, 16, seed=2)
    q, out = torch.zeros(20, 2, 64, dtype=torch.float16, device="cuda"), torch.zeros(20, 2, 64, dtype=torch.float16, device="cuda")
    for starts in ([0, 500, 7], [-4, 3, 9], [30, 40, 50], [5, 2, 1]):
        cache.status.zero_()
        qkv.paged_prompt(cache.pages, q, torch.tensor(starts, dtype=torch.int32, device="cuda"), 0.125, out, status=cache.status)
        assert int(cache.status) == qkv.STATUS_BAD_ROW, starts


@pytest.mark.parametrize("rows", [63, 64, 65])
def test_rows_around_a_wave(rows):
    new = [(i * 5) % 4 for i in range(rows - 1)] + [9]
    cache = Cache([n + i % 40 for i, n in enumerate(new)], 1, 64, 16, seed=rows)
    got = run(cache, new, 2, 64, 0.125)
    check(cache, new, got, expected(cache, new, got[0], 0.125), 64)
    assert int(cache.status) == 0


def test_rows_that_share_pages_and_queries_that_share_values():
    """Two rows with the same pages, all heads with the same query (strides of 0): every result stands twice, for each head of a kv head."""
    cache = Cache([0, 700], 2, 128, 16, seed=31)
    cache.glens[0], cache.gtable[0] = 700, cache.gtable[1]
    x = torch.randn(14, 128, generator=torch.Generator().manual_seed(1)).half()
    x[7:] = x[:7]
    q = x.cuda()[:, None].expand(14, 8, 128)
    starts = torch.tensor([0, 7, 14], dtype=torch.int32, device="cuda")
    out, lse = torch.empty(14, 8, 128, dtype=torch.float16, device="cuda"), torch.empty(14, 8, device="cuda")
    qkv.paged_prompt(cache.pages, q, starts, 0.09, out, lse)
    assert torch.equal(out[:7], out[7:]) and torch.equal(lse[:7], lse[7:])
    for h in range(8):
        assert torch.equal(out[:, h], out[:, h // 4 * 4]) and torch.equal(lse[:, h], lse[:, h // 4 * 4])
    want = paged_ref.attend(x[:7].double().numpy()[:, None].repeat(8, 1), *cache.rows()[1], list(range(693, 700)), 0.09, 0, 0, ())
    check_prompt(out[:7].double().cpu().numpy(), lse[:7].double().cpu().numpy(), want, 128, 700, "fp16", float(np.abs(cache.rows()[1][1]).max()))


@pytest.mark.parametrize("new,old", [([5, 2], [3000, 1500]), ([80, 33], [40, 0])])
def test_in_a_graph_whose_lengths_change(new, old):
    """Captured once (with parts, where few queries stand behind many keys), replayed while lengths, starts and queries change, with eager calls in between."""
    cache = Cache([a + b + 40 for a, b in zip(new, old)], 2, 128, 16, seed=33)
    tokens = sum(new)
    q = torch.randn(tokens, 8, 128, generator=torch.Generator().manual_seed(2)).half().cuda()
    starts = torch.tensor([0, new[0], tokens], dtype=torch.int32, device="cuda")
    workspace = torch.empty(qkv.paged_prompt_workspace(cache.pages, 8, tokens), dtype=torch.uint8, device="cuda")
    other = torch.empty_like(workspace)
    out, lse = torch.empty_like(q), torch.empty(tokens, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        qkv.paged_prompt(cache.pages, q, starts, 0.09, out, lse, workspace=workspace, status=cache.status)
    for step in range(4):
        cache.glens.copy_(torch.tensor([a + b + 13 * step for a, b in zip(new, old)], dtype=torch.int32))
        starts[1] = new[0] - step // 2
        q.mul_(-1.0)
        out.fill_(3.0)
        lse.fill_(3.0)
        graph.replay()
        eager, eager_lse = torch.empty_like(q), torch.empty_like(lse)
        qkv.paged_prompt(cache.pages, q, starts, 0.09, eager, eager_lse, workspace=other)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse), step
    assert int(cache.status) == 0


@pytest.mark.parametrize("kind,dim,new,old,q_heads,heads,window", [("fp16", 128, [2100], [17000], 32, 8, 0), ("bf16", 256, [2100], [25000], 16, 8, 0),
                                                                   ("fp16", 64, [1500, 2, 0, 2700], [16500, 33000, 9, 100], 16, 8, 0),
                                                                   ("bf16", 128, [1100], [24000], 32, 8, 17000)])
def test_workgroups_that_would_leave_the_chip_idle(kind, dim, new, old, q_heads, heads, window):
    """Long keys in a few parts behind many queries, short sequences among them whole: some tokens of each row against the definition."""
    cache = Cache([a + b for a, b in zip(new, old)], heads, dim, 64, kind, seed=41)
    space = qkv.paged_prompt_workspace(cache.pages, q_heads, sum(new) + 3)
    assert space >= 2 * (sum(new) + 3) * q_heads * (dim + 2) * 4
    q, out, lse = run(cache, new, q_heads, dim, dim ** -0.5, window=window, sinks=5 if window else 0)
    at = 0
    for b, (K, V) in enumerate(cache.rows()):
        pick = sorted({0, 1, new[b] // 2, new[b] - 130, new[b] - 2, new[b] - 1} & set(range(new[b])))
        if pick:
            mine = [at + i for i in pick]
            want = paged_ref.attend(q[mine].double().numpy(), K, V, [old[b] + i for i in pick], dim ** -0.5, window, 5 if window else 0)
            check_prompt(out[mine], lse[mine], want, dim, cache.lens[b], kind, float(np.abs(V).max()))
        at += new[b]
    assert np.isfinite(out).all() and np.isfinite(lse).all() and int(cache.status) == 0


def test_two_streams_at_once():
    cache = Cache([4000, 900], 2, 128, 64, seed=35)
    q = torch.randn(12, 8, 128, generator=torch.Generator().manual_seed(2)).half().cuda()
    starts = torch.tensor([0, 7, 12], dtype=torch.int32, device="cuda")
    want, _ = qkv.paged_prompt(cache.pages, q, starts, 0.09, torch.empty_like(q))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(2)]
    spaces = [torch.empty(qkv.paged_prompt_workspace(cache.pages, 8, 12), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for _ in range(20):
        for stream, out, space in zip(streams, outs, spaces):
            with torch.cuda.stream(stream):
                qkv.paged_prompt(cache.pages, q, starts, 0.09, out, workspace=space)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_without_lse_the_same_bits():
    cache = Cache([200], 2, 128, 16, seed=9)
    _, a, _ = run(cache, [150], 8, 128, 0.1)
    _, b, none = run(cache, [150], 8, 128, 0.1, with_lse=False)
    assert none is None and np.array_equal(a, b)


def test_tensors_that_are_refused():
    cache = Cache([40], 2, 64, 16)
    q, starts = torch.zeros(6, 4, 64, dtype=torch.float16, device="cuda"), torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    for bad in (dict(q=q.float()), dict(q=q.transpose(0, 2)), dict(out=out.float()), dict(out=out[:3]), dict(starts=starts.long()), dict(starts=starts[:1]),
                dict(starts=starts.cpu()), dict(lse=out)):
        with pytest.raises(ValueError):
            a = {"q": q, "out": out, "starts": starts, **bad}
            qkv.paged_prompt(cache.pages, a.pop("q"), a.pop("starts"), 0.1, a.pop("out"), **a)
    with pytest.raises(qkv.QkvError):
        qkv.paged_prompt(cache.pages, q[:0], starts, 0.1, out[:0])
