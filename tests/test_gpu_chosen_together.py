"""Chosen pages as a receiver uses them: a context goes into pages and gets its digests, agents go on from it, ask and answer over the pages that their queries choose,
joined with attention over a card; on streams of the caller's own."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import as_sets, as_words, draw_choices, expected, ragged
from oracle import chosen_ref, paged_ref
from paged_case import Cache, check_attend, check_prompt
from test_gpu_paged_together import D, H, HQ, L, SIZE, a_card, empty_pages, ints

pytestmark = pytest.mark.gpu

REP = HQ // H


def host(x):
    return x.double().cpu().numpy()


class Mirror:
    """What the rows hold, dense [L, H, T, D] in float64, and what follows from it."""

    def __init__(self, rows, exponents):
        self.k, self.v = [np.zeros((L, H, 0, D))] * rows, [np.zeros((L, H, 0, D))] * rows
        self.exponents = exponents

    def add(self, b, k, v):
        self.k[b], self.v[b] = (np.concatenate([x, y], axis=2) for x, y in ((self.k[b], k), (self.v[b], v)))

    def choice(self, b, layer, head, place, q, most, first, last):
        """As the definition has it: entries are the sequence's own page numbers, digests those of its full pages."""
        full = self.k[b].shape[2] // SIZE
        digests = np.zeros((full + 1, 2, D), dtype=np.int8)
        for j in range(full):
            digests[j] = chosen_ref.digest(self.k[b][layer, head:head + 1, j * SIZE:(j + 1) * SIZE], self.exponents[layer, head:head + 1])[0]
        return chosen_ref.choose(q, place, SIZE, list(range(full + 1)), full + 1, digests, self.exponents[layer, head], most, first, last)

    def attend(self, b, layer, place, q, sets):
        """One query [HQ, D] over the chosen pages, per kv head."""
        parts = [np.zeros((1, HQ, D)), np.full((1, HQ), -np.inf), np.zeros((1, HQ, D)), np.zeros((1, HQ)), np.zeros((1, HQ))]
        for h in range(H):
            tokens = [t for j in sorted(sets[h]) for t in range(j * SIZE, (j + 1) * SIZE) if t <= place]
            if tokens:
                some = slice(h * REP, (h + 1) * REP)
                got = paged_ref.attend(q[None, some], self.k[b][layer, h:h + 1][:, tokens], self.v[b][layer, h:h + 1][:, tokens], [len(tokens) - 1], 0.125)
                for part, x in zip(parts, got):
                    part[:, some] = x
        return parts


def test_agents_that_choose():
    tokens, gen = 203, torch.Generator(device="cuda").manual_seed(4)
    half = lambda *s: torch.randn(*s, generator=gen, device="cuda").half()  # noqa: E731
    desc, card, dense = a_card(tokens)
    pages, status = empty_pages(4, 90, 20)
    exponents = torch.frexp(torch.stack([x.float().abs().amax((0, 2)) for x in dense[0].unsqueeze(1)]) / 127)[1].to(torch.int8)
    layers = [torch.zeros(90, H, 2, D, dtype=torch.int8, device="cuda") for _ in range(L)]
    digests = qkv.Digests.make(pages, layers, exponents.contiguous())
    mirror = Mirror(4, exponents.cpu().numpy())
    starts, slot = ints(0, 0, 0, 0, 0), torch.zeros(tokens, dtype=torch.int64, device="cuda")

    # the card, rebuilt, goes into row 0, and its full pages get digests in all layers
    more = ints(tokens, 0, 0, 0)
    qkv.pages_reserve(pages, more, status)
    qkv.pages_slots(pages, starts, slot=slot, more=more, status=status)
    qkv.pages_append(pages, dense[0].transpose(1, 2), dense[1].transpose(1, 2), starts=starts, status=status)
    qkv.pages_digest(pages, digests, count=L, starts=starts, tokens=tokens, status=status)
    mirror.add(0, host(dense[0]), host(dense[1]))
    k_pool = pages.tensors[0][0]
    assert torch.equal(k_pool.transpose(1, 2).reshape(-1, H, D)[slot], dense[0][0].transpose(0, 1))
    # two agents go on from it; the pages they share have digests already
    qkv.pages_fork(pages, ints(0, 0), ints(2, 3), status)
    for b in (2, 3):
        mirror.k[b], mirror.v[b] = mirror.k[0], mirror.v[0]

    # each asks: a ragged batch in a padded one of fixed size, layer by layer
    more, room = ints(0, 0, 30, 6), 40
    qkv.pages_reserve(pages, more, status)
    row, place = (torch.zeros(room, dtype=torch.int32, device="cuda") for _ in range(2))
    qkv.pages_slots(pages, starts, row=row, place=place, more=more, status=status)
    assert row.tolist() == [2] * 30 + [3] * 6 + [-1] * 4 and place.tolist() == [*range(tokens, tokens + 30), *range(tokens, tokens + 6)] + [-1] * 4
    asked = [half(L, room, H, D) for _ in range(2)]
    for b, lo, n in ((2, 0, 30), (3, 30, 6)):
        mirror.add(b, *(host(x)[:, lo:lo + n].transpose(0, 2, 1, 3) for x in asked))
    for layer in range(L):
        q = half(room, HQ, D)
        qkv.pages_append(pages, asked[0][layer], asked[1][layer], layer=layer, starts=starts, status=status)
        qkv.pages_digest(pages, digests, layer=layer, starts=starts, tokens=room, status=status)
        choice = qkv.paged_choose(pages, digests, q, 5, first=1, last=2, layer=layer, starts=starts, status=status)
        out, lse = torch.full_like(q, 7.0), torch.full((room, HQ), 7.0, device="cuda")
        qkv.paged_prompt_chosen(pages, choice, q, starts, 0.125, out, lse, layer=layer, status=status)
        sets = as_sets(choice, 20)
        assert sets[36:] == [[set()] * H] * 4 and bool((out[36:] == 7.0).all()) and bool((lse[36:] == 7.0).all())
        for i in list(range(0, 36, 5)) + [29, 35]:
            b, p = int(row[i]), int(place[i])
            want = [mirror.choice(b, layer, h, p, q[i, h * REP:(h + 1) * REP].float().cpu().numpy(), 5, 1, 2) for h in range(H)]
            assert sets[i] == want, (layer, i)
            check_prompt(host(out)[i:i + 1], host(lse)[i:i + 1], mirror.attend(b, layer, p, host(q)[i], want), D, tokens + 30, "fp16", 100.0)

    # the shared context is dropped by row 0 and the pool moved together: digests are made again, of all that the rows hold
    qkv.pages_free(pages, ints(0), status=status)
    mirror.k[0], mirror.v[0] = (np.zeros((L, H, 0, D)) for _ in range(2))
    qkv.pages_compact(pages, status)
    held = sum(x.shape[2] for x in mirror.k)
    qkv.pages_slots(pages, starts, more=pages.tensors[3].clone(), tokens=held, status=status)
    for x in layers:
        x.fill_(77)
    qkv.pages_digest(pages, digests, count=L, starts=starts, tokens=held, status=status)

    # both answer, a token at a time, past several page borders
    for step in range(20):
        qkv.pages_reserve(pages, ints(0, 0, 1, 1), status)
        new = [half(L, 4, H, D) for _ in range(2)]
        for b in (2, 3):
            mirror.add(b, *(host(x)[:, b:b + 1].transpose(0, 2, 1, 3) for x in new))
        for layer in range(L):
            q = half(4, HQ, D)
            qkv.pages_append(pages, new[0][layer], new[1][layer], layer=layer, status=status)
            qkv.pages_digest(pages, digests, layer=layer, status=status)
            choice = qkv.paged_choose(pages, digests, q, 6, first=2, last=1, layer=layer, status=status)
            out, lse = torch.empty(4, HQ, D, device="cuda"), torch.empty(4, HQ, device="cuda")
            qkv.paged_attend_chosen(pages, choice, q, 0.125, out, lse, layer=layer, most=6, status=status)
            if step % 4 != 3:
                continue
            sets = as_sets(choice, 20)
            assert sets[0] == sets[1] == [set()] * H and bool((out[:2] == 0).all())
            for b in (2, 3):
                p = mirror.k[b].shape[2] - 1
                want = [mirror.choice(b, layer, h, p, q[b, h * REP:(h + 1) * REP].float().cpu().numpy(), 6, 2, 1) for h in range(H)]
                assert sets[b] == want, (step, layer, b)
                check_attend(host(out)[b:b + 1], host(lse)[b:b + 1], mirror.attend(b, layer, p, host(q)[b], want), D, p + 1)
    assert int(status) == 0


def test_joined_with_a_card():
    """A receiver that attends over the card itself and over the chosen ones of its own pages: together that is attention over both."""
    tokens, own = 96, 150
    desc, card, dense = a_card(tokens)
    cache = Cache([own], H, D, SIZE, layers=L, seed=5)
    q = torch.randn(L, HQ, D, generator=torch.Generator().manual_seed(6)).half()
    out, lse = torch.empty(L, HQ, D, device="cuda"), torch.empty(L, HQ, device="cuda")
    qkv.card_attend(card, desc, q.cuda(), 0.125, out, lse)
    choices = draw_choices(cache, [0], H, 0.5, 7)
    for layer in range(L):
        both, both_lse = torch.empty(1, HQ, D, device="cuda"), torch.empty(1, HQ, device="cuda")
        qkv.paged_attend_chosen(cache.pages, as_words(choices, cache.table.shape[1]), q[layer:layer + 1].cuda(), 0.125, both, both_lse, layer=layer,
                                prior=(out[layer:layer + 1], lse[layer:layer + 1]), status=cache.status)
        K, V = cache.rows(layer)[0]
        for h in range(H):
            seen = [t for j in sorted(choices[0][h]) for t in range(j * SIZE, (j + 1) * SIZE) if t < own]
            k, v = (np.concatenate([host(x)[layer, h:h + 1], y[h:h + 1][:, seen]], axis=1) for x, y in ((dense[0], K), (dense[1], V)))
            some = slice(h * REP, (h + 1) * REP)
            want = paged_ref.attend(q[layer:layer + 1, some].double().numpy(), k, v, [k.shape[1] - 1], 0.125)
            check_attend(host(both)[:, some], host(both_lse)[:, some], want, D, tokens + own)


def test_streams_of_the_callers_own():
    """Two chains of calls on two streams at once, each with a pool and scratch memory of its own that the binding finds: the results of one after the other."""
    cases, want = [], []
    for seed in (1, 2):
        cache = Cache([900, 0, 333], 2, 64, 16, layers=1, seed=seed)
        exponents = torch.randint(-4, -1, (1, 2, 64), dtype=torch.int8, generator=torch.Generator().manual_seed(seed)).cuda()
        layers = [torch.zeros(cache.k.shape[1], 2, 2, 64, dtype=torch.int8, device="cuda")]
        digests = qkv.Digests.make(cache.pages, layers, exponents)
        q = torch.randn(3, 6, 64, generator=torch.Generator().manual_seed(seed)).half().cuda()
        rows, _, starts = ragged(cache, [200, 0, 100])
        qp = torch.randn(300, 6, 64, generator=torch.Generator().manual_seed(seed + 9)).half().cuda()
        cases.append((cache, digests, q, starts, qp))

    def chain(case, stream):
        cache, digests, q, starts, qp = case
        out, lse, po = torch.zeros(3, 6, 64, device="cuda"), torch.zeros(3, 6, device="cuda"), torch.zeros_like(qp)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        every, held = torch.zeros(4, dtype=torch.int32, device="cuda"), cache.glens.clone()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        qkv.pages_slots(cache.pages, every, more=held, tokens=1300, stream=stream)
        qkv.pages_digest(cache.pages, digests, starts=every, tokens=1300, stream=stream)
        choice = qkv.paged_choose(cache.pages, digests, q, 9, stream=stream)
        qkv.paged_attend_chosen(cache.pages, choice, q, 0.125, out, lse, stream=stream)
        prompt = qkv.paged_choose(cache.pages, digests, qp, 9, starts=starts, stream=stream)
        qkv.paged_prompt_chosen(cache.pages, prompt, qp, starts, 0.125, po, stream=stream)
        return choice, out, lse, prompt, po

    for case in cases:
        want.append([x.clone() for x in chain(case, None)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = [chain(case, stream) for case, stream in zip(cases, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_pages_behind_4_gb():
    """Offsets beyond 32 bits: the last pages of a pool of more than 4 GB, of keys, of values and in the digests' own order."""
    size, heads, dim = 256, 8, 256
    per = heads * size * dim * 2
    pages = (1 << 32) // per + 9
    k = torch.zeros(pages, heads, size, dim, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    last = [pages - 1, pages - 3, pages - 2, 0]
    gen = torch.Generator().manual_seed(8)
    rows = [torch.randn(len(last), heads, size, dim, generator=gen).half() for _ in range(2)]
    for i, page in enumerate(last):
        k[page], v[page] = rows[0][i].cuda(), rows[1][i].cuda()
    length = 3 * size + 100
    table, lens = ints(*last).view(1, 4), ints(length)
    p, status = qkv.Pages.make([k], [v], table, lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    exponents = torch.full((1, heads, dim), -5, dtype=torch.int8)
    digest = torch.zeros(pages, heads, 2, dim, dtype=torch.int8, device="cuda")
    digests = qkv.Digests.make(p, [digest], exponents.cuda())
    qkv.pages_digest(p, digests, starts=ints(0, length), tokens=length, status=status)
    for i in range(3):
        assert np.array_equal(digest[last[i], 1:2].cpu().numpy(), chosen_ref.digest(rows[0][i, 1:2].double().numpy(), exponents[0, 1:2].numpy()))
    q = torch.randn(40, heads, dim, generator=gen).half()
    dense = [x.permute(1, 0, 2, 3).reshape(heads, -1, dim)[:, :length].double().numpy() for x in rows]
    choice = qkv.paged_choose(p, digests, q.cuda(), 3, first=1, last=1, starts=ints(0, 40), status=status)
    out, lse = torch.empty(40, heads, dim, dtype=torch.float16, device="cuda"), torch.empty(40, heads, device="cuda")
    qkv.paged_prompt_chosen(p, choice, q.cuda(), ints(0, 40), 0.0625, out, lse, status=status)
    one = torch.empty(1, heads, dim, device="cuda")
    one_lse = torch.empty(1, heads, device="cuda")
    qkv.paged_attend_chosen(p, choice[39:40].contiguous(), q[39:40].cuda(), 0.0625, one, one_lse, status=status)
    sets = as_sets(choice, 4)
    for i in (0, 17, 39):
        place = length - 40 + i
        for h in (0, 7):
            full = np.stack([chosen_ref.digest(rows[0][j, h:h + 1].double().numpy(), exponents[0, h:h + 1].numpy())[0] for j in range(3)])
            assert sets[i][h] == chosen_ref.choose(q[i, h:h + 1].float().numpy(), place, size, [0, 1, 2, 3], 4, np.concatenate([full, full[:1]]), exponents[0, h].numpy(), 3, 1, 1)
            tokens = [t for j in sorted(sets[i][h]) for t in range(j * size, (j + 1) * size) if t <= place]
            want = paged_ref.attend(q[i:i + 1, h:h + 1].double().numpy(), dense[0][h:h + 1][:, tokens], dense[1][h:h + 1][:, tokens], [len(tokens) - 1], 0.0625)
            check_prompt(host(out)[i:i + 1, h:h + 1], host(lse)[i:i + 1, h:h + 1], want, dim, length, "fp16", 6.0)
            if i == 39:
                check_attend(host(one)[:, h:h + 1], host(one_lse)[:, h:h + 1], want, dim, length)
    assert int(status) == 0


def test_places_next_to_the_largest():
    """Sequences of almost 2^31 tokens, whose pages are a few that are shared: sums of places stay within 32 bits."""
    size, row_pages, heads, dim = 16, (1 << 27) - 2, 1, 64
    gen = torch.Generator().manual_seed(9)
    k, v = (torch.randn(4, heads, size, dim, generator=gen).half() for _ in range(2))
    gk, gv = k.cuda(), v.cuda()
    table = (torch.arange(row_pages, device="cuda", dtype=torch.int32) % 4).view(1, -1)
    length = row_pages * size
    p, status = qkv.Pages.make([gk], [gv], table, ints(length)), torch.zeros(1, dtype=torch.int32, device="cuda")
    chosen = [{0, 5, row_pages - 2, row_pages - 1}, {row_pages - 3, row_pages - 2}, {1 << 26, row_pages - 1}]
    words = torch.zeros(3, heads, (row_pages + 31) // 32, dtype=torch.int32, device="cuda")
    for i, some in enumerate(chosen):
        for j in some:
            bit = 1 << (j % 32)
            words[i, 0, j // 32] |= bit - (1 << 32 if bit >> 31 else 0)
    q = torch.randn(3, 2, dim, generator=gen).half()
    out, lse = torch.empty(3, 2, dim, dtype=torch.float16, device="cuda"), torch.empty(3, 2, device="cuda")
    qkv.paged_prompt_chosen(p, words, q.cuda(), ints(0, 3), 0.125, out, lse, status=status)
    one, one_lse = torch.empty(1, 2, dim, device="cuda"), torch.empty(1, 2, device="cuda")
    qkv.paged_attend_chosen(p, words[2:3], q[2:3].cuda(), 0.125, one, one_lse, most=4, status=status)
    for i in range(3):
        place = length - 3 + i
        tokens = [t for j in sorted(chosen[i]) for t in range(j * size, (j + 1) * size) if t <= place]
        K, V = (torch.stack([x[(t // size) % 4, 0, t % size] for t in tokens]).double().numpy()[None] for x in (k, v))
        want = paged_ref.attend(q[i:i + 1].double().numpy(), K, V, [len(tokens) - 1], 0.125)
        check_prompt(host(out)[i:i + 1], host(lse)[i:i + 1], want, dim, 64, "fp16", 6.0)
        if i == 2:
            check_attend(host(one), host(one_lse), want, dim, 64)
    assert int(status) == 0


def test_odd_lists_next_to_the_largest():
    """What stands for a half of a tile that a list of odd length has not is behind every place there may be."""
    size, row_pages, heads, dim = 16, (1 << 27) - 2, 1, 64
    gen = torch.Generator().manual_seed(10)
    k, v = (torch.randn(4, heads, size, dim, generator=gen).half() for _ in range(2))
    table = (torch.arange(row_pages, device="cuda", dtype=torch.int32) % 4).view(1, -1)
    p = qkv.Pages.make([k.cuda()], [v.cuda()], table, ints(row_pages * size))
    near = set(range(row_pages - 10, row_pages - 2))                   # pages of 2^31 - 192 and on
    chosen = [{1 << 26} | near, {1 << 26}, near - {row_pages - 8}]
    words = torch.zeros(3, heads, (row_pages + 31) // 32, dtype=torch.int32, device="cuda")
    for i, some in enumerate(chosen):
        for j in some:
            words[i, 0, j // 32] |= (1 << (j % 32)) - (1 << 32 if j % 32 == 31 else 0)
    q = torch.randn(3, 2, dim, generator=gen).half()
    out, lse = torch.empty(3, 2, dim, dtype=torch.float16, device="cuda"), torch.empty(3, 2, device="cuda")
    qkv.paged_prompt_chosen(p, words, q.cuda(), ints(0, 3), 0.125, out, lse)
    for i in range(3):
        tokens = [t for j in sorted(chosen[i]) for t in range(j * size, (j + 1) * size)]
        K, V = (torch.stack([x[(t // size) % 4, 0, t % size] for t in tokens]).double().numpy()[None] for x in (k, v))
        want = paged_ref.attend(q[i:i + 1].double().numpy(), K, V, [len(tokens) - 1], 0.125)
        check_prompt(host(out)[i:i + 1], host(lse)[i:i + 1], want, dim, 64, "fp16", 6.0)


def test_tensors_that_are_refused():
    """On the host, before anything is enqueued."""
    cache = Cache([40, 3], 2, 64, 16)
    pages, count = cache.pages, cache.k.shape[1]
    bounds, exponents = torch.zeros(count, 2, 2, 64, dtype=torch.int8, device="cuda"), torch.zeros(1, 2, 64, dtype=torch.int8, device="cuda")
    for layers, steps in (([], exponents), ([bounds, bounds], exponents), ([bounds[1:]], exponents), ([bounds.short()], exponents), ([bounds.cpu()], exponents),
                          ([bounds.transpose(2, 3).contiguous().transpose(2, 3)], exponents), ([bounds], exponents[0]), ([bounds], exponents.int()), ([bounds], exponents.cpu())):
        with pytest.raises(ValueError):
            qkv.Digests.make(pages, layers, steps)
    digests = qkv.Digests.make(pages, [bounds], exponents)
    other = Cache([40, 3], 2, 64, 16, spare=9)
    q, words = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda"), torch.zeros(2, 2, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        qkv.pages_digest(other.pages, digests)
    with pytest.raises(ValueError):
        qkv.paged_choose(other.pages, digests, q, 3)
    for bad in (dict(starts=ints(0, 1, 2)), dict(tokens=3), dict(starts=ints(0, 1), tokens=2), dict(starts=ints(0, 1, 2).long(), tokens=2),
                dict(status=torch.zeros(1, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            qkv.pages_digest(pages, digests, **bad)
    for bad in (dict(q=q.float()), dict(q=q[..., :32]), dict(q=q[0]), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(choice=words[:1]), dict(choice=words.long()),
                dict(starts=ints(0, 2)), dict(workspace=torch.zeros(8, device="cuda"))):
        with pytest.raises(ValueError):
            qkv.paged_choose(**{"pages": pages, "digests": digests, "q": q, "most": 3, **bad})
    for bad in (dict(most=1), dict(last=0), dict(layer=1), dict(q=q[:1]), dict(q=q[:, :3])):
        with pytest.raises(qkv.QkvError):
            qkv.paged_choose(**{"pages": pages, "digests": digests, "q": q, "most": 3, **bad})
    out = torch.zeros(2, 4, 64, device="cuda")
    for bad in (dict(choice=words.long()), dict(choice=words[:, :1]), dict(choice=words.expand(2, 2, 2)), dict(q=q.float()), dict(out=out.half()),
                dict(prior=(out, out)), dict(lse=out)):
        with pytest.raises(ValueError):
            qkv.paged_attend_chosen(**{"pages": pages, "choice": words, "q": q, "softmax_scale": 0.1, "out": out, **bad})
        if "prior" not in bad:
            with pytest.raises(ValueError):
                more = {**bad, "out": out} if "out" in bad else bad
                qkv.paged_prompt_chosen(**{"pages": pages, "choice": words, "q": q, "softmax_scale": 0.1, "out": out.half(), "starts": ints(0, 1, 2), **more})
    with pytest.raises(ValueError):
        qkv.paged_prompt_chosen(pages, words, q, ints(0, 2), 0.1, out.half())
    starts, row = ints(0, 0, 0), ints(0, 0)
    for bad in (dict(), dict(row=row, tokens=3), dict(row=row.long()), dict(row=row, place=ints(0)), dict(slot=row), dict(row=row, more=ints(1))):
        with pytest.raises(ValueError):
            qkv.pages_slots(pages, starts, **bad)
