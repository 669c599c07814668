"""The cache in pages as a receiver uses it: a card goes into pages, agents fork the sequence, ask and answer, pages are given back and moved;
and a receiver that attends over the card itself and over its own tokens in pages."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
import qkv_synth
from oracle import paged_ref
from paged_case import check_attend, check_prompt

pytestmark = pytest.mark.gpu

L, H, HQ, D, SIZE = 2, 2, 8, 64, 16


def a_card(tokens):
    k, v = (x.cuda() for x in qkv_synth.make_kv(L, H, tokens, D, 11, "llama"))
    desc = qkv.Desc.make(L, H, tokens, D, 32)
    bits, counts = qkv.assign_bits(qkv_synth.make_scores(tokens, 12).cuda(), 5.0)
    card = torch.zeros(qkv.card_bytes(desc, counts), dtype=torch.uint8, device="cuda")
    qkv.quantize_pack(desc, k, v, bits, counts, card)
    dense = [torch.empty_like(k), torch.empty_like(v)]
    qkv.unpack_dequant(card, desc, *dense)
    return desc, card, dense


def empty_pages(rows, pages, row_pages):
    k, v = (torch.full((L, pages, H, SIZE, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.full((rows, row_pages), -1, dtype=torch.int32, device="cuda")
    lens, refs = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(pages, dtype=torch.int32, device="cuda")
    return qkv.Pages.make(list(k), list(v), table, lens, refs), torch.zeros(1, dtype=torch.int32, device="cuda")


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_card_shared_by_agents():
    tokens, gen = 137, torch.Generator(device="cuda").manual_seed(3)
    half = lambda *s: torch.randn(*s, generator=gen, device="cuda").half()  # noqa: E731
    desc, card, dense = a_card(tokens)
    pages, status = empty_pages(4, 64, 20)
    host = lambda x: x.double().cpu().numpy()  # noqa: E731
    history = [[np.zeros((L, H, 0, D))] * 2 for _ in range(4)]
    add = lambda b, k, v: history.__setitem__(b, [np.concatenate([h, x], axis=2) for h, x in zip(history[b], (k, v))])  # noqa: E731
    # the card, rebuilt, goes into row 0
    qkv.pages_reserve(pages, ints(tokens, 0, 0, 0), status)
    qkv.pages_append(pages, dense[0].transpose(1, 2), dense[1].transpose(1, 2), starts=ints(0, tokens, tokens, tokens, tokens), status=status)
    add(0, host(dense[0]), host(dense[1]))
    # two agents go on from it
    qkv.pages_fork(pages, ints(0, 0), ints(2, 3), status)
    history[2], history[3] = list(history[0]), list(history[0])
    # each asks: a ragged batch of new tokens, layer by layer
    new = [0, 0, 21, 6]
    starts = ints(0, 0, 0, 21, 27)
    qkv.pages_reserve(pages, ints(*new), status)
    for layer in range(L):
        k, v, q = half(27, H, D), half(27, H, D), half(27, HQ, D)
        qkv.pages_append(pages, k, v, layer=layer, starts=starts, status=status)
        if layer == 0:
            asked = [[k], [v]]
        else:
            asked = [[asked[0][0], k], [asked[1][0], v]]
        out, lse = torch.empty_like(q), torch.empty(27, HQ, device="cuda")
        qkv.paged_prompt(pages, q, starts, 0.125, out, lse, layer=layer, window=100, sinks=3, status=status)
        for b, lo, n in ((2, 0, 21), (3, 21, 6)):
            K, V = (np.concatenate([h[layer], host(x)[lo:lo + n].transpose(1, 0, 2)], axis=1) for h, x in zip(history[b], (k, v)))
            want = paged_ref.attend(host(q)[lo:lo + n], K, V, list(range(tokens, tokens + n)), 0.125, 100, 3)
            check_prompt(host(out)[lo:lo + n], host(lse)[lo:lo + n], want, D, tokens + n, "fp16", float(np.abs(V).max()))
    k, v = (torch.stack(x).permute(0, 2, 1, 3) for x in asked)
    add(2, host(k)[:, :, :21], host(v)[:, :, :21])
    add(3, host(k)[:, :, 21:], host(v)[:, :, 21:])
    # the shared context is dropped by row 0, the pool is moved together, and both answer; row 1 stays empty, row 0 holds nothing
    qkv.pages_free(pages, ints(0), status=status)
    history[0] = [np.zeros((L, H, 0, D))] * 2
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    qkv.pages_compact(pages, status, live=live)
    assert int(live) == 8 + 2 + 1
    for step in range(20):
        qkv.pages_reserve(pages, ints(0, 0, 1, 1), status)
        k, v, q = half(L, 4, H, D), half(L, 4, H, D), half(L, 4, HQ, D)
        qkv.pages_append(pages, k, v, status=status)
        for b in (2, 3):
            add(b, host(k)[:, b][:, :, None], host(v)[:, b][:, :, None])
        out, lse = torch.empty(4, HQ, D, device="cuda"), torch.empty(4, HQ, device="cuda")
        for layer in range(L):
            qkv.paged_attend(pages, q[layer], 0.125, out, lse, layer=layer, status=status)
            if step % 7 == 0:
                parts = [paged_ref.attend(host(q)[layer, b:b + 1], history[b][0][layer], history[b][1][layer], [history[b][0].shape[2] - 1], 0.125) for b in range(4)]
                check_attend(host(out), host(lse), [np.concatenate(x) for x in zip(*parts)], D, 200)
    assert int(status) == 0
    qkv.pages_free(pages, status=status)
    assert not pages.tensors[4].any() and int(status) == 0


def test_attention_over_a_card_and_over_pages():
    """The card is read as it is; the receiver's own tokens, in pages, see it and each other."""
    tokens, own = 300, 45
    desc, card, dense = a_card(tokens)
    pages, status = empty_pages(1, 8, 4)
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn(L, own, H, D, generator=gen, device="cuda").half() for _ in range(2))
    qkv.pages_reserve(pages, ints(own), status)
    qkv.pages_append(pages, k, v, starts=ints(0, own), status=status)
    q = torch.randn(L, HQ, D, generator=gen, device="cuda").half()
    out, lse = torch.empty(L, HQ, D, device="cuda"), torch.empty(L, HQ, device="cuda")
    qkv.card_attend(card, desc, q, 0.125, out, lse)
    host = lambda x: x.double().cpu().numpy()  # noqa: E731
    for layer in range(L):
        both, both_lse = torch.empty(1, HQ, D, device="cuda"), torch.empty(1, HQ, device="cuda")
        qkv.paged_attend(pages, q[layer:layer + 1], 0.125, both, both_lse, layer=layer, prior=(out[layer:layer + 1], lse[layer:layer + 1]), status=status)
        K, V = (np.concatenate([host(d)[layer], host(x)[layer].transpose(1, 0, 2)], axis=1) for d, x in zip(dense, (k, v)))
        check_attend(host(both), host(both_lse), paged_ref.attend(host(q)[layer:layer + 1], K, V, [tokens + own - 1], 0.125), D, tokens + own)
    assert int(status) == 0


def test_steps_in_a_graph():
    """A captured step - room, rows, attention - replayed while the sequences grow, between eager work of another pool."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows, steps = 3, 40
    made = [empty_pages(rows, 40, 12) for _ in range(2)]
    spaces = [torch.empty(qkv.paged_attend_workspace(p, HQ), dtype=torch.uint8, device="cuda") for p, _ in made]
    assert spaces[0].numel() > 0
    k, v, q = (torch.empty(L, rows, h, D, dtype=torch.float16, device="cuda") for h in (H, H, HQ))
    outs = [torch.empty(L, rows, HQ, D, device="cuda") for _ in range(2)]
    lses = [torch.empty(L, rows, HQ, device="cuda") for _ in range(2)]
    more = ints(1, 0, 4)
    starts = ints(0, 1, 1, 3)                                     # of the four new tokens of row 2 two are written: the last ones

    def step(i):
        pages, status = made[i]
        qkv.pages_reserve(pages, more, status)
        qkv.pages_append(pages, k, v, starts=starts, status=status)
        for layer in range(L):
            qkv.paged_attend(pages, q[layer], 0.125, outs[i][layer], lses[i][layer], layer=layer, window=50, sinks=1, workspace=spaces[i], status=status)

    for pages, status in made:                                    # what nobody writes is a number
        for t in (*pages.tensors[0], *pages.tensors[1]):
            t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k.normal_(generator=gen), v.normal_(generator=gen), q.normal_(generator=gen)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(0)
    for _ in range(steps):
        for t in (k, v, q):
            t.normal_(generator=gen)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert int(made[0][1]) == int(made[1][1]) == 0
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1])
        assert torch.equal(made[0][0].tensors[2], made[1][0].tensors[2]) and torch.equal(made[0][0].tensors[3], made[1][0].tensors[3])
    assert made[0][0].tensors[3].tolist() == [steps, 0, 4 * steps]
    assert torch.isinf(lses[0][:, 1]).all() and not outs[0][:, 1].any()
