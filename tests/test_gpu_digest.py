"""Digests of pages - bounds of their keys in 8 bits - against the definition, code by code."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from oracle import chosen_ref
from paged_case import TYPES, Cache

pytestmark = pytest.mark.gpu


def digests_of(cache, layers, exponents=None, seed=1):
    pages, heads, dim = cache.k.shape[1], cache.k.shape[2], cache.k.shape[4]
    gen = torch.Generator().manual_seed(seed)
    first = torch.randint(-128, 128, (layers, pages, heads, 2, dim), generator=gen, dtype=torch.int8)
    if exponents is None:
        exponents = torch.randint(-6, 1, (layers, heads, dim), generator=gen, dtype=torch.int8)
    held = first.cuda()
    return first, held, exponents, qkv.Digests.make(cache.pages, list(held), exponents.cuda())


def check(cache, first, held, exponents, filled, layers):
    """`filled`: (row, page of the row) that are written, in `layers`; every other byte stays."""
    want = first.clone()
    for layer in layers:
        for b, j in filled:
            page = int(cache.table[b, j])
            want[layer, page] = torch.from_numpy(chosen_ref.digest(cache.k[layer, page].double().numpy(), exponents[layer].numpy()))
    assert torch.equal(held.cpu(), want)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [1, 2, 16, 64, 128])
def test_one_token_of_every_row(kind, dim, size):
    """Only rows whose new token has filled a page."""
    lens = [0, 1, size, 2 * size, 2 * size + 1, 3 * size - 1 if size > 1 else 5, 4 * size]
    cache = Cache(lens, 3, dim, size, kind, layers=2, layout="tokens" if size == 16 else "heads", seed=dim + size)
    first, held, exponents, digests = digests_of(cache, 2)
    qkv.pages_digest(cache.pages, digests, layer=1, status=cache.status)
    torch.cuda.synchronize()
    check(cache, first, held, exponents, [(b, n // size - 1) for b, n in enumerate(lens) if n and n % size == 0], [1])
    assert int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 8, 32, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens", "both"])
def test_ragged_batches(size, layout):
    lens = [700, 0, 3, 64, 65, 31, 300, 257]
    new = [700, 0, 1, 64, 2, 31, 0, 200]
    cache = Cache(lens, 2, 64, size, layers=3, layout=layout, seed=size)
    first, held, exponents, digests = digests_of(cache, 3)
    starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    qkv.pages_digest(cache.pages, digests, count=2, starts=starts, tokens=sum(new) + 9, status=cache.status)
    torch.cuda.synchronize()
    filled = [(b, j) for b, (n, c) in enumerate(zip(lens, new)) for j in range((n - c) // size, n // size)]
    assert filled
    check(cache, first, held, exponents, filled, [0, 1])
    assert int(cache.status) == 0


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [4, 128])
def test_every_value_and_every_step(kind, size):
    """Infinities, no numbers, the smallest values of the type and steps of every size; codes at the ends of their range."""
    cache = Cache([3 * size], 2, 64, size, kind, seed=3)
    gen = torch.Generator().manual_seed(9)
    raw = torch.randint(-32768, 32768, cache.k.shape, generator=gen, dtype=torch.int16).view(TYPES[kind])
    raw[..., ::5] = (torch.randn(raw[..., ::5].shape, generator=gen) * 127).to(TYPES[kind])
    for i, x in enumerate((float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 2.0 ** -24, -2.0 ** -24)):
        raw[:, :, :, :, 10 + i] = torch.tensor(x).to(TYPES[kind])
    raw[0, :, 0, :, 20] = float("nan")
    raw[0, :, 0, 0, 20] = 1.0
    cache.k = raw
    cache.gpu()
    exponents = torch.arange(-64, 64, dtype=torch.int8).repeat(1)[: 2 * 64].view(1, 2, 64).contiguous()
    exponents[0, 1] *= 2
    exponents[0, 0, :3] = torch.tensor([-128, 127, 0], dtype=torch.int8)
    first, held, exponents, digests = digests_of(cache, 1, exponents)
    qkv.pages_digest(cache.pages, digests, starts=torch.tensor([0, 3 * size], dtype=torch.int32).cuda(), tokens=3 * size, status=cache.status)
    torch.cuda.synchronize()
    check(cache, first, held, exponents, [(0, 0), (0, 1), (0, 2)], [0])


def test_bounds_hold():
    """Where a step leaves room for all keys, codes times the step are bounds, and no further off than a step."""
    cache = Cache([640], 4, 128, 16, seed=5)
    step = torch.frexp(cache.k[:, :, :, :, :].nan_to_num(0, 0, 0).abs().float().amax((1, 3)) / 127)[1].to(torch.int8)
    first, held, exponents, digests = digests_of(cache, 1, step)
    qkv.pages_digest(cache.pages, digests, starts=torch.tensor([0, 640], dtype=torch.int32).cuda(), tokens=640)
    got = held.cpu().double() * torch.pow(2.0, step.double())[:, None, :, None, :]
    for j in range(40):
        page = int(cache.table[0, j])
        k = cache.k[0, page].double()
        up, down = got[0, page, :, 0] - k.amax(1), k.amin(1) - got[0, page, :, 1]
        assert (up >= 0).all() and (down >= 0).all() and (up < torch.pow(2.0, step[0].double())).all() and (down < torch.pow(2.0, step[0].double())).all()


def test_rows_and_entries_that_may_not_be():
    cache = Cache([64, 64, 64, 64], 2, 64, 16, seed=6)
    first, held, exponents, digests = digests_of(cache, 1)
    cache.gtable[0, 1] = -1
    cache.gtable[1, 2] = cache.k.shape[1]
    starts = torch.tensor([0, 64, 128, 192, 256], dtype=torch.int32).cuda()
    qkv.pages_digest(cache.pages, digests, starts=starts, tokens=256, status=cache.status)
    torch.cuda.synchronize()
    check(cache, first, held, exponents, [(b, j) for b in range(4) for j in range(4) if (b, j) not in ((0, 1), (1, 2))], [0])
    assert int(cache.status) == qkv.STATUS_BAD_PAGE

    first, held, exponents, digests = digests_of(cache, 1, seed=7)
    cache.status.zero_()
    starts = torch.tensor([0, 64, 140, 204, 300], dtype=torch.int32).cuda()      # row 1 has more than its length, row 3 ends behind the batch
    qkv.pages_digest(cache.pages, digests, starts=starts, tokens=256, status=cache.status)
    torch.cuda.synchronize()
    check(cache, first, held, exponents, [(0, 0), (0, 2), (0, 3)] + [(2, j) for j in range(4)], [0])
    assert int(cache.status) == qkv.STATUS_BAD_ROW | qkv.STATUS_BAD_PAGE


def test_forked_pages_need_nothing_and_moved_ones_are_made_again():
    cache = Cache([40, 0, 23], 2, 64, 16, layers=2, spare=6, seed=8)
    first, held, exponents, digests = digests_of(cache, 2)
    every = torch.tensor([0, 40, 40, 63], dtype=torch.int32).cuda()
    qkv.pages_digest(cache.pages, digests, count=2, starts=every, tokens=63)
    before = held.clone()
    qkv.pages_fork(cache.pages, torch.tensor([0], dtype=torch.int32).cuda(), torch.tensor([1], dtype=torch.int32).cuda(), cache.status)
    assert torch.equal(cache.gtable[1, :2], cache.gtable[0, :2]) and torch.equal(before, held)
    qkv.pages_free(cache.pages, torch.tensor([2], dtype=torch.int32).cuda(), status=cache.status)
    qkv.pages_compact(cache.pages, cache.status)
    qkv.pages_digest(cache.pages, digests, count=2, starts=torch.tensor([0, 40, 80, 80], dtype=torch.int32).cuda(), tokens=80, status=cache.status)
    torch.cuda.synchronize()
    table = cache.gtable.cpu()
    for layer in range(2):
        for j in range(2):
            page = int(table[0, j])
            want = chosen_ref.digest(cache.gk[layer, page].double().cpu().numpy(), exponents[layer].numpy())
            assert np.array_equal(held[layer, page].cpu().numpy(), want)
    assert int(cache.status) == 0
