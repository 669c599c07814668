"""Maps of a ragged batch against the definition, number by number."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from oracle import chosen_ref
from paged_case import Cache

pytestmark = pytest.mark.gpu


def run(cache, more, tokens, which=("row", "place", "slot")):
    maps = {name: torch.full((tokens,), 77, dtype=torch.int64 if name == "slot" else torch.int32, device="cuda") for name in which}
    starts = torch.full((len(cache.lens) + 1,), 77, dtype=torch.int32, device="cuda")
    cache.status.zero_()
    qkv.pages_slots(cache.pages, starts, more=None if more is None else torch.tensor(more, dtype=torch.int32).cuda(), tokens=tokens, status=cache.status, **maps)
    torch.cuda.synchronize()
    return starts.tolist(), {k: v.tolist() for k, v in maps.items()}, int(cache.status)


def check(cache, more, tokens, which=("row", "place", "slot")):
    starts, maps, status = run(cache, more, tokens, which)
    table = cache.gtable.cpu().tolist()
    want = chosen_ref.slots(more, cache.lens, table, cache.k.shape[1], cache.size, tokens)
    assert starts == want[0]
    for name, values in zip(("row", "place", "slot"), want[1:4]):
        if name in maps:
            assert maps[name] == values, name
    if "slot" in maps:
        assert status == want[4]


@pytest.mark.parametrize("size", [1, 16, 256])
@pytest.mark.parametrize("lens", [[5], [0], [300, 0, 17, 1, 0, 0], [33] * 70, [3] * 300 + [0] + [9] * 400])
def test_batches(lens, size):
    cache = Cache(lens, 1, 64, size, seed=size + len(lens))
    check(cache, None, len(lens))
    check(cache, None, len(lens) + 5)
    gen = np.random.default_rng(len(lens))
    more = [int(gen.integers(0, n + 1)) for n in lens]
    for spare in (0, 1, 300):
        check(cache, more, max(1, sum(more) + spare))
    check(cache, lens, max(1, sum(lens)), ("slot",))
    check(cache, more, max(1, sum(more)), ("place",))
    check(cache, more, max(1, sum(more)), ())


def test_many_rows():
    """More rows than a workgroup works out by itself."""
    gen = np.random.default_rng(1)
    lens = gen.integers(0, 4, 5000).tolist()
    cache = Cache(lens, 1, 64, 2, seed=1)
    more = [int(gen.integers(0, n + 1)) for n in lens]
    check(cache, more, sum(more) + 13)
    check(cache, None, 5000)
    check(cache, more, sum(more) // 2)
    more[4321] = -1
    check(cache, more, sum(more) + 20)


@pytest.mark.parametrize("at", [0, 1, 63, 64, 150, 255, 256, 299])
def test_room_that_does_not_do(at):
    """The first row that does not fit, and all behind it, have none."""
    lens = [7] * 300
    cache = Cache(lens, 1, 64, 4, seed=2)
    check(cache, [3] * 300, 3 * at + 1)
    check(cache, [3] * 300, 3 * at + 3)
    check(cache, [0] * at + [7] + [0] * (299 - at), 5)


def test_numbers_and_entries_that_may_not_be():
    cache = Cache([20, 20, 0, 20], 1, 64, 8, seed=3)
    check(cache, [3, -1, 1, 21], 30)
    check(cache, [3, 0x7FFFFFFF, -0x80000000, 2], 30)
    cache.gtable[0, 2] = -1
    cache.gtable[3, 1] = cache.k.shape[1]
    check(cache, [20, 5, 0, 20], 50)
    cache.glens[1] = 1 << 20                                        # longer than the row has entries for
    cache.lens[1] = cache.table.shape[1] * 8
    cache.gtable[1] = 0
    check(cache, [0, 4, 0, 0], 6)


def test_sums_beyond_32_bits():
    """Rows that share their pages can have more tokens than a batch of 2^31 has."""
    pages, rows, size = 2, 3000, 1 << 18
    k = torch.zeros(pages, 1, size, 64, dtype=torch.float16, device="cuda")
    table = torch.zeros(rows, 8, dtype=torch.int32, device="cuda")
    lens = torch.full((rows,), 8 * size, dtype=torch.int32, device="cuda")
    p, status = qkv.Pages.make([k], [k], table, lens), torch.zeros(1, dtype=torch.int32, device="cuda")
    starts = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    qkv.pages_slots(p, starts, more=lens, tokens=3 * 8 * size + 5, status=status)
    want = [min(i, 3) * 8 * size for i in range(rows + 1)]
    assert starts.tolist() == want and int(status) == qkv.STATUS_BAD_ROW


def test_maps_name_where_append_writes():
    cache = Cache([40, 3, 0, 17], 2, 64, 8, layout="tokens", seed=4)
    more = [40, 2, 0, 10]
    tokens = sum(more)
    starts, maps, status = run(cache, more, tokens + 4)
    new = torch.randn(tokens, 2, 64).to(torch.float16).cuda()
    qkv.pages_append(cache.pages, new, new, starts=torch.tensor(starts, dtype=torch.int32).cuda(), status=cache.status)
    for i in range(tokens):
        page, slot = divmod(maps["slot"][i], 8)
        assert torch.equal(cache.gk[0, page, :, slot], new[i])
    assert maps["slot"][tokens:] == [-1] * 4 and int(cache.status) == 0
