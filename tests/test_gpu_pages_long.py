"""Rows of new tokens of the longest batches there may be: 2^27 - 1 tokens, more than one launch takes."""
import pytest
import torch

import paper_2605_03884_amd as qkv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [0, (1 << 25) - 3, (1 << 26) - 3, (1 << 27) - 10])
def test_append_of_as_many_tokens_as_there_may_be(first):
    """Seven tokens of the batch, from `first` on, belong to rows; what stands in front of them and behind them belongs to none.  The batch's rows of
    values overlap (strides of 8 elements), so that it is 2 GB."""
    tokens, dim = (1 << 27) - 1, 64
    base = (torch.arange((tokens + 8) * 8 + 8, dtype=torch.int32, device="cuda") * -1640531527 >> 16).to(torch.int16)
    new = [base[8 * i:].as_strided((tokens, 1, dim), (8, 64, 1)).view(torch.float16) for i in range(2)]
    pools = [torch.zeros(5, 1, 4, dim, dtype=torch.float16, device="cuda") for _ in range(2)]
    table = torch.tensor([[3, 1], [4, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    starts = torch.tensor([first, first + 2, first + 7], dtype=torch.int32, device="cuda")
    qkv.pages_append(qkv.Pages.make([pools[0]], [pools[1]], table, lens), *new, starts=starts, status=status)
    torch.cuda.synchronize()
    places = [(3, 3), (1, 0)] + [(4, 1), (4, 2), (4, 3), (0, 0), (0, 1)]
    for pool, x in zip(pools, new):
        want = torch.zeros(5, 1, 4, dim, dtype=torch.int16)
        for i, (page, place) in enumerate(places):
            want[page, 0, place] = x[first + i, 0].view(torch.int16).cpu()
        assert torch.equal(pool.view(torch.int16).cpu(), want)
    assert int(status) == 0
