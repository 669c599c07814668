"""Attention of many new tokens over chosen pages where there are more query tiles than CUs: one workgroup to a tile, or two to four that share a long sequence's keys."""
import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from chosen_case import draw_choices
from paged_case import Cache
from test_gpu_prompt_chosen import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("fp16", 64), ("bf16", 128), ("fp16", 128), ("bf16", 256)])
@pytest.mark.parametrize("size", [4, 16, 64])
def test_long_keys_in_a_few_parts(kind, dim, size):
    """300 tiles of two tokens each behind 12409: with 64, 128 and 256 dimensions in 2, 3 and 3 parts."""
    length, tokens = 13000, 591
    cache = Cache([length, 30], 1, dim, size, kind, seed=dim + size)
    width = cache.table.shape[1]
    gen = np.random.default_rng(size)
    new = [tokens, 9]
    choices = [[set(gen.integers(0, width, 20).tolist()) | {0, (length - tokens + i) // size}] for i in range(tokens)] + [[{0, i}] for i in range(9)]
    choices[1], choices[2], choices[3] = [set()], [{5}], [set(range(0, width, 3))]
    with pytest.raises(qkv.QkvError):
        run(cache, new, choices, 64, dim, 0.1, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    need = qkv.paged_prompt_chosen_workspace(cache.pages, 64, tokens + 9 + 2)
    workspace = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    check(cache, new, choices, 64, dim, 0.1, spare=2, some=[0, 1, 2, 3, 4, 350, 351, 590, 591, 599], workspace=workspace[:need])
    assert bool((workspace[need:] == 0xFF).all()) and int(cache.status) == 0


@pytest.mark.parametrize("size", [1, 16, 64])
@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("fp16", 128), ("bf16", 128), ("fp16", 256)])
def test_more_tiles_than_cus(size, kind, dim):
    """600 tiles and short sequences, which stay whole."""
    cache = Cache([500, 0, 640, 128], 2, dim, size, kind, seed=size)
    new = [450, 0, 600, 100]
    choices = draw_choices(cache, range(1150), 2, 0.1, size)
    _, _ = check(cache, new, choices, 128, dim, 0.09, some=[0, 1, 2, 63, 64, 449, 450, 451, 1049, 1050, 1149], workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert int(cache.status) == 0
