"""Scratch memory that the binding allocates itself belongs to the stream the call runs on: given back when the call returns, it may be handed out
again at once, and only work that is queued behind the call's may have it."""
import contextlib
import types

import numpy as np
import pytest
import torch

import paper_2605_03884_amd as qkv
from paper_2605_03884_amd import binding

SIDE = types.SimpleNamespace(cuda_stream=0x51DE)


class Library:
    """Answers every call with success, workspaces with 4096 bytes, and notes the stream each one was given."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                args[-1]._obj.value = 4096
            else:
                self.calls.append((name, args[-1]))
            return 0
        return call


@pytest.fixture
def host(monkeypatch):
    """The binding with a library that does nothing, on tensors in host memory; `made`: the stream that was current at each allocation."""
    library, made, active = Library(), [], [None]

    @contextlib.contextmanager
    def stream(s):
        before, active[0] = active[0], s
        yield
        active[0] = before

    empty = torch.empty

    def noted(*args, **more):
        made.append(active[0])
        return empty(*args, **more)

    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(binding, "_dev_ptr", lambda t, dtype=None, name="": t.data_ptr())
    monkeypatch.setattr(binding, "_current_device", lambda: None)
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: 0xC0)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", noted)
    return types.SimpleNamespace(library=library, made=made)


def calls():
    half, full = torch.zeros(2, 4, 64, dtype=torch.float16), torch.zeros(2, 4, 64)
    word, card = torch.zeros(1, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
    p = types.SimpleNamespace(device=half.device, dtype=torch.float16, rows=1, head_dim=64)
    desc = binding.Desc()
    starts = torch.zeros(2, dtype=torch.int32)
    return {
        "qkv_paged_attend": lambda **s: qkv.paged_attend(p, half[:1], 0.1, full[:1], **s),
        "qkv_paged_prompt": lambda **s: qkv.paged_prompt(p, half, starts, 0.1, half.clone(), **s),
        "qkv_pages_compact": lambda **s: qkv.pages_compact(p, word, **s),
        "qkv_card_attend": lambda **s: qkv.card_attend(card, desc, half, 0.1, full, **s),
        "qkv_card_attend_kc": lambda **s: qkv.card_attend_kc(card, desc, half, 0.1, full, **s),
    }


@pytest.mark.parametrize("name", ["qkv_paged_attend", "qkv_paged_prompt", "qkv_pages_compact", "qkv_card_attend", "qkv_card_attend_kc"])
def test_scratch_is_of_the_stream_that_was_passed(host, name):
    calls()[name](stream=SIDE)
    assert host.made == [SIDE] and host.library.calls == [(name, SIDE.cuda_stream)]


@pytest.mark.parametrize("name", ["qkv_paged_attend", "qkv_paged_prompt", "qkv_pages_compact", "qkv_card_attend", "qkv_card_attend_kc"])
def test_without_a_stream_it_is_of_the_current_one(host, name):
    calls()[name]()
    assert host.made == [None] and host.library.calls == [(name, 0xC0)]


def cut_cache():
    """Two rows long enough to be cut for single tokens and for prompts."""
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn(80, 2, 64, 128, generator=gen).half().cuda() for _ in range(2))
    table = torch.randperm(80, generator=gen).to(torch.int32).view(2, 40).cuda()
    lens = torch.tensor([2500, 1300], dtype=torch.int32, device="cuda")
    return qkv.Pages.make([k], [v], table, lens), torch.randn(2, 8, 128, generator=gen).half().cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("prompt", [False, True])
def test_memory_that_the_current_stream_gets_meanwhile_is_other_memory(prompt):
    """A call on a side stream that waits, scratch of its own, while the current stream allocates as much and writes over it."""
    pages, q = cut_cache()
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")

    def call(**more):
        if prompt:
            return qkv.paged_prompt(pages, q, starts, 0.09, torch.empty_like(q), **more)[0]
        return qkv.paged_attend(pages, q, 0.09, torch.empty(2, 8, 128, device="cuda"), **more)[0]

    size = qkv.paged_prompt_workspace(pages, 8, 2) if prompt else qkv.paged_attend_workspace(pages, 8)
    assert size > 0
    want = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = call(stream=side)
    for _ in range(4):
        torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    assert np.array_equal(got.float().cpu().numpy(), want.float().cpu().numpy())


@pytest.mark.gpu
def test_compaction_on_a_side_stream():
    k, v = (torch.randn(64, 1, 16, 64, device="cuda").half() for _ in range(2))
    table = torch.arange(63, 31, -1, dtype=torch.int32, device="cuda").view(1, 32).contiguous()
    lens, refs = torch.tensor([500], dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    refs[32:] = 1
    before = [x[table[0].long()].clone() for x in (k, v)]
    pages, status = qkv.Pages.make([k], [v], table, lens, refs), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    live, side = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    qkv.pages_compact(pages, status, live=live, stream=side)
    for _ in range(4):
        torch.empty(qkv.pages_compact_workspace(pages), dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    assert int(status) == 0 and int(live) == 32
    assert sorted(table[0].tolist()) == list(range(32)) and refs.tolist() == [1] * 32 + [0] * 32
    assert torch.equal(k[table[0].long()], before[0]) and torch.equal(v[table[0].long()], before[1])
