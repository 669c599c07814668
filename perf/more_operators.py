"""Attention over those pages of a receiver's cache that a cheap score chooses for each query, and the maps of a ragged batch: what each call
computes, in elementary torch operations, and the calls of paper_2605_03884_amd that do the same (where `own` is true).

The cache is that of operators.py: a pool of pages of page_tokens tokens, a table of page numbers and a length for every sequence.

  digest    of every page that the new tokens have filled: for each kv head and channel the smallest and the largest key, held in 8 bits (codes of a
            step 2^e that the channel has for all pages, rounded away from each other, so they bound the keys)
  choose    pages for every query token and kv head: the first and the last ones up to the query's own place, and of the others those with the highest score.
            A page's score bounds <q, k> over its keys, summed over the query heads that share the kv head; queries too are held in 8 bits, so scores are
            whole numbers.  Equal scores: the lowest page first.  A choice is a bit for each page of the sequence, 32 to a word
  attend    one new token of every sequence over the pages chosen for it: out and lse in 32 bits; optionally joined with attention over other tokens
  prompt    many new tokens of every sequence, each over the pages chosen for it, up to its own place; out in the cache's type, lse in 32 bits
  slots     where the tokens of a ragged batch go, from how many each sequence has: starts, and for every token its sequence, its place in it and
            the place in the pool; -1 behind the last token

A case is a dict of plain values.  Lengths are a fixed function of the case; contents and the order of the pages come from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _digest(layers, rows, longest_new, longest_old, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, **more):
    return dict(op="digest", layers=layers, rows=rows, longest_new=longest_new, longest_old=longest_old, kv_heads=kv_heads, head_dim=head_dim,
                kind=kind, page_tokens=page_tokens, **more)


def _chosen(op, rows, longest_new, longest_old, most, q_heads=32, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, first=1, last=2, prior=False, **more):
    """longest_new 0: one new token of every sequence, whose lengths go up to longest_old."""
    return dict(op=op, rows=rows, longest_new=longest_new, longest_old=longest_old, most=most, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                kind=kind, page_tokens=page_tokens, first=first, last=last, prior=prior, **more)


def _slots(rows, longest_new, longest_old, page_tokens=16, padded=0, **more):
    return dict(op="slots", rows=rows, longest_new=longest_new, longest_old=longest_old, page_tokens=page_tokens, padded=padded, kv_heads=1, head_dim=64,
                kind="fp16", **more)


def listed():
    return [
        # a decode step of a batch, in one layer: some sequences have filled a page with their new token, most have not
        _digest(1, 64, 0, 8192, kind="bf16", name="digest_step"),
        # a card that was rebuilt and written into pages: all of them, in all layers
        _digest(32, 1, 4100, 64, page_tokens=32, name="digest_layers_4100"),
        # a serving batch of a Llama-3.1-8B shaped layer, lengths all over, one place in the batch empty: 64 pages of 16 tokens each
        _chosen("choose", 48, 0, 8192, 64, name="choose_batch_8k"),
        # one sequence with a full 128K context, 256 pages of 16
        _chosen("choose", 1, 0, 131071, 256, kind="bf16", first=4, name="choose_one_128k"),
        # two long prompts behind what is cached, every token of them with a choice of its own
        _chosen("choose", 2, 4000, 8000, 40, page_tokens=32, name="choose_prompts_4k_behind_8k"),
        # the same serving batch: attention over what was chosen, joined with what attention over a handed-over card gave each sequence
        _chosen("attend", 48, 0, 8192, 64, prior=True, name="attend_chosen_batch_8k"),
        # the same context in larger pages: few rows, what was chosen has to be split
        _chosen("attend", 1, 0, 131071, 64, page_tokens=64, first=4, name="attend_chosen_one_128k"),
        # short questions behind short contexts, ragged: not much to choose from, latency counts
        _chosen("prompt", 6, 150, 300, 8, first=1, last=3, name="prompt_chosen_short"),
        # a whole 8K prompt, a token at 16 pages of 64
        _chosen("prompt", 1, 8192, 0, 16, page_tokens=64, name="prompt_chosen_8k"),
        # a question of 1000 tokens behind a 32K context of a bf16 model of smaller heads, eight query heads to a key head
        _chosen("prompt", 1, 1000, 32768, 64, q_heads=64, head_dim=64, kind="bf16", page_tokens=32, name="prompt_chosen_behind_32k"),
        # one decode step of a batch: a token for every sequence
        _slots(64, 0, 8192, name="slots_step"),
        # many prompts at once, in a batch that is padded to a fixed size
        _slots(300, 200, 3000, padded=4000, name="slots_prompts"),
    ]


_HEADS = ((32, 8, 128), (64, 8, 64), (16, 2, 256), (8, 8, 128), (28, 4, 128), (5, 1, 64), (32, 2, 64), (20, 1, 128))


def _between(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.999)))))))


def draw(rng):
    q_heads, kv_heads, head_dim = rng.choice(_HEADS)
    row = kv_heads * head_dim
    shape = dict(kv_heads=kv_heads, head_dim=head_dim, kind=rng.choice(("fp16", "bf16")), page_tokens=rng.choice((8, 16, 32, 64, 128)))
    op = rng.choice(("digest", "choose", "choose", "attend", "attend", "prompt", "prompt", "slots"))
    if op == "slots":
        rows = _between(rng, 1, 2000)
        new = _between(rng, 1, max(1, 60000 // rows)) if rng.random() < 0.7 else 0
        return _slots(rows, new, _between(rng, 1, 16384), page_tokens=shape["page_tokens"], padded=_between(rng, 1, 5000) if new and rng.random() < 0.5 else 0)
    if op == "digest":
        layers, rows = _between(rng, 1, 32), _between(rng, 1, 64)
        new = _between(rng, 1, max(1, min(8192, 100_000_000 // (layers * rows * row)))) if rng.random() < 0.7 else 0
        return _digest(layers, rows, new, _between(rng, 1, max(1, min(4096, 100_000_000 // (layers * rows * row)))), **shape)
    few = dict(first=rng.choice((0, 1, 1, 4)), last=rng.choice((1, 2, 2, 5)))
    size = shape["page_tokens"]
    if op == "attend" or (op == "choose" and rng.random() < 0.6):
        rows = _between(rng, 1, 128)
        new, old = 0, _between(rng, 1, min(131072, 90_000_000 // (rows * row)))
    else:
        rows = _between(rng, 1, 8)
        new = _between(rng, 1, 6000 // rows)
        old = _between(rng, 1, min(40000, 700_000_000 // (rows * new * q_heads))) if rng.random() < 0.6 else 0
    most = few["first"] + few["last"] + _between(rng, 1, 4096) // size
    if op == "choose":                                            # there is something to choose from
        old = max(old, 3 * (few["first"] + few["last"] + 1) * size + 8)
        most = few["first"] + few["last"] + _between(rng, 1, max(1, (new + old) // size // 3))
    return _chosen(op, rows, new, old, most, q_heads=q_heads, prior=op == "attend" and rng.random() < 0.3, **few, **shape)


def _spread(case, word, rows, longest, least=0):
    """Lengths of the case's sequences: the longest first, the others anywhere below; the third of a large batch is as short as may be."""
    rng = random.Random("%s %d %d %d" % (word, rows, longest, case["page_tokens"]))
    got = [longest] + [rng.randint(min(least, longest), longest) for _ in range(rows - 1)]
    if rows > 16:
        got[2] = min(least, longest)
    return got


def _pages_of(length, page_tokens):
    return -(-length // page_tokens)


def _plan(case):
    """Sequences' lengths with the new tokens, and their new tokens (None: one of each, where there is any)."""
    old = _spread(case, "old", case["rows"], case["longest_old"])
    if not case["longest_new"]:
        return old, None
    new = _spread(case, "new", case["rows"], case["longest_new"], 1)
    return [a + b for a, b in zip(new, old[::-1])], new            # the longest prompt is not the one behind the longest context


def _counts(lens, new):
    return [1 if n else 0 for n in lens] if new is None else new


def _power(x):
    """2^x in 64 bits, x whole and within +- 1000: exact."""
    return ((x.long() + 1023) << 52).view(torch.float64)


def _segments(tokens, gen, longest=160):
    """A topic for each of `tokens` tokens, out of 48, that changes every now and then."""
    lengths = torch.randint(longest // 4, longest, (1 + 4 * tokens // longest,), generator=gen, device="cuda")
    which = torch.randint(0, 48, lengths.shape, generator=gen, device="cuda")
    at = torch.searchsorted(torch.cumsum(lengths, 0), torch.arange(tokens, device="cuda"), right=True)
    return which[at.clamp(max=lengths.numel() - 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, size = TYPES[case["kind"]], case["page_tokens"]
    heads, dim, layers, op = case["kv_heads"], case["head_dim"], case.get("layers", 1), case["op"]
    lens, new = _plan(case)
    rows = len(lens)
    used, width = sum(_pages_of(n, size) for n in lens), max(1, max(_pages_of(n, size) for n in lens)) + 1
    pages = used + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for row, n in enumerate(lens):
        count = _pages_of(n, size)
        table[row, :count] = order[at:at + count]
        at += count
    state = dict(case=case, table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), spare=order[at].long(),
                 status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    counts = _counts(lens, new)
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    tokens = rows if new is None else starts[-1]
    if op == "slots":
        # a cache of one small head stands for any: what the maps say does not depend on the heads
        state["tokens"] = rows if new is None else tokens + case["padded"]
        state["k"] = state["v"] = torch.zeros((1, pages, heads, size, dim), dtype=kind, device="cuda")
        state["more"] = None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
        for name, n, wide in (("starts", rows + 1, torch.int32), ("row", state["tokens"], torch.int32), ("place", state["tokens"], torch.int32),
                              ("slot", state["tokens"], torch.int64)):
            state[name] = torch.empty(n, dtype=wide, device="cuda")
    else:
        state["starts"] = None if new is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
        # keys with a few strong channels and a topic that runs through some dozens of tokens; values of every token's own size
        k = torch.randn((layers, pages, heads, size, dim), generator=gen, device="cuda", dtype=torch.float16)
        strong = torch.randperm(dim, generator=gen, device="cuda")[: max(1, dim // 50)]
        k[..., strong] *= 6.0
        topics = torch.randn((48, heads, dim), generator=gen, device="cuda", dtype=torch.float16)
        for row, n in enumerate(lens):
            if op != "digest" and n:
                mine = topics[_segments(_pages_of(n, size) * size, gen)].view(-1, size, heads, dim).transpose(1, 2)
                k[:, table[row, : _pages_of(n, size)].long()] += mine * 1.2
        state["k"] = k.to(kind)
        if op in ("attend", "prompt"):
            v = torch.randn(k.shape, generator=gen, device="cuda", dtype=torch.float16)
            v *= torch.rand(v.shape[:-1] + (1,), generator=gen, device="cuda", dtype=torch.float32).mul_(2.0).add_(0.5).to(v.dtype)
            state["v"] = v.to(kind)
        else:
            state["v"] = state["k"]                               # not looked at
        del k
        # steps with room for the largest key of a channel: 127 steps of 2^e and no power of two less
        largest = state["k"].abs().amax((1, 3)).float() / 127.0
        state["exponents"] = torch.frexp(largest)[1].to(torch.int8).contiguous()
        # what earlier calls left there
        state["digest"] = torch.randint(-128, 128, (layers, pages, heads, 2, dim), generator=gen, device="cuda", dtype=torch.int8)
    if op in ("choose", "attend", "prompt"):
        hq = case["q_heads"]
        wide = torch.randn(tokens, (hq + 2 * heads) * dim, generator=gen, device="cuda").to(kind)          # a fused projection's result
        q = wide[:, : hq * dim].view(tokens, heads, hq // heads, dim)
        q += (topics[_segments(tokens, gen, 60)] * 0.8).to(kind).unsqueeze(2)                              # neighbours ask about the same
        state["q"] = q.view(tokens, hq, dim)
        state["digest"][0] = _digest_of(state["k"], state["exponents"])[0]                                 # of full pages; others are never looked at
        words = (width + 31) // 32
        state["choice"] = torch.empty((tokens, heads, words), dtype=torch.int32, device="cuda")
        if op != "choose":
            state["choice"].copy_(_run_choose(state, case))
            state["out"] = torch.empty(tokens, hq, dim, dtype=torch.float32 if op == "attend" else kind, device="cuda")
            state["lse"] = torch.empty(tokens, hq, dtype=torch.float32, device="cuda")
            if case["prior"]:
                state["prior_out"] = torch.randn(tokens, hq, dim, generator=gen, device="cuda") * 0.3
                state["prior_lse"] = torch.randn(tokens, hq, generator=gen, device="cuda") + math.log(1 + sum(lens) / rows)
    if own:
        import paper_2605_03884_amd as qkv
        state["pages"] = qkv.Pages.make(list(state["k"]), list(state["v"]), table, state["lens"])
        if op in ("digest", "choose"):
            state["digests"] = qkv.Digests.make(state["pages"], list(state["digest"]), state["exponents"])
            state["batch"] = None if new is None else tokens      # a caller knows the size of its batch
        size_of = {"choose": lambda: qkv.paged_choose_workspace(state["pages"], tokens),
                   "attend": lambda: qkv.paged_attend_chosen_workspace(state["pages"], case["q_heads"], case["most"]),
                   "prompt": lambda: qkv.paged_prompt_chosen_workspace(state["pages"], case["q_heads"], tokens)}.get(op)
        if size_of:
            state["workspace"] = torch.empty(size_of(), dtype=torch.uint8, device="cuda")
    return state


def _digest_of(k, exponents):
    """Codes [layers, pages, heads, 2, dim] (largest, smallest) of pages [layers, pages, heads, size, dim], in 32 bits: the steps are powers of two."""
    step = _power(-exponents.long()).float()[:, None, :, :]
    top, low = k.amax(3).float() * step, k.amin(3).float() * step
    top, low = torch.ceil(top).clamp(-128, 127), torch.floor(low).clamp(-128, 127)
    return torch.stack((torch.where(torch.isnan(top), 127, top), torch.where(torch.isnan(low), -128, low)), 3).to(torch.int8)


def _run_digest(s, case):
    size, most = case["page_tokens"], 1 + case["longest_new"] // case["page_tokens"]
    lens = s["lens"].long()
    count = (lens > 0).long() if s["starts"] is None else (s["starts"][1:] - s["starts"][:-1]).long()
    first, end = (lens - count) // size, lens // size                      # the pages that the new tokens have filled
    # every sequence has room for as many as the longest may fill; behind its last one the last one stands again, and where there is none a page in nobody's use
    entry = torch.minimum(first.unsqueeze(1) + torch.arange(most, device="cuda"), end.unsqueeze(1) - 1)
    some = (end > first).unsqueeze(1)
    page = torch.where(some, s["table"].gather(1, entry.clamp(min=0)).long(), s["spare"]).view(-1)
    got = _digest_of(s["k"][:, page], s["exponents"])
    s["digest"][:, page] = torch.where(some.expand(-1, most).reshape(1, -1, 1, 1, 1), got, s["digest"][:, page])
    return s["digest"]


def _query_codes(q, exponents):
    """Codes [tokens, heads, 2 dim] of queries [tokens, heads, rep, dim] in 32 bits: positive and negative parts, each summed over the heads in their order."""
    above, below = torch.zeros_like(q[:, :, 0]), torch.zeros_like(q[:, :, 0])
    for r in range(q.shape[2]):
        above, below = above + q[:, :, r].clamp(min=0), below + q[:, :, r].clamp(max=0)
    largest = torch.maximum(above, -below)
    e = exponents.long()
    height = torch.where(largest > 0, torch.frexp(largest)[1].long() - 1 + e, -900).amax(-1, keepdim=True)
    step = _power((e - height + 6).clamp(-1000, 1000))
    return torch.cat((torch.round(above * step).clamp(max=127), torch.round(below * step).clamp(min=-127)), -1).float()


def _places(s, case):
    """Of every token its sequence, its number among that one's new tokens, and its place in it."""
    if s["starts"] is None:
        row = torch.arange(case["rows"], device="cuda")
        return row, torch.zeros_like(row), s["lens"].long() - 1
    starts = s["starts"].long()
    every = torch.arange(s["q"].shape[0], device="cuda")
    row = torch.searchsorted(starts, every, right=True) - 1
    return row, every - starts[row], s["lens"][row].long() - starts[row + 1] + every


def _packed(chosen):
    """Truth values [..., pages] as words of 32."""
    words = (chosen.shape[-1] + 31) // 32
    chosen = torch.nn.functional.pad(chosen, (0, words * 32 - chosen.shape[-1])).view(chosen.shape[:-1] + (words, 32))
    x = (chosen.long() << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _unpacked(choice, pages):
    return ((choice.unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(-2)[..., :pages].bool()


def _run_choose(s, case):
    size, heads, table = case["page_tokens"], case["kv_heads"], s["table"]
    rows, width = table.shape
    row, number, place = _places(s, case)
    tokens, hq, dim = s["q"].shape
    codes = _query_codes(s["q"].float().view(tokens, heads, hq // heads, dim), s["exponents"][0])
    most_new = max(1, case["longest_new"])
    padded = torch.zeros(rows, most_new, heads, 2 * dim, device="cuda")
    padded[row, number] = codes
    bounds = s["digest"][0, table.clamp(min=0).long()].float().permute(0, 2, 4, 3, 1)                   # [rows, heads, dim, 2, width]
    bounds = bounds.transpose(2, 3).reshape(rows, heads, 2 * dim, width)
    scores = (padded.transpose(1, 2) @ bounds).transpose(1, 2)[row, number].long()                      # whole numbers below 2^24: exact in 32 bits
    page = torch.arange(width, device="cuda")
    mine = (place // size).view(-1, 1, 1)
    there = ((page <= mine) & (place.view(-1, 1, 1) >= 0) & (table >= 0)[row].unsqueeze(1)).expand(-1, heads, -1)
    always = (page < case["first"]) | (page > mine - case["last"])
    rank = torch.where(always, 1 << 30, scores) * (1 << 24) - page                                      # equal scores: the lowest page first
    rank = torch.where(there, rank, -(1 << 62))
    best = rank.topk(min(case["most"], width), -1).indices
    return _packed(torch.zeros_like(there).scatter(-1, best, True) & there)


def _softmax_product(scores, seen, values):
    """exp(scores) over what is seen, times the values; rows that see nothing give 0 and -inf."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    weight = torch.exp(scores - top)
    total = weight.sum(-1, keepdim=True)
    out = weight @ values / torch.where(total == 0, torch.ones_like(total), total)
    return out, (top + torch.log(total)).squeeze(-1)


def _run_attend(s, case):
    size, heads, table = case["page_tokens"], case["kv_heads"], s["table"]
    rows, width = table.shape
    hq, dim = s["q"].shape[1:]
    chosen = _unpacked(s["choice"], width)                                                               # [rows, heads, width]
    entry = torch.where(chosen, width - torch.arange(width, device="cuda"), 0).topk(min(case["most"], width), -1).values       # the lowest first, then 0
    held, entry = entry > 0, (width - entry) % width
    page = table.gather(1, entry.flatten(1)).view(entry.shape).clamp(min=0).long()
    head = torch.arange(heads, device="cuda").view(1, -1, 1)
    k, v = (x[0][page, head].reshape(rows, heads, -1, dim).float() for x in (s["k"], s["v"]))
    token = entry.unsqueeze(-1) * size + torch.arange(size, device="cuda")
    seen = ((token < s["lens"].view(-1, 1, 1, 1)) & held.unsqueeze(-1)).flatten(2).unsqueeze(2)
    q = s["q"].float().view(rows, heads, -1, dim)
    out, lse = _softmax_product(q @ k.transpose(-1, -2) * dim ** -0.5, seen, v)
    out, lse = out.reshape(rows, -1, dim), lse.reshape(rows, -1)
    if case["prior"]:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = out * torch.exp(lse - both).unsqueeze(-1) + s["prior_out"] * torch.exp(s["prior_lse"] - both).unsqueeze(-1)
        lse = both
    return out, lse


def _run_prompt(s, case):
    size, heads, table = case["page_tokens"], case["kv_heads"], s["table"]
    rows, width = table.shape
    row, number, place = _places(s, case)
    total, hq, dim = s["q"].shape
    most = case["longest_new"]
    k, v = (x[0][table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(rows, heads, 1, width * size, dim).float() for x in (s["k"], s["v"]))
    q = torch.zeros(rows, most, heads, hq // heads, dim, device="cuda")
    q[row, number] = s["q"].float().view(total, heads, -1, dim)
    q = q.permute(0, 2, 3, 1, 4)                                                                        # [rows, heads, rep, most, dim]
    choice = torch.zeros((rows, most) + s["choice"].shape[1:], dtype=torch.int32, device="cuda")
    choice[row, number] = s["choice"]
    own_place = torch.full((rows, most), -1, device="cuda")
    own_place[row, number] = place
    seen = _unpacked(choice, width).transpose(1, 2).repeat_interleave(size, -1)                         # [rows, heads, most, width * size]
    seen = (seen & (torch.arange(width * size, device="cuda") <= own_place[:, None, :, None])).unsqueeze(2)
    scores = (q.flatten(2, 3) @ k.squeeze(2).transpose(-1, -2)).view(rows, heads, -1, most, width * size) * dim ** -0.5
    out, lse = _softmax_product(scores, seen, v)
    out = out.permute(0, 3, 1, 2, 4)[row, number].reshape(total, -1, dim)
    lse = lse.permute(0, 3, 1, 2)[row, number].reshape(total, -1)
    return out.to(s["k"].dtype), lse


def _run_slots(s, case):
    size, table = case["page_tokens"], s["table"]
    lens = s["lens"].long()
    count = (lens > 0).long() if s["more"] is None else s["more"].long()
    ends = torch.cumsum(count, 0)
    every = torch.arange(s["tokens"], device="cuda")
    row = torch.searchsorted(ends, every, right=True)
    there = row < case["rows"]
    row = row.clamp(max=case["rows"] - 1)
    place = lens[row] - ends[row] + every
    page = table[row, (place // size).clamp(0, table.shape[1] - 1)].long()
    starts = torch.nn.functional.pad(ends, (1, 0)).to(torch.int32)
    return (starts, torch.where(there, row, -1).to(torch.int32), torch.where(there, place, -1).to(torch.int32),
            torch.where(there, page * size + place % size, -1))


def _run_own(s, case):
    import paper_2605_03884_amd as qkv
    op, pages, status = case["op"], s["pages"], s["status"]
    if op == "digest":
        qkv.pages_digest(pages, s["digests"], count=case["layers"], starts=s["starts"], tokens=s["batch"], status=status)
        return s["digest"]
    if op == "choose":
        return qkv.paged_choose(pages, s["digests"], s["q"], case["most"], s["choice"], first=case["first"], last=case["last"], starts=s["starts"],
                                workspace=s["workspace"], status=status)
    if op == "attend":
        prior = (s["prior_out"], s["prior_lse"]) if case["prior"] else None
        return qkv.paged_attend_chosen(pages, s["choice"], s["q"], case["head_dim"] ** -0.5, s["out"], s["lse"], most=case["most"], prior=prior,
                                       workspace=s["workspace"], status=status)
    if op == "prompt":
        return qkv.paged_prompt_chosen(pages, s["choice"], s["q"], s["starts"], case["head_dim"] ** -0.5, s["out"], s["lse"], workspace=s["workspace"],
                                       status=status)
    qkv.pages_slots(pages, s["starts"], s["row"], s["place"], s["slot"], more=s["more"], status=status)
    return s["starts"], s["row"], s["place"], s["slot"]


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"digest": _run_digest, "choose": _run_choose, "attend": _run_attend, "prompt": _run_prompt, "slots": _run_slots}[case["op"]](state, case)


def _seen_count(place, case):
    """Tokens that a query at `place` sees: its own page up to there, and of the full ones in front of it as many as may be chosen."""
    if place < 0:
        return 0
    size = case["page_tokens"]
    return min(place // size, case["most"] - 1) * size + place % size + 1


def work(case):
    lens, new = _plan(case)
    counts, size, op = _counts(lens, new), case["page_tokens"], case["op"]
    heads, dim = case["kv_heads"], case["head_dim"]
    if op == "digest":
        filled = sum(n // size - (n - c) // size for n, c in zip(lens, counts))
        return {"bytes": case["layers"] * heads * (filled * dim * (2 * size + 2) + dim), "flops": 0}
    if op == "slots":
        tokens = len(lens) if new is None else sum(counts) + case["padded"]
        return {"bytes": 16 * tokens + 12 * len(lens) + 4 * sum(n // size - (n - c) // size + 1 for n, c in zip(lens, counts) if c), "flops": 0}
    hq, tokens = case["q_heads"], sum(counts)
    places = [range(n - c, n) for n, c in zip(lens, counts)]
    if op == "choose":
        scored = [max(0, p // size + 1 - case["first"] - case["last"]) for x in places for p in x]
        read = sum(max(0, (n - 1) // size + 1 - case["first"] - case["last"]) for n in lens if n)
        words = (max(_pages_of(n, size) for n in lens) + 1 + 31) // 32
        return {"bytes": read * heads * 2 * dim + tokens * (hq * dim * 2 + heads * words * 4), "flops": 4 * dim * heads * sum(scored)}
    seen = sum(_seen_count(p, case) for x in places for p in x)
    if op == "attend":
        answer = tokens * hq * (dim * 6 + 4) + (tokens * hq * (dim * 4 + 4) if case["prior"] else 0)
        return {"bytes": seen * heads * dim * 4 + answer, "flops": 4 * seen * hq * dim}
    read = sum(min(n, sum(_seen_count(p, case) for p in x)) for n, x in zip(lens, places))
    return {"bytes": read * heads * dim * 4 + tokens * hq * (dim * 4 + 4), "flops": 4 * seen * hq * dim}


def _exact_choice(s, case, lens, counts):
    """A choice written out: 64-bit whole numbers, sorted by score and place."""
    size, heads, table = case["page_tokens"], case["kv_heads"], s["table"].cpu()
    width = table.shape[1]
    words = (width + 31) // 32
    e = s["exponents"][0].cpu().double()
    out, at = [], 0
    for row, (n, c) in enumerate(zip(lens, counts)):
        full = n // size
        bounds = s["digest"][0, table[row, :full].long().cuda()].double()                               # [full, heads, 2, dim]
        # one token of each sequence, an empty place among them, where there are no starts
        for first in range(0, max(c, 1 if s["starts"] is None else 0), 512):
            here = min(512, c - first) if c else 1
            bits = torch.zeros(here, heads, words * 32, dtype=torch.bool)
            if c:
                q = s["q"][at + first:at + first + here].float().cpu().view(here, heads, -1, case["head_dim"])
                pos, neg = q[:, :, 0].clamp(min=0), q[:, :, 0].clamp(max=0)
                for r in range(1, q.shape[2]):                    # sums in 32 bits, as they are defined
                    pos, neg = pos + q[:, :, r].clamp(min=0), neg + q[:, :, r].clamp(max=0)
                real = torch.maximum(pos, -neg).double() * torch.pow(2.0, e)
                unit = torch.pow(2.0, torch.floor(torch.log2(real.amax(-1, keepdim=True))) - 6)
                p = torch.round(pos.double() * torch.pow(2.0, e) / unit).clamp(max=127)
                m = torch.round(neg.double() * torch.pow(2.0, e) / unit).clamp(min=-127)
                score = torch.stack([p[:, h].cuda() @ bounds[:, h, 0].T + m[:, h].cuda() @ bounds[:, h, 1].T for h in range(heads)], 1).cpu()
                ranked = torch.sort(-score, dim=-1, stable=True).indices
                for i in range(here):
                    mine = (n - c + first + i) // size
                    lo, hi = min(case["first"], mine + 1), max(0, mine + 1 - case["last"])
                    bits[i, :, :lo] = True
                    bits[i, :, hi:mine + 1] = True
                    more = max(0, case["most"] - int(bits[i, 0].sum()))
                    order = ranked[i]
                    order = order[(order >= lo) & (order < hi)].view(heads, -1)[:, :more]
                    bits[i].scatter_(1, order, True)
            x = (bits.view(here, heads, words, 32).long() << torch.arange(32)).sum(-1)
            out.append(torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32))
        at += max(c, 1 if s["starts"] is None else 0)
    return torch.cat(out)


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _plan(case)
    counts, size, op = _counts(lens, new), case["page_tokens"], case["op"]
    table = s["table"].tolist()
    if op == "digest":
        for n, c, numbers in zip(lens, counts, table):
            for j in range((n - c) // size, n // size):
                real = s["k"][:, numbers[j]].double() / torch.pow(2.0, s["exponents"].double()).unsqueeze(2)
                s["digest"][:, numbers[j], :, 0] = torch.ceil(real.amax(2)).clamp(-128, 127).to(torch.int8)
                s["digest"][:, numbers[j], :, 1] = torch.floor(real.amin(2)).clamp(-128, 127).to(torch.int8)
        return s["digest"]
    if op == "choose":
        return _exact_choice(s, case, lens, counts)
    if op == "slots":
        starts, row, place, slot = [0], [], [], []
        for b, (n, c) in enumerate(zip(lens, counts)):
            starts.append(starts[-1] + c)
            row += [b] * c
            place += range(n - c, n)
            slot += [table[b][p // size] * size + p % size for p in range(n - c, n)]
        behind = [-1] * (s["tokens"] - len(row))
        return [torch.tensor(x, dtype=t) for x, t in ((starts, torch.int32), (row + behind, torch.int32), (place + behind, torch.int32), (slot + behind, torch.int64))]
    hq, dim, heads = case["q_heads"], case["head_dim"], case["kv_heads"]
    outs, lses, at = [], [], 0
    for b, (n, c) in enumerate(zip(lens, counts)):
        if op == "attend":
            c = 1
        out = torch.zeros(c, hq, dim, dtype=torch.float64, device="cuda")
        lse = torch.full((c, hq), -math.inf, dtype=torch.float64, device="cuda")
        if n:
            numbers = s["table"][b, : _pages_of(n, size)].long()
            t = torch.arange(n, device="cuda")
            for h in range(heads):
                k, v = (x[0, numbers, h].reshape(-1, dim)[:n].double() for x in (s["k"], s["v"]))
                for lo in range(0, c, 1024):
                    hi = min(c, lo + 1024)
                    word = s["choice"][at + lo:at + hi, h].long()
                    hidden = ((word[:, (t // size) // 32] >> ((t // size) % 32)) & 1) == 0
                    hidden |= t > torch.arange(n - c + lo, n - c + hi, device="cuda").unsqueeze(1)
                    for r in range(h * (hq // heads), (h + 1) * (hq // heads)):
                        score = (s["q"][at + lo:at + hi, r].double() @ k.T) / math.sqrt(dim)
                        score[hidden] = -math.inf
                        lse[lo:hi, r] = torch.logsumexp(score, 1)
                        out[lo:hi, r] = torch.softmax(score, 1).nan_to_num(0.0) @ v
        outs.append(out)
        lses.append(lse)
        at += c
    out, lse = torch.cat(outs), torch.cat(lses)
    if case["prior"]:
        a, b = lse, s["prior_lse"].double()
        top = torch.maximum(a, b)
        wa, wb = torch.exp(a - top), torch.exp(b - top)
        out = (out * wa[..., None] + s["prior_out"].double() * wb[..., None]) / (wa + wb)[..., None]
        lse = top + torch.log(wa + wb)
    return out, lse
