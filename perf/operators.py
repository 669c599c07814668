"""A receiver's own cache in pages, and the attention that reads it: what each call computes, in elementary torch operations, and the
calls of paper_2605_03884_amd that do the same (where `own` is true).

A cache is a pool of pages of page_tokens tokens, tensors [layers, pages, kv_heads, page_tokens, head_dim] for keys and values; a sequence
is a row of a table of page numbers and a length.  A page may belong to several sequences (refs counts them); 0 means free.

  attend    one new token of every sequence over its pages: out [rows, q_heads, head_dim] and lse, in 32 bits; optionally joined with the
            (out, lse) of attention over tokens that are somewhere else (a card)
  prompt    many new tokens of every sequence over its pages, each up to its own position; out in the cache's type, lse in 32 bits
            both optionally with a sliding window: a query at position p sees tokens t with p - window < t <= p, and t < sinks
  append    rows of new tokens into the pages
  fork      sequences that go on from another one: full pages are shared, the tokens in a last page that is not full are copied
  compact   pages that are in use move to the lowest places, tables follow

A case is a dict of plain values.  Lengths are a fixed function of the case; contents and the order of the pages come from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _attend(rows, longest, q_heads=32, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, window=0, sinks=0, prior=False, **more):
    return dict(op="attend", rows=rows, longest=longest, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, kind=kind,
                page_tokens=page_tokens, window=window, sinks=sinks, prior=prior, **more)


def _prompt(rows, longest_new, longest_old, q_heads=32, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, window=0, sinks=0, **more):
    return dict(op="prompt", rows=rows, longest_new=longest_new, longest_old=longest_old, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, kind=kind, page_tokens=page_tokens, window=window, sinks=sinks, **more)


def _append(layers, rows, longest_new, longest_old, dense, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, **more):
    return dict(op="append", layers=layers, rows=rows, longest_new=longest_new, longest_old=longest_old, dense=dense, kv_heads=kv_heads,
                head_dim=head_dim, kind=kind, page_tokens=page_tokens, **more)


def _fork(layers, parents, children, longest, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, **more):
    return dict(op="fork", layers=layers, parents=parents, children=children, longest=longest, kv_heads=kv_heads, head_dim=head_dim,
                kind=kind, page_tokens=page_tokens, **more)


def _compact(layers, rows, longest, spare, kv_heads=8, head_dim=128, kind="fp16", page_tokens=16, **more):
    return dict(op="compact", layers=layers, rows=rows, longest=longest, spare=spare, kv_heads=kv_heads, head_dim=head_dim, kind=kind,
                page_tokens=page_tokens, **more)


def listed():
    return [
        # the first tokens of one answer: launches and latency only
        _attend(1, 37, name="attend_one_short"),
        # a serving batch of a Llama-3.1-8B shaped layer, lengths all over, one place in the batch empty, joined with what attention over a
        # handed-over card gave each sequence
        _attend(48, 8192, prior=True, name="attend_batch_8k_joined"),
        # one sequence with a full 128K context: few rows, the length has to be split
        _attend(1, 131071, page_tokens=64, name="attend_one_128k"),
        # a bf16 model of smaller heads, eight query heads to a key head, that sees a window and the first four tokens
        _attend(64, 16384, q_heads=64, head_dim=64, kind="bf16", page_tokens=32, window=1000, sinks=4, name="attend_window_bf16"),
        # short questions behind short contexts, ragged
        _prompt(6, 150, 300, name="prompt_short_ragged"),
        # a whole 8K prompt
        _prompt(1, 8192, 0, page_tokens=64, name="prompt_8k"),
        # two long prompts of a bf16 model with a window and sinks, one continued behind what is cached
        _prompt(2, 8000, 3000, head_dim=64, kind="bf16", page_tokens=32, window=1024, sinks=4, name="prompt_window_bf16"),
        # a question of 61 tokens behind a shared 32K context: few queries, many keys
        _prompt(1, 61, 32768, page_tokens=128, name="prompt_61_behind_32k"),
        # one decode step of a batch: a row of keys and of values for every sequence, parts of a fused projection's result
        _append(1, 64, 1, 8192, False, kind="bf16", name="append_step"),
        # a card that was rebuilt as a dense cache goes into pages, all layers at once
        _append(32, 1, 4100, 64, True, page_tokens=64, name="append_dense_4100"),
        # agents that go on from four shared contexts, six each
        _fork(16, 4, 24, 3000, page_tokens=64, name="fork_24"),
        # a pool with as many holes as pages in use
        _compact(16, 40, 1400, 800, page_tokens=32, name="compact_half"),
    ]


_HEADS = ((32, 8, 128), (64, 8, 64), (16, 2, 256), (8, 8, 128), (28, 4, 128), (5, 1, 64), (32, 2, 64), (20, 1, 128))


def _between(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.999)))))))


def draw(rng):
    q_heads, kv_heads, head_dim = rng.choice(_HEADS)
    kind = rng.choice(("fp16", "bf16"))
    page_tokens = rng.choice((8, 16, 32, 64, 128, 256))
    shape = dict(kv_heads=kv_heads, head_dim=head_dim, kind=kind, page_tokens=page_tokens)
    row = kv_heads * head_dim
    op = rng.choice(("attend", "attend", "prompt", "prompt", "append", "fork", "compact"))
    window = _between(rng, 16, 4096) if rng.random() < 0.4 else 0
    sinks = rng.choice((0, 1, 4, 63)) if window else 0
    if op == "attend":
        rows = _between(rng, 1, 128)
        return _attend(rows, _between(rng, 1, min(131072, 90_000_000 // (rows * row))), q_heads=q_heads, window=window, sinks=sinks,
                       prior=rng.random() < 0.3, **shape)
    if op == "prompt":
        rows = _between(rng, 1, 8)
        new = _between(rng, 1, 6000 // rows)
        old = _between(rng, 1, min(40000, 700_000_000 // (rows * new * q_heads))) if rng.random() < 0.6 else 0
        return _prompt(rows, new, old, q_heads=q_heads, window=window, sinks=sinks, **shape)
    if op == "append":
        layers, rows = _between(rng, 1, 32), _between(rng, 1, 32)
        new = _between(rng, 1, max(1, min(8192, 100_000_000 // (layers * rows * row))))
        return _append(layers, rows, new, rng.randrange(0, 300), rng.random() < 0.5, **shape)
    layers = _between(rng, 1, 32)
    if op == "fork":
        parents = _between(rng, 1, 4)
        children = parents * _between(rng, 1, 8)
        longest = _between(rng, 1, max(1, min(4096, 60_000_000 // (layers * row * (parents + 1)))))
        return _fork(layers, parents, children, longest, **shape)
    rows = _between(rng, 1, 40)
    longest = _between(rng, 1, max(1, min(4096, 40_000_000 // (layers * row * rows))))
    return _compact(layers, rows, longest, 1 + _between(rng, 1, 2 * rows * (1 + longest // page_tokens)), **shape)


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
    """Sequences' lengths (for prompt and append with the new tokens) and new tokens, and how many pages the pool has and how many stand in tables."""
    op, size = case["op"], case["page_tokens"]
    if op == "attend":
        lens, new = _spread(case, "attend", case["rows"], case["longest"]), None
    elif op in ("prompt", "append"):
        new = _spread(case, "new", case["rows"], case["longest_new"], 1)
        old = _spread(case, "old", case["rows"], case["longest_old"])
        if op == "prompt":
            old = old[::-1]                                   # the longest prompt is not the one behind the longest context
        lens = [a + b for a, b in zip(new, old)]
    elif op == "fork":
        lens = _spread(case, "parents", case["parents"], case["longest"], 1)
        lens += _spread(case, "children", case["children"], max(1, case["longest"] // 4))
        new = None
    else:
        lens, new = _spread(case, "rows", case["rows"], case["longest"], 1), None
    used = sum(_pages_of(n, size) for n in lens)
    spare = case["spare"] if op == "compact" else (case["children"] * 2 + 8) if op == "fork" else 3
    return lens, new, used + spare, used


def _keys_and_values(shape, kind, gen):
    """Keys with a few strong channels, values of every token's own size: what a model's cache looks like, roughly."""
    k = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32 if math.prod(shape) < 1 << 28 else torch.float16)
    v = torch.randn(shape, generator=gen, device="cuda", dtype=k.dtype)
    strong = torch.randperm(shape[-1], generator=gen, device="cuda")[: max(1, shape[-1] // 50)]
    k[..., strong] *= 8.0
    v *= torch.rand(shape[:-1] + (1,), generator=gen, device="cuda", dtype=torch.float32).mul_(2.0).add_(0.5).to(v.dtype)
    return k.to(kind), v.to(kind)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, size = TYPES[case["kind"]], case["page_tokens"]
    heads, dim, layers, op = case["kv_heads"], case["head_dim"], case.get("layers", 1), case["op"]
    lens, new, pages, used = _plan(case)
    rows = len(lens)
    width = max(1, max(_pages_of(n, size) for n in lens)) + 1
    k, v = _keys_and_values((layers, pages, heads, size, dim), kind, gen)
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for row, n in enumerate(lens):
        count = _pages_of(n, size)
        table[row, :count] = order[at:at + count]
        at += count
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[order[:at].long()] = 1
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    state = dict(case=case, k=k, v=v, table=table, lens=length, refs=refs, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if op in ("attend", "prompt"):
        tokens = rows if op == "attend" else sum(new)
        hq = case["q_heads"]
        wide = torch.randn(tokens, (hq + 2 * heads) * dim, generator=gen, device="cuda").to(kind)      # a fused projection's result
        state["q"] = wide[:, : hq * dim].view(tokens, hq, dim)
        state["out"] = torch.empty(tokens, hq, dim, dtype=torch.float32 if op == "attend" else kind, device="cuda")
        state["lse"] = torch.empty(tokens, hq, dtype=torch.float32, device="cuda")
        if op == "prompt":
            starts = [0]
            for n in new:
                starts.append(starts[-1] + n)
            state["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        elif case["prior"]:
            state["prior_out"] = torch.randn(tokens, hq, dim, generator=gen, device="cuda") * 0.3
            state["prior_lse"] = torch.randn(tokens, hq, generator=gen, device="cuda") + math.log(1 + sum(lens) / rows)
    elif op == "append":
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        state["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        tokens = starts[-1]
        if case["dense"]:        # [layers, heads, tokens, dim], a dense cache
            nk, nv = _keys_and_values((layers, heads, tokens, dim), kind, gen)
            state["new_k"], state["new_v"] = nk.transpose(1, 2), nv.transpose(1, 2)
        else:                    # parts of a fused projection's result, with room for four times the query heads
            wide = torch.randn(layers, tokens, 6 * heads * dim, generator=gen, device="cuda").to(kind)
            state["new_k"] = wide[..., 4 * heads * dim: 5 * heads * dim].view(layers, tokens, heads, dim)
            state["new_v"] = wide[..., 5 * heads * dim:].view(layers, tokens, heads, dim)
    elif op == "fork":
        parents, children = case["parents"], case["children"]
        state["source"] = torch.arange(children, dtype=torch.int32, device="cuda") % parents
        state["target"] = parents + torch.randperm(children, generator=gen, device="cuda").to(torch.int32)
    else:
        state["first_table"], state["first_refs"] = table.clone(), refs.clone()
        state["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2605_03884_amd as qkv
        state["pages"] = qkv.Pages.make(list(k), list(v), table, length, refs)
        if op == "attend":
            state["workspace"] = torch.empty(qkv.paged_attend_workspace(state["pages"], case["q_heads"]), dtype=torch.uint8, device="cuda")
        elif op == "prompt":
            state["workspace"] = torch.empty(qkv.paged_prompt_workspace(state["pages"], case["q_heads"], sum(new)), dtype=torch.uint8, device="cuda")
        elif op == "compact":
            state["workspace"] = torch.empty(qkv.pages_compact_workspace(state["pages"]), dtype=torch.uint8, device="cuda")
    return state


def _gathered(pool, table):
    """One layer's pages [pages, heads, size, dim] as [rows, heads, width * size, dim] in 32 bits; entries that name no page give page 0."""
    rows, width = table.shape
    _, heads, size, dim = pool.shape
    return pool[table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(rows, heads, width * size, dim).float()


def _visible(position, tokens, window, sinks):
    """Whether a query at `position` [...] sees token 0 .. tokens - 1: [..., tokens]."""
    t = torch.arange(tokens, device=position.device)
    p = position.unsqueeze(-1)
    seen = t <= p
    if window:
        seen = seen & ((t > p - window) | (t < sinks))
    return seen


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
    k, v = _gathered(s["k"][0], s["table"]), _gathered(s["v"][0], s["table"])
    rows, heads, tokens, dim = k.shape
    q = s["q"].float().reshape(rows, heads, -1, dim)
    seen = _visible(s["lens"] - 1, tokens, case["window"], case["sinks"])
    out, lse = _softmax_product(q @ k.transpose(-1, -2) * dim ** -0.5, seen[:, None, None, :], v)
    out, lse = out.reshape(rows, -1, dim), lse.reshape(rows, -1)
    if case["prior"]:
        both = torch.logaddexp(lse, s["prior_lse"])
        out = out * torch.exp(lse - both).unsqueeze(-1) + s["prior_out"] * torch.exp(s["prior_lse"] - both).unsqueeze(-1)
        lse = both
    return out, lse


def _run_prompt(s, case):
    k, v = _gathered(s["k"][0], s["table"]), _gathered(s["v"][0], s["table"])
    rows, heads, tokens, dim = k.shape
    starts, total = s["starts"], s["q"].shape[0]
    every = torch.arange(total, device="cuda")
    row = torch.searchsorted(starts, every.to(torch.int32), right=True) - 1
    place = every - starts[row]
    most = case["longest_new"]
    q = torch.zeros(rows, most, heads, case["q_heads"] // heads, dim, device="cuda")
    q[row, place] = s["q"].float().view(total, heads, -1, dim)
    q = q.permute(0, 2, 3, 1, 4).reshape(rows, heads, -1, dim)
    count = starts[1:] - starts[:-1]
    position = (s["lens"] - count).unsqueeze(1) + torch.arange(most, device="cuda")
    seen = _visible(position, tokens, case["window"], case["sinks"])[:, None, None]
    scores = (q @ k.transpose(-1, -2)).view(rows, heads, -1, most, tokens) * dim ** -0.5
    out, lse = _softmax_product(scores, seen, v.unsqueeze(2))
    out = out.permute(0, 3, 1, 2, 4)[row, place].reshape(total, -1, dim)
    lse = lse.permute(0, 3, 1, 2)[row, place].reshape(total, -1)
    return out.to(s["k"].dtype), lse


def _run_append(s, case):
    starts, size = s["starts"], case["page_tokens"]
    every = torch.arange(s["new_k"].shape[1], device="cuda")
    row = torch.searchsorted(starts, every.to(torch.int32), right=True) - 1
    position = s["lens"][row] - starts[row + 1] + every
    page, slot = s["table"][row, position // size].long(), position % size
    s["k"][:, page, :, slot] = s["new_k"].transpose(0, 1)
    s["v"][:, page, :, slot] = s["new_v"].transpose(0, 1)
    return s["k"], s["v"]


def _run_fork(s, case):
    table, lens, refs, size = s["table"], s["lens"], s["refs"], case["page_tokens"]
    source, target = s["source"].long(), s["target"].long()
    entry = torch.arange(table.shape[1], device="cuda")
    mine = table[target]
    held = (entry < ((lens[target] + size - 1) // size).unsqueeze(1)) & (mine >= 0)
    refs.index_add_(0, mine.clamp(min=0).long().view(-1), -held.to(torch.int32).view(-1))
    length = lens[source]
    full, part = length // size, length % size
    shared = entry < full.unsqueeze(1)
    given = table[source]
    refs.index_add_(0, given.clamp(min=0).long().view(-1), (shared & (given >= 0)).to(torch.int32).view(-1))
    free = torch.argsort((refs > 0).to(torch.int32), stable=True)                 # free pages first, the lowest in front
    wants = part > 0
    page = free[(torch.cumsum(wants, 0) - 1).clamp(min=0)].to(torch.int32)
    last = (entry == full.unsqueeze(1)) & wants.unsqueeze(1)
    table[target] = torch.where(shared, given, torch.where(last, page.unsqueeze(1), mine))
    refs.index_add_(0, page.long(), wants.to(torch.int32))
    lens[target] = length
    old = given.gather(1, ((length - 1).clamp(min=0) // size).long().unsqueeze(1)).squeeze(1).clamp(min=0).long()     # a parent's page: none is written
    copied = (torch.arange(size, device="cuda") < part.unsqueeze(1)).view(1, -1, 1, size, 1)
    to = torch.where(wants, page.long(), old)
    for pool in (s["k"], s["v"]):
        pool[:, to] = torch.where(copied, pool[:, old], pool[:, to])
    return table, lens, refs, s["k"], s["v"]


def _run_compact(s, case):
    table, refs = s["table"], s["refs"]
    table.copy_(s["first_table"])              # the same holes in every pass: a move leaves its source's contents where they were
    refs.copy_(s["first_refs"])
    pages = refs.numel()
    used = (refs > 0).to(torch.int32)
    live = used.sum(dtype=torch.int32)
    place = torch.arange(pages, device="cuda")
    low = place < live
    hole_first = torch.argsort(torch.where(low & (used == 0), 0, 1), stable=True)       # holes in order, then the rest
    mover_first = torch.argsort(torch.where(~low & (used == 1), 0, 1), stable=True)
    moves = (low & (used == 0)).sum()
    moving = place < moves
    takes = place.clone()                      # whose contents a page has afterwards
    takes[hole_first] = torch.where(moving, mover_first, hole_first)
    goes = place.clone()                       # where a page in use is afterwards
    goes[mover_first] = torch.where(moving, hole_first, mover_first)
    refs.copy_(torch.where(low, refs[takes], torch.zeros_like(refs)))
    mine = torch.arange(table.shape[1], device="cuda") < ((s["lens"] + case["page_tokens"] - 1) // case["page_tokens"]).unsqueeze(1)
    table.copy_(torch.where(mine & (table >= 0), goes[table.clamp(min=0).long()].to(torch.int32), table))
    s["k"].copy_(s["k"][:, takes])
    s["v"].copy_(s["v"][:, takes])
    return table, refs, live.view(1), s["k"], s["v"]


def _run_own(s, case):
    import paper_2605_03884_amd as qkv
    op, pages, status = case["op"], s["pages"], s["status"]
    if op == "attend":
        prior = (s["prior_out"], s["prior_lse"]) if case["prior"] else None
        return qkv.paged_attend(pages, s["q"], case["head_dim"] ** -0.5, s["out"], s["lse"], window=case["window"], sinks=case["sinks"],
                                prior=prior, workspace=s["workspace"], status=status)
    if op == "prompt":
        return qkv.paged_prompt(pages, s["q"], s["starts"], case["head_dim"] ** -0.5, s["out"], s["lse"], window=case["window"],
                                sinks=case["sinks"], workspace=s["workspace"], status=status)
    if op == "append":
        qkv.pages_append(pages, s["new_k"], s["new_v"], starts=s["starts"], status=status)
        return s["k"], s["v"]
    if op == "fork":
        qkv.pages_fork(pages, s["source"], s["target"], status)
        return s["table"], s["lens"], s["refs"], s["k"], s["v"]
    s["table"].copy_(s["first_table"])
    s["refs"].copy_(s["first_refs"])
    qkv.pages_compact(pages, status, live=s["live"], workspace=s["workspace"])
    return s["table"], s["refs"], s["live"], s["k"], s["v"]


def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"attend": _run_attend, "prompt": _run_prompt, "append": _run_append, "fork": _run_fork, "compact": _run_compact}[case["op"]](state, case)


def _seen_count(position, window, sinks):
    """How many tokens a query at `position` sees."""
    if position < 0:
        return 0
    if not window or position < window:
        return position + 1
    return window + min(sinks, position - window + 1)


def work(case):
    lens, new, pages, used = _plan(case)
    row = case["kv_heads"] * case["head_dim"] * 2 * 2                     # bytes of a token's keys and values in a layer
    op, size = case["op"], case["page_tokens"]
    if op == "attend":
        seen = sum(_seen_count(n - 1, case["window"], case["sinks"]) for n in lens)
        heads = len(lens) * case["q_heads"]
        answer = heads * (case["head_dim"] * 6 + 4) + (heads * (case["head_dim"] * 4 + 4) if case["prior"] else 0)
        return {"bytes": seen * row + answer, "flops": 4 * seen * case["q_heads"] * case["head_dim"]}
    if op == "prompt":
        seen = sum(_seen_count(p, case["window"], case["sinks"]) for n, count in zip(lens, new) for p in range(n - count, n))
        read = 0
        for n, count in zip(lens, new):
            first = n - count
            reach = min(first + 1, case["window"] + min(case["sinks"], max(0, first + 1 - case["window"]))) if case["window"] else first + 1
            read += reach + count - 1
        heads = sum(new) * case["q_heads"]
        return {"bytes": read * row + heads * (case["head_dim"] * 4 + 4), "flops": 4 * seen * case["q_heads"] * case["head_dim"]}
    if op == "append":
        return {"bytes": 2 * sum(new) * row * case["layers"], "flops": 0}
    if op == "fork":
        copied = sum(lens[i % case["parents"]] % size for i in range(case["children"]))
        shared = sum(lens[i % case["parents"]] // size for i in range(case["children"]))
        return {"bytes": 2 * copied * row * case["layers"] + 8 * shared + 4 * pages, "flops": 0}
    moved = used * (pages - used) / pages                                 # of pages in use at random places, those that lie too high
    return {"bytes": 2 * moved * size * row * case["layers"] + 8 * used + 8 * pages, "flops": 0}


def _exact_rows(s, case, row, positions, q):
    """One sequence's queries in 64 bits: q [n, q_heads, dim] at `positions`."""
    n, hq, dim = q.shape
    size, length = case["page_tokens"], int(s["lens"][row])
    heads = case["kv_heads"]
    rep = hq // heads
    out = torch.zeros(n, hq, dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
    if not length or not n:
        return out, lse
    numbers = s["table"][row, : _pages_of(length, size)].long()
    t = torch.arange(length, device="cuda")
    for h in range(heads):
        k = s["k"][0, numbers, h].reshape(-1, dim)[:length].double()
        v = s["v"][0, numbers, h].reshape(-1, dim)[:length].double()
        for r in range(rep):
            for lo in range(0, n, 2048):
                p = positions[lo:lo + 2048, None]
                hidden = t[None] > p
                if case["window"]:
                    hidden |= (t[None] <= p - case["window"]) & (t[None] >= case["sinks"])
                e = (q[lo:lo + 2048, h * rep + r].double() @ k.T) / math.sqrt(dim)
                e[hidden] = -math.inf
                lse[lo:lo + 2048, h * rep + r] = torch.logsumexp(e, 1)
                out[lo:lo + 2048, h * rep + r] = torch.softmax(e, 1).nan_to_num(0.0) @ v
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    op, size = case["op"], case["page_tokens"]
    lens, new, _, _ = _plan(case)
    if op in ("attend", "prompt"):
        outs, lses, at = [], [], 0
        for row, n in enumerate(lens):
            count = 1 if op == "attend" else new[row]
            o, l = _exact_rows(s, case, row, torch.arange(n - count, n, device="cuda"), s["q"][at:at + count])
            outs.append(o)
            lses.append(l)
            at += count
        out, lse = torch.cat(outs), torch.cat(lses)
        if op == "attend" and case["prior"]:
            a, b = lse, s["prior_lse"].double()
            top = torch.maximum(a, b)
            wa, wb = torch.exp(a - top), torch.exp(b - top)
            out = (out * wa[..., None] + s["prior_out"].double() * wb[..., None]) / (wa + wb)[..., None]
            lse = top + torch.log(wa + wb)
        return out, lse
    table = s["table"].tolist()
    if op == "append":
        at = 0
        for row, n in enumerate(lens):
            for first in range(n - new[row], n):
                if first % size and first != n - new[row]:
                    continue
                here = min(size - first % size, n - first)
                page = table[row][first // size]
                for pool, rows in ((s["k"], s["new_k"]), (s["v"], s["new_v"])):
                    pool[:, page, :, first % size:first % size + here] = rows[:, at:at + here].transpose(1, 2)
                at += here
        return s["k"], s["v"]                                             # copies: their own values are exact
    length, refs = s["lens"].tolist(), s["refs"].tolist()
    if op == "fork":
        pairs = list(zip(s["source"].tolist(), s["target"].tolist()))
        for _, b in pairs:
            for page in table[b][: _pages_of(length[b], size)]:
                refs[page] -= 1
        for a, _ in pairs:
            for page in table[a][: length[a] // size]:
                refs[page] += 1
        free = [i for i, r in enumerate(refs) if r == 0]
        for a, b in pairs:
            full, part = length[a] // size, length[a] % size
            table[b][:full] = table[a][:full]
            if part:
                page = free.pop(0)
                refs[page] = 1
                table[b][full] = page
                for pool in (s["k"], s["v"]):
                    pool[:, page, :, :part] = pool[:, table[a][full], :, :part]
            length[b] = length[a]
        return [torch.tensor(x, dtype=torch.int32) for x in (table, length, refs)] + [s["k"], s["v"]]
    live = sum(r > 0 for r in refs)
    holes = [i for i in range(live) if refs[i] == 0]
    movers = [i for i in range(live, len(refs)) if refs[i] > 0]
    goes = dict(zip(movers, holes))
    for a, b in goes.items():
        refs[a], refs[b] = 0, refs[a]
        for pool in (s["k"], s["v"]):
            pool[:, b] = pool[:, a]
    table = [[goes.get(p, p) if j < _pages_of(length[i], size) else p for j, p in enumerate(t)] for i, t in enumerate(table)]
    return [torch.tensor(x, dtype=torch.int32) for x in (table, refs, [live])] + [s["k"], s["v"]]
