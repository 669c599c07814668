"""What the GPU tests of attention over chosen pages share: choices as sets and as words, and what a choice makes of the definition in 64 bits."""
import numpy as np
import torch

from oracle import chosen_ref, paged_ref


def draw_choices(cache, places, heads, share, seed):
    """A set of page numbers of its sequence for every query token and kv head, a `share` of all there is room for: pages behind a query's own among them."""
    gen = np.random.default_rng(seed)
    width = cache.table.shape[1]
    return [[set(np.flatnonzero(gen.random(width) < share).tolist()) for _ in range(heads)] for _ in places]


def as_words(choices, row_pages):
    got = np.stack([np.stack([chosen_ref.words(c, row_pages) for c in token]) for token in choices])
    return torch.from_numpy(got.view(np.int32)).cuda()


def as_sets(words, row_pages):
    w = words.cpu().numpy().view(np.uint32)
    bits = (w[..., None] >> np.arange(32, dtype=np.uint32)) & 1
    bits = bits.reshape(w.shape[0], w.shape[1], -1)
    assert not bits[..., row_pages:].any()
    return [[set(np.flatnonzero(h).tolist()) for h in token] for token in bits]


def expected(cache, q, rows, places, choices, scale, layer=0, lost=()):
    """Attention of queries q [n, Hq, D] (float64) of sequence rows[i] at places[i] over choices[i][kv head]; `lost`: (row, page of the sequence) without a page."""
    dense = cache.rows(layer)
    n, Hq, D = q.shape
    heads = len(choices[0])
    rep = Hq // heads
    parts = [np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, D)), np.zeros((n, Hq)), np.zeros((n, Hq))]
    for i in range(n):
        K, V = dense[rows[i]]
        for h in range(heads):
            some = slice(h * rep, (h + 1) * rep)
            tokens = [t for j in sorted(choices[i][h]) if (rows[i], j) not in lost for t in range(j * cache.size, (j + 1) * cache.size) if t <= places[i]]
            if not tokens:
                continue
            got = paged_ref.attend(q[i:i + 1, some], K[h:h + 1][:, tokens], V[h:h + 1][:, tokens], [len(tokens) - 1], scale)
            for part, x in zip(parts, got):
                part[i:i + 1, some] = x
    return parts


def ragged(cache, new):
    """Rows and places of the query tokens of a ragged batch, and its starts."""
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = [b for b, n in enumerate(new) for _ in range(n)]
    places = [cache.lens[b] - n + i for b, n in enumerate(new) for i in range(n)]
    return rows, places, torch.from_numpy(starts).cuda()
