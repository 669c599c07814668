"""What the GPU tests of the cache in pages share: a pool in a chosen layout with chosen contents, and the bounds results are held to."""
import numpy as np
import torch

import paper_2605_03884_amd as qkv

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Cache:
    """Pages [layers][pages, heads, size, dim] on the GPU, `lens` tokens in rows whose pages are drawn at random, and the same rows as a list of
    dense [heads, length, dim] arrays.  What no row holds is NaN or infinite.  layout: "heads" (a page's heads one after the other),
    "tokens" (a page's tokens one after the other, all heads of each) or "both" (keys and values of a page in one tensor, room behind each row)."""

    def __init__(self, lens, heads, dim, size, kind="fp16", layers=1, spare=3, extra_entries=1, layout="heads", seed=0, strong=4.0):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.size, self.kind = list(lens), size, kind
        held = [-(-n // size) for n in lens]
        pages, width = sum(held) + spare, max(held + [1]) + extra_entries
        order = torch.randperm(pages, generator=gen).to(torch.int32)
        self.table = torch.full((len(lens), width), 0x7FFFFFF0, dtype=torch.int32)        # behind a row's pages: nothing that is looked at
        at = 0
        for b, count in enumerate(held):
            self.table[b, :count] = order[at:at + count]
            at += count
        self.refs = torch.zeros(pages, dtype=torch.int32)
        self.refs[order[:at].long()] = 1
        dense = []
        for _ in range(2):
            x = torch.randn(layers, pages, heads, size, dim, generator=gen)
            x[..., : max(1, dim // 50)] *= strong
            dense.append(x.to(TYPES[kind]))
        used = torch.zeros(pages, size, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(held[b]):
                used[self.table[b, j], : max(0, min(size, n - j * size))] = True
        for i, x in enumerate(dense):
            x.permute(1, 3, 0, 2, 4)[~used] = (float("nan"), float("inf"))[i]
        self.k, self.v = dense
        self.layout = layout
        self.gpu()

    def rows(self, layer=0, poison=()):
        """[(K, V)] of every row, float64."""
        got = []
        for b, n in enumerate(self.lens):
            pages = self.table[b, : -(-n // self.size)].long()
            got.append(tuple(x[layer, pages].permute(1, 0, 2, 3).reshape(x.shape[2], -1, x.shape[4])[:, :n].double().numpy() for x in (self.k, self.v)))
        return got

    def gpu(self):
        layers, pages, heads, size, dim = self.k.shape
        made = []
        if self.layout == "both":
            wide = torch.full((layers, pages, 2, heads, size, dim + 8), float("nan"), dtype=self.k.dtype, device="cuda")
            made = [wide[:, :, i, :, :, :dim] for i in range(2)]
        else:
            for _ in range(2):
                made.append(torch.empty((layers, pages, heads, size, dim) if self.layout == "heads" else (layers, pages, size, heads, dim), dtype=self.k.dtype, device="cuda"))
                if self.layout == "tokens":
                    made[-1] = made[-1].transpose(2, 3)
        self.gk, self.gv = made
        self.gk.copy_(self.k)
        self.gv.copy_(self.v)
        self.gtable, self.glens, self.grefs = self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), self.refs.cuda()
        self.pages = qkv.Pages.make(list(self.gk), list(self.gv), self.gtable, self.glens, self.grefs)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


def score_bound(terms, top, dim):
    """How far a score may be off, in units of the exponent: products are exact in fp32, a sum of `dim` of them is off by at most dim 2^-24 times the sum of
    their sizes; the scale (rounded to fp32 as it is handed over, and once more with log2 e in it), the product with it and the maximum
    that is taken off round once each, relative to a score of at most `top`, and the difference once more."""
    return dim * 2.0 ** -24 * terms + 6 * 2.0 ** -24 * top + 2.0 ** -23


def check_attend(got, lse, want, dim, tokens):
    """out in fp32 with weights of 22 bits (2^-22): each weight is off by the factor e^(2 score bound) (its own and the sum's), the exponential is off by at most two
    steps (2^-22), fp32 sums of `tokens` terms by tokens 2^-24 relative to the sum of sizes (`size`); joining parts takes a handful of roundings more."""
    out, want_lse, size, terms, top = want
    s = score_bound(terms, top, dim)
    each = 2 * s + 2.0 ** -22 * 6 + (tokens + 16) * 2.0 ** -24
    err = np.abs(got - out)
    bound = each[..., None] * size + 2.0 ** -23 * np.abs(out)
    assert np.array_equal(np.isfinite(got), np.isfinite(out))
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-300)).max()
    if lse is not None:
        some = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(lse), ~some)
        assert (np.abs(lse[some] - want_lse[some]) <= s[some] + 2.0 ** -21 + tokens * 2.0 ** -24 + 2.0 ** -22 * np.abs(want_lse[some])).all()


def check_prompt(got, lse, want, dim, tokens, kind, most):
    """out in the pages' type: beside what check_attend counts, every weight is rounded to the type (half a step u, relative; fp16 below 2^-14: 2^-25 absolute, and a
    weight of 1 is 2^7 or more), and so is the result (u; fp16 subnormals: 2^-25).  `most`: the largest |V|."""
    out, want_lse, size, terms, top = want
    u = HALF_STEP[kind]
    s = score_bound(terms, top, dim)
    each = 2 * s + u + 2.0 ** -22 * 6 + (tokens + 16) * 2.0 ** -24
    tiny = (2.0 ** -25 + tokens * 2.0 ** -32 * most) if kind == "fp16" else 0.0
    err = np.abs(got - out)
    bound = (each[..., None] * size) * (1 + u) + u * np.abs(out) + tiny
    assert np.array_equal(np.isfinite(got), np.isfinite(out))
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-300)).max()
    if lse is not None:
        some = np.isfinite(want_lse)
        assert np.array_equal(np.isneginf(lse), ~some)
        assert (np.abs(lse[some] - want_lse[some]) <= s[some] + 2.0 ** -21 + tokens * 2.0 ** -24 + 2.0 ** -22 * np.abs(want_lse[some])).all()
