"""Plain 64-bit forms of the operators over paged caches, on the CPU, and the
batches that their tests share."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128


def bf16(t):
    return t.to(torch.bfloat16)


def randn(g, shape, std=1.0):
    return bf16(torch.randn(shape, generator=g) * std)


class Batch:
    """Packed rows over shuffled pages: sequence b holds lens[b] tokens of which the last new[b] are
    rows starts[b] .. of `rows`; the rows are in a shuffled order of sequences with gaps between them.
    Unused table entries are -1, unused slots of the caches NaN."""

    def __init__(self, seed, lens, new, page, hq, hkv, gap=0, spare=3):
        g = self.g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.new, self.page, self.hq, self.hkv = list(lens), list(new), page, hq, hkv
        n = len(self.lens)
        pages = [-(-max(x, 0) // page) for x in self.lens]
        order = rng.permutation(sum(pages) + spare)
        self.num_pages = len(order)
        self.table = np.full((n, max(pages) + 2), -1, np.int32)
        at = 0
        for b, m in enumerate(pages):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.starts = np.zeros(n, np.int32)
        row = gap
        for b in rng.permutation(n):
            self.starts[b] = row
            row += self.new[b] + gap
        self.rows = max(row, 1)
        self.k = torch.full((self.num_pages, page, hkv, D), float("nan"), dtype=torch.bfloat16)
        self.v = self.k.clone()
        for b in range(n):
            for t in range(max(self.lens[b], 0)):
                p, s = self.table[b, t // page], t % page
                self.k[p, s] = randn(g, (hkv, D))
                self.v[p, s] = randn(g, (hkv, D))
        self.q = randn(g, (self.rows, hq, D))

    def slot(self, b, t):
        """Page and place of a token, None where the table names no page of the cache."""
        j = t // self.page
        if j >= self.table.shape[1] or not 0 <= self.table[b, j] < self.num_pages:
            return None
        return int(self.table[b, j]), t % self.page

    def row_of(self):
        """(sequence, position) of every packed row, None where a row is no sequence's."""
        where = [None] * self.rows
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            for i in range(m):
                where[self.starts[b] + i] = (b, n - m + i)
        return where


def rotated(x, pos, inv_freq, interleaved):
    """x [..., D] in 64 bits, rotated to position pos."""
    x = x.double().clone()
    n = len(inv_freq)
    if n == 0:
        return x
    u = torch.tensor([math.fmod(float(pos) * float(f), 2 * math.pi) for f in inv_freq], dtype=torch.float64)
    cos, sin = torch.cos(u), torch.sin(u)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, c = x[..., first].clone(), x[..., second].clone()
    x[..., first] = a * cos - c * sin
    x[..., second] = c * cos + a * sin
    return x


def normed(x, weight, eps):
    x = x.double()
    if weight is None:
        return x
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()


def append_reference(bt: Batch, q, k, v, inv_freq, interleaved=False, positions=None, q_norm=None, k_norm=None,
                     eps=1e-6):
    """q_out and caches (64 bits), the same with the sizes that went into each value (for the error bound)."""
    kc, vc, qo = bt.k.double(), bt.v.double(), torch.full((bt.rows, bt.hq, D), float("nan"), dtype=torch.float64)
    ks, qs = torch.zeros_like(kc), torch.zeros_like(qo)
    for j, at in enumerate(bt.row_of()):
        if at is None:
            continue
        b, p = at
        pos = p if positions is None else int(positions[j])

        def both(x, w):
            x = normed(x, w, eps)
            size = rotated(torch.ones_like(x), 0, [], False) * 0
            n = len(inv_freq)
            size += x.abs()
            if n:
                f, s = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
                total = x[..., f].abs() + x[..., s].abs()
                size[..., f] = total
                size[..., s] = total
            return rotated(x, pos, inv_freq, interleaved), size

        if q is not None:
            qo[j], qs[j] = both(q[j], q_norm)
        slot = bt.slot(b, p)
        if slot is not None:
            kc[slot], ks[slot] = both(k[j], k_norm)
            vc[slot] = v[j].double()
    return qo, kc, vc, qs, ks


def seen_tokens(length, p, window=0, prefix=0, doc=0):
    """Tokens that a query at position p sees, as a boolean vector."""
    t = torch.arange(max(length, 0))
    low = max(doc, p - window + 1 if window else 0)
    return (t < prefix) | ((t >= low) & (t <= p))


def attention_reference(bt: Batch, scale, softcap=0.0, window=0, slopes=None, prefix=None, docs=None, per_row=True,
                        spread=False):
    """Outputs [rows, Hq, D] in 64 bits (NaN in rows of no sequence) of every packed row against bt's
    caches; docs per packed row, or per sequence (per_row False).  spread: also the weighted mean of
    |value - output|, which bounds what a relative error of the weights does to the output."""
    out = torch.full((bt.rows, bt.hq, D), float("nan"), dtype=torch.float64)
    wide = torch.zeros_like(out)
    g = bt.hq // bt.hkv
    cache = {}
    for j, at in enumerate(bt.row_of()):
        if at is None:
            continue
        b, p = at
        n = max(bt.lens[b], 0)
        if b not in cache:
            kb, vb = torch.zeros((n, bt.hkv, D), dtype=torch.float64), torch.zeros((n, bt.hkv, D), dtype=torch.float64)
            there = torch.zeros(n, dtype=torch.bool)
            for t in range(n):
                slot = bt.slot(b, t)
                if slot is not None:
                    kb[t], vb[t], there[t] = bt.k[slot].double(), bt.v[slot].double(), True
            cache[b] = kb, vb, there
        kb, vb, there = cache[b]
        doc = 0 if docs is None else int(docs[j if per_row else b])
        see = seen_tokens(n, p, window, 0 if prefix is None else int(prefix[b]), doc) & there
        out[j] = 0
        if not see.any():
            continue
        t = torch.nonzero(see)[:, 0]
        s = torch.einsum("hgd,thd->hgt", bt.q[j].double().view(bt.hkv, g, D), kb[t]) * scale
        if softcap:
            s = softcap * torch.tanh(s / softcap)
        if slopes is not None:
            s = s - slopes.double().view(bt.hkv, g, 1) * (p - t).abs().double()
        w = torch.softmax(s, -1)
        o = torch.einsum("hgt,thd->hgd", w, vb[t])
        out[j] = o.reshape(bt.hq, D)
        if spread:
            far = (vb[t].permute(1, 0, 2)[:, None] - o[:, :, None]).abs()
            wide[j] = (w[..., None] * far).sum(2).reshape(bt.hq, D)
    return (out, wide) if spread else out
