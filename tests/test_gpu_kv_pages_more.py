"""Compaction of sequences longer than their rows of the block table, and resizes either side of the rule
that chooses how many launches they take."""
import pytest
import torch

import test_gpu_kv_pages as pages_tests
from paper_2609_36608_amd import DecodeAttention
from test_gpu_kv_pages import Kept, i32

pytestmark = pytest.mark.gpu


def test_tokens_past_the_table():
    """They are on no page: nothing moves to or from them, and the others move as they would."""
    page, hkv, lens, new = 16, 2, [70, 40, 100], [30, 20, 60]
    kept = [[1, 4, 17, 18, 29], [0, 2, 19], [3, 8, 9, 30, 59]]
    c = Kept(3, lens, new, kept, page, hkv)
    width = 3  # 48 tokens
    want = []
    for x in (c.k, c.v):
        flat = x.view(torch.int16).clone().view(-1, hkv * 128)
        old = flat.clone()
        for b, (n, m, t) in enumerate(zip(lens, new, kept)):
            for i, s in enumerate(t):
                if n - m + s < width * page and n - m + i < width * page:
                    flat[c.row(b, n - m + i)] = old[c.row(b, n - m + s)]
        want.append(flat.view(x.shape))
    with DecodeAttention(hkv, hkv, 3, 4096, page_tokens=page) as attn:
        got = attn.compact_paged(c.k, c.v, i32(c.table[:, :width].copy()), i32(lens), i32(c.starts), i32(new), i32(c.keep),
                                 i32([len(t) for t in kept]))
    assert got.tolist() == [n - m + len(t) for n, m, t in zip(lens, new, kept)]
    assert torch.equal(c.k.view(torch.int16), want[0]) and torch.equal(c.v.view(torch.int16), want[1])


@pytest.mark.parametrize("seqs,width,pages", [(16, 256, 3000), (16, 257, 3000), (17, 256, 3000), (15, 200, 70001),
                                              (18, 200, 140003), (2, 3, 65537)])
def test_either_side_of_one_launch(seqs, width, pages):
    pages_tests.test_random_lives(seqs, width, 16, pages)
