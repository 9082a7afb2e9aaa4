"""More of ctx_kv_append_run_paged: lengths below zero, the kernels of many rows in every form, with
the large calls that pass the caches by, and batches whose rows do not fit their sequences."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import DecodeAttention, Rotary

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, randn
from test_gpu_paged_append import bits, close, inv_freq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
def test_a_length_below_zero_counts_as_zero(packed):
    """The lowest length too, whose newest position would wrap round to the highest."""
    bt = Batch(43, [0, 0, 0, 20], [0, 0, 0, 1], 16, 8, 2)
    lens = [-2 ** 31, -1, 0, 20]
    bt.table[:3] = 0  # pages that would take a token
    q, k, v = (randn(bt.g, (4, h, D)).to(dev()) for h in (8, 2, 2))
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    out = torch.full((4, 8, D), -777.0, dtype=torch.bfloat16, device=dev())
    rows = dict(q_starts=up_i32([0, 1, 2, 3]), q_lens=up_i32([1, 1, 1, 1])) if packed else {}
    with DecodeAttention(8, 2, 4, 32, page_tokens=16) as attn:
        attn.append_paged(k, v, kc, vc, up_i32(bt.table), up_i32(lens), q=q, q_out=out,
                          rotary=Rotary(inv_freq(128).to(dev())), **rows)
        torch.cuda.synchronize()
    assert (out[:3] == -777.0).all() and (out[3] != -777.0).all()
    page, at = bt.slot(3, 19)
    changed = np.zeros((bt.num_pages, 16), bool)
    changed[page, at] = True
    for new, old in ((kc.cpu(), bt.k), (vc.cpu(), bt.v)):
        assert torch.equal(bits(new[~changed]), bits(old[~changed]))
    assert torch.equal(bits(vc.cpu()[page, at]), bits(v[3].cpu()))


class Rows:
    """Packed rows of a fused projection on the device: `seqs` sequences of `new` tokens each over
    `hist` ones, in order and with `gap` rows of no sequence behind each; the caches hold a pattern."""

    def __init__(self, seed, seqs, new, hist, page, hq, hkv, gap, width=0):
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.page, self.hq, self.hkv = page, hq, hkv
        self.rows = seqs * (new + gap)
        used = -(-(new + hist) // page)
        self.pages = seqs * used + 2
        self.table = torch.randperm(self.pages, generator=g, device=dev()).to(torch.int32)[:seqs * used].view(seqs, used)
        self.lens, self.starts, self.new = (torch.tensor(x, dtype=torch.int32, device=dev()) for x in (
            [new + hist] * seqs, [b * (new + gap) for b in range(seqs)], [new] * seqs))
        x = torch.randn((self.rows, (hq + 2 * hkv) * D + width), generator=g, device=dev()) * 2
        self.x = x.to(torch.bfloat16)
        self.q, self.k, self.v = self.x[:, :(hq + 2 * hkv) * D].unflatten(1, (-1, D)).split([hq, hkv, hkv], 1)
        shape = (self.pages, page, hkv, D)
        self.kc, self.vc = (torch.full(shape, float(i), dtype=torch.bfloat16, device=dev()) for i in (321, 123))
        row = torch.arange(self.rows, device=dev())
        self.seq, i = row // (new + gap), row % (new + gap)
        self.live = i < new
        self.p = hist + i
        page_of = self.table.long()[self.seq, (self.p // page).clamp(max=used - 1)]
        self.slot = (page_of * page + self.p % page)[self.live]

    def both(self, x, weight, f, pos, interleaved, eps):
        """Normed and rotated in 64 bits, and the sizes that went into each value."""
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
        y, size, n = x.clone(), x.abs(), len(f)
        if n:
            u = pos.double()[:, None, None] * f.double()
            a, c = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
            y[..., a] = x[..., a] * u.cos() - x[..., c] * u.sin()
            y[..., c] = x[..., c] * u.cos() + x[..., a] * u.sin()
            size[..., a] = size[..., c] = x[..., a].abs() + x[..., c].abs()
        return y, size

    def check(self, rot=128, interleaved=False, norm="both", positions=False, queries=True, eps=1e-6):
        g = torch.Generator(device=dev()).manual_seed(rot)
        w = [(1 + 0.2 * torch.randn(D, generator=g, device=dev())).to(torch.bfloat16) for _ in range(2)]
        q_norm, k_norm = (w[i] if norm in ("both", "qk"[i]) else None for i in range(2))
        pos = torch.randint(0, 1 << 20, (self.rows,), generator=g, device=dev(), dtype=torch.int32) if positions else None
        f = inv_freq(rot).to(dev())
        out = torch.full((self.rows, self.hq, D), -777.0, dtype=torch.bfloat16, device=dev()) if queries else None
        with DecodeAttention(self.hq, self.hkv, len(self.lens), int(self.lens.max()), page_tokens=self.page) as attn:
            attn.append_paged(self.k, self.v, self.kc, self.vc, self.table, self.lens, q=self.q if queries else None,
                              q_out=out, q_starts=self.starts, q_lens=self.new,
                              rotary=Rotary(f if rot else None, interleaved, pos, q_norm, k_norm, eps))
            torch.cuda.synchronize()
        at = (self.p if pos is None else pos)[self.live]
        if queries:
            close(out[self.live], *self.both(self.q[self.live], q_norm, f, at, interleaved, eps))
            assert (out[~self.live] == -777.0).all()
        k, v = (t.view(-1, self.hkv, D) for t in (self.kc, self.vc))
        close(k[self.slot], *self.both(self.k[self.live], k_norm, f, at, interleaved, eps))
        assert torch.equal(bits(v[self.slot]), bits(self.v[self.live]))
        rest = torch.ones(len(k), dtype=torch.bool, device=dev())
        rest[self.slot] = False
        assert rest.any() and (k[rest] == 321).all() and (v[rest] == 123).all()


def cus():
    return torch.cuda.get_device_properties(dev()).multi_processor_count


@pytest.mark.parametrize("norm", ["none", "q", "both"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot,positions", [(128, False), (64, True), (16, False), (0, False)])
def test_a_row_per_wave(norm, interleaved, rot, positions):
    """From 11 rows per CU on: slices of one projection, in every form."""
    r = Rows(rot + len(norm), 24, 125, 37, 16, 6, 2, gap=3, width=8)
    assert 11 * cus() <= r.rows and r.rows * (6 + 2 * 2) * D * 4 <= 256 << 20
    r.check(rot, interleaved, norm, positions)


def test_a_row_per_wave_without_queries():
    r = Rows(5, 3, 1030, 0, 48, 7, 7, gap=1)
    assert 11 * cus() <= r.rows
    r.check(96, queries=False)


@pytest.mark.parametrize("norm,interleaved,rot,positions", [
    ("both", False, 128, False), ("none", True, 64, True), ("k", True, 128, False), ("none", False, 0, False),
    ("q", False, 32, True)])
def test_calls_larger_than_the_last_level_cache(norm, interleaved, rot, positions):
    """More than 256 MiB read and written: reads and writes past the caches."""
    r = Rows(7, 9, 1300, 211, 16, 32, 8, gap=2)
    assert r.rows * (32 + 2 * 8) * D * 4 > 256 << 20
    r.check(rot, interleaved, norm, positions)


def test_rows_that_do_not_fit_their_sequences_touch_nothing_else():
    """More new tokens than tokens, and rows past the arrays: rows before position 0, everything past
    the arrays and every slot that no row has a position for stay as they were."""
    bt = Batch(31, [3, 20], [3, 20], 16, 8, 2)
    lens, starts, new = [3, 20], [0, 15], [10, 100]
    n = bt.rows
    q, k, v = (randn(bt.g, (n, h, D)).to(dev()) for h in (8, 2, 2))
    # the arrays lie within larger ones
    buf = torch.full((n + 128, 8, D), -777.0, dtype=torch.bfloat16, device=dev())
    out = buf[64:64 + n]
    wide = [torch.full((bt.num_pages + 8, 16, 2, D), -777.0, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    for w, old in zip(wide, (bt.k, bt.v)):
        w[4:4 + bt.num_pages] = old.to(dev())
    before = [w.clone() for w in wide]
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        attn.append_paged(k, v, wide[0][4:-4], wide[1][4:-4], up_i32(bt.table), up_i32(lens), q=q, q_out=out,
                          q_starts=up_i32(starts), q_lens=up_i32(new))
        torch.cuda.synchronize()
    took = {}  # row: its slot
    for b in range(2):
        for i in range(new[b]):
            p = lens[b] - new[b] + i
            if p >= 0 and starts[b] + i < n:
                took[starts[b] + i] = bt.slot(b, p)
    assert sorted(took) == [7, 8, 9]
    rows = torch.tensor([64 + j for j in took], device=dev())
    assert torch.equal(bits(buf[rows]), bits(q[rows - 64]))
    keep = torch.ones(len(buf), dtype=torch.bool, device=dev())
    keep[rows] = False
    assert (buf[keep] == -777.0).all()
    for w, old, x in zip(wide, before, (k, v)):
        for j, (page, at) in took.items():
            assert torch.equal(bits(w[4 + page, at]), bits(x[j]))
            old[4 + page, at] = x[j]
        assert torch.equal(bits(w), bits(old))
