"""The attention calls over paged caches with random batches in which everything meets: caps, slopes
of either sign, windows, prefixes, documents, padding rows anywhere, pages outside the cache, short
tables, rows of no sequence, and NaN or infinities in every slot that no query of its sequence sees."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import AttnScores, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, attention_reference, seen_tokens
from test_gpu_paged_prefill import F32, ROUNDED, SCALE, U, slopes_of

pytestmark = pytest.mark.gpu


def scores_of(rng, bt, rows):
    """What a call changes, each part by the toss of a coin, and each row's document."""
    kw = {}
    coin = lambda: rng.random() < 0.5  # noqa: E731
    if coin():
        kw["softcap"] = float(rng.choice([3.0, 30.0, 700.0]))
    if coin():
        kw["slopes"] = slopes_of(bt.hq) * float(rng.choice([1.0, -0.3, 0.05]))
    if coin():
        kw["window"] = int(np.exp(rng.uniform(0, 6)))
    if coin():
        kw["prefix"] = rng.integers(-3, 90, len(bt.lens))
    docs = np.zeros(rows, np.int64)
    if coin():
        kw["docs"] = docs
    return kw, docs


def hide(bt, kw, rng, per_row):
    """Puts NaN and infinities where no query of the sequence looks."""
    docs, prefix, window = kw.get("docs"), kw.get("prefix"), kw.get("window", 0)
    for b, (n, m) in enumerate(zip(bt.lens, bt.new)):
        # (slots of tokens past the table or on pages outside the cache are none)
        seen = torch.zeros(n, dtype=torch.bool)
        for i in range(m):
            doc = 0 if docs is None else int(docs[bt.starts[b] + i if per_row else b])
            seen |= seen_tokens(n, n - m + i, window, 0 if prefix is None else int(prefix[b]), doc)
        for t in torch.nonzero(~seen)[:, 0].tolist():
            slot = bt.slot(b, t)
            if slot is not None:
                bt.k[slot] = float(rng.choice([np.nan, np.inf, -np.inf]))
                bt.v[slot] = float(rng.choice([np.nan, np.inf, -np.inf]))


def batch(seed, decode):
    rng = np.random.default_rng(seed)
    hq, hkv = [(16, 8), (8, 2), (7, 7), (12, 2), (6, 2), (16, 1)][rng.integers(6)]
    page = int(rng.choice([16, 32, 48]))
    n = int(rng.integers(1, 12))
    lens = rng.integers(0, int(np.exp(rng.uniform(3, 6.5))), n)
    if decode:
        new = np.ones(n, int)
        bt = Batch(seed, lens, new, page, hq, hkv)
        bt.starts, bt.rows = np.arange(n, dtype=np.int32), n
        bt.q = bt.q[:n].clone()
    else:
        new = np.array([rng.integers(0, x + 1) for x in lens])
        if rng.random() < 0.3:
            new = np.minimum(new, 3)
        bt = Batch(seed, lens, new, page, hq, hkv, gap=int(rng.integers(0, 3)))
    kw, docs = scores_of(rng, bt, n if decode else bt.rows)
    if "docs" in kw:
        for b, (length, m) in enumerate(zip(bt.lens, bt.new)):
            first = 0
            for i in range(m):
                p = length - m + i
                if rng.random() < 0.05:
                    first = int(rng.integers(0, p + 1)) if p >= 0 else 0
                pad = rng.random() < 0.1
                docs[b if decode else bt.starts[b] + i] = p + 1 + int(rng.integers(0, 9)) if pad else first
    hide(bt, kw, rng, not decode)
    for b in range(n):  # after it: what lies on these pages is not seen either
        if rng.random() < 0.3 and bt.lens[b] > 0:
            bt.table[b, rng.integers(0, -(-bt.lens[b] // page))] = rng.choice([-1, bt.num_pages, 2 ** 31 - 1, -2 ** 31])
    if rng.random() < 0.2:
        bt.table = np.ascontiguousarray(bt.table[:, :max(1, bt.table.shape[1] // 2)])
    bound = int(max(max(bt.lens), 1) if rng.random() < 0.5 else rng.choice([4096, 32768]))
    return bt, kw, bound


def call(bt, kw, bound, out_dtype, decode, split_p=False):
    out = torch.full((bt.rows, bt.hq, D), -777.0, dtype=out_dtype, device=dev())
    up = lambda t: None if t is None else up_i32(t)  # noqa: E731
    slopes = kw.get("slopes")
    sc = AttnScores(kw.get("softcap", 0.0), kw.get("window", 0), None if slopes is None else slopes.to(dev()),
                    up(kw.get("prefix")), up(kw.get("docs")), split_p=split_p)
    args = [t.to(dev()) for t in (bt.q, bt.k, bt.v)] + [up_i32(bt.table), up_i32(bt.lens)]
    with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), bound, page_tokens=bt.page, out_dtype=out_dtype) as attn:
        if decode:
            attn.run_paged(*args, SCALE, out, scores=sc)
        else:
            attn.prefill_paged(*args, up_i32(bt.starts), up_i32(bt.new), max(max(bt.new), 1), SCALE, out, scores=sc)
        torch.cuda.synchronize()
    return out.cpu()


def reference(bt, kw, decode):
    """The plain form, whose own values in unseen slots are zeros."""
    kept = bt.k, bt.v
    bt.k, bt.v = (t.nan_to_num(0.0, 0.0, 0.0) for t in kept)
    kw = dict(kw)
    if "prefix" in kw:
        kw["prefix"] = [min(max(int(x), 0), max(n, 0)) for x, n in zip(kw["prefix"], bt.lens)]
    if decode:
        lens = bt.lens
        bt.new = [1 if n > 0 else 0 for n in lens]
    ref, spread = attention_reference(bt, SCALE, spread=True, per_row=not decode, **kw)
    if decode:
        ref[torch.tensor([n <= 0 for n in bt.lens])] = 0
        spread[torch.tensor([n <= 0 for n in bt.lens])] = 0
    bt.k, bt.v = kept
    return ref, spread


def within(got, ref, spread, rounded, bf16):
    bound = F32 + rounded * (spread + (ref.abs() if rounded == U * U else 0))
    if bf16:
        bound = bound + U * (ref.abs() + bound)
    worst = ((got.double() - ref).abs() - bound).max().item()
    assert worst <= 0, f"worst excess {worst:.3e}"


@pytest.mark.parametrize("seed", range(40))
def test_prefill(seed):
    bt, kw, bound = batch(seed, False)
    live = torch.tensor([at is not None for at in bt.row_of()])
    ref, spread = reference(bt, kw, False)
    for out_dtype, split_p in ((torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)):
        got = call(bt, kw, bound, out_dtype, False, split_p)
        assert (got[~live] == -777.0).all()
        if live.any():
            assert got[live].isfinite().all()
            rounded = 0.0 if out_dtype == torch.float32 else U * U if split_p else ROUNDED
            within(got[live], ref[live], spread[live], rounded, out_dtype == torch.bfloat16)


@pytest.mark.parametrize("seed", range(100, 130))
def test_decode(seed):
    bt, kw, bound = batch(seed, True)
    ref, spread = reference(bt, kw, True)
    for out_dtype in (torch.float32, torch.bfloat16):
        got = call(bt, kw, bound, out_dtype, True)
        assert got.isfinite().all()
        within(got, ref, spread, U * U if out_dtype == torch.bfloat16 else 0.0, out_dtype == torch.bfloat16)
