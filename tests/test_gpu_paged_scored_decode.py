"""ctx_decode_attn_run_paged_scored against a plain 64-bit form: caps, biases,
windows, prefixes and documents over shuffled pages, rows that see nothing, and
slots that no query sees."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd import binding as bd
from paper_2609_36608_amd.binding import AttnScores, CtxError, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, attention_reference, randn

pytestmark = pytest.mark.gpu

SCALE = D ** -0.5

# fp32 outputs.  A logit is a sum of 128 exact products in fp32 (at most 2^-24 of the sum of
# their sizes each step; the sizes here sum to about 128 * 0.64 * scale = 7, 30 with queries of
# 4 times the size), a product with the scale or a tanh (2^-23) and a bias (2^-24 of some tens):
# below 30 * 2^-21 = 1.5e-5 in the worst case.  A weight is off by that share, its exponential by
# 2^-22; the weights' three bf16 terms and the sums of some thousand products add 2^-20.  The
# output is a convex combination of values of up to 4.5: below 4.5 * 2e-5 = 9e-5.  Half a step
# of bf16 more for bf16 outputs; two bf16 terms of a weight there, 2^-17 of it.
F32 = 9e-5


def close(got, ref, out_dtype):
    assert got.isfinite().all()
    err = (got.double() - ref).abs()
    bound = F32 + (2.0 ** -8 * (ref.abs() + F32) if out_dtype == torch.bfloat16 else 0)
    assert (err <= bound).all(), f"worst {err.max().item():.3e}"


def batch(seed, lens, page=16, hq=16, hkv=8, qstd=1.0):
    bt = Batch(seed, lens, [1] * len(lens), page, hq, hkv)
    bt.starts = np.arange(len(lens), dtype=np.int32)
    bt.q = randn(bt.g, (len(lens), hq, D), qstd)
    bt.rows = len(lens)
    return bt


def run(bt, softcap=0.0, window=0, slopes=None, prefix=None, docs=None, out_dtype=torch.float32, split=0, scale=SCALE,
        max_seq_len=None):
    up = lambda t: None if t is None else t.to(dev())  # noqa: E731
    i32 = lambda t: None if t is None else up_i32(t)  # noqa: E731
    n = len(bt.lens)
    buf = torch.full((n + 1, bt.hq, D), -777.0, dtype=out_dtype, device=dev())
    kc, vc = up(bt.k), up(bt.v)
    with DecodeAttention(bt.hq, bt.hkv, n, max_seq_len or max(max(bt.lens), 1), page_tokens=bt.page,
                         out_dtype=out_dtype, split_tokens=split) as attn:
        attn.run_paged(up(bt.q), kc, vc, up_i32(bt.table), up_i32(bt.lens), scale, buf[:n],
                       scores=AttnScores(softcap, window, up(slopes), i32(prefix), i32(docs)))
        torch.cuda.synchronize()
    assert (buf[n] == -777.0).all()
    assert torch.equal(kc.cpu().view(torch.int16), bt.k.view(torch.int16))
    return buf[:n].cpu()


def check(bt, out_dtype=torch.float32, split=0, scale=SCALE, max_seq_len=None, **kw):
    got = run(bt, out_dtype=out_dtype, split=split, scale=scale, max_seq_len=max_seq_len, **kw)
    ref = attention_reference(bt, scale, per_row=False, **kw)
    close(got, ref, out_dtype)
    return got


def slopes_of(hq):
    return 2.0 ** (-8.0 * torch.arange(1, hq + 1, dtype=torch.float32) / hq)


LENS = [1, 2, 15, 16, 17, 31, 33, 64, 100, 257, 0, 600]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("split", [0, 16, 48])
@pytest.mark.parametrize("kind", ["none", "cap", "bias", "window", "prefix", "docs", "all"])
def test_scores_and_masks(kind, split, out_dtype):
    bt = batch(3, LENS, qstd=4.0 if kind == "cap" else 1.0)
    rng = np.random.default_rng(4)
    every = kind == "all"
    kw = {}
    if kind == "cap" or every:
        kw["softcap"] = 5.0
    if kind == "bias" or every:
        kw["slopes"] = slopes_of(bt.hq)
    if kind == "window" or every:
        kw["window"] = 37
    if kind == "prefix" or every:
        kw["prefix"] = rng.integers(0, 40, len(LENS))
    if kind == "docs" or every:
        kw["docs"] = np.array([rng.integers(0, n + 1) for n in LENS])
    check(bt, out_dtype, split, **kw)


@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4), (16, 1), (5, 1), (9, 3), (7, 7), (30, 10), (1, 1)])
@pytest.mark.parametrize("page", [16, 48, 64])
def test_heads_and_pages(hq, hkv, page):
    bt = batch(hq + page, [1, page, page + 1, 3 * page + 7, 200], page, hq, hkv)
    check(bt, softcap=20.0, window=90, slopes=slopes_of(hq), prefix=[0, 3, page, 17, 40])


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 32, 33, 1000])
def test_window_edges(window):
    check(batch(window, LENS), window=window)


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 100, 10 ** 6, -5])
def test_prefix_edges(prefix):
    bt = batch(prefix & 255, LENS)
    got = run(bt, window=8, prefix=[prefix] * len(LENS))
    close(got, attention_reference(bt, SCALE, window=8, prefix=[min(max(prefix, 0), n) for n in LENS], per_row=False),
          torch.float32)


def test_rows_that_see_nothing_or_their_prefix_alone():
    bt = batch(11, [40, 40, 40, 16, 1, 300])
    docs = [40, 2 ** 31 - 1, 41, 16, 1, 300]
    got = check(bt, docs=docs)
    assert (got == 0).all()
    got = check(bt, docs=docs, prefix=[0, 5, 16, 17, 0, 33], slopes=slopes_of(16) * 50)
    assert (got[0] == 0).all() and (got[4] == 0).all() and (got[1] != 0).any()
    check(bt, docs=[-3, 39, 0, 15, 0, 256])


def test_unseen_slots_may_hold_anything():
    """NaN and infinities in tokens that the masks hide, whole blocks of them and within a block."""
    bt = batch(13, [200, 70, 35])
    docs = [150, 0, 20]
    prefix = [21, 3, 0]
    clean = run(bt, docs=docs, prefix=prefix, window=40)
    for b, n in enumerate(bt.lens):
        low = max(docs[b], n - 40)
        for t in range(prefix[b], low):
            for cache, bad in ((bt.k, float("nan")), (bt.v, float("inf") if t % 2 else float("nan"))):
                cache[bt.slot(b, t)] = bad
    assert torch.equal(run(bt, docs=docs, prefix=prefix, window=40), clean)


def test_pages_outside_the_cache_are_not_seen():
    bt = batch(17, [200, 100, 90, 33])
    bt.table[0, 3] = -1
    bt.table[0, 12] = bt.num_pages
    bt.table[1, :] = 2 ** 31 - 1  # nothing left
    bt.table = np.ascontiguousarray(bt.table[:, :13])
    bt.table[2, 0] = -2 ** 31
    got = check(bt, softcap=30.0)
    assert (got[1] == 0).all()
    check(bt, split=16, window=150)
    bt.table = np.ascontiguousarray(bt.table[:, :2])  # tokens past the table
    bt.table[2, 0] = bt.table[2, 1]
    check(bt)
    check(bt, window=80, slopes=slopes_of(16))  # the window counts from the newest token
    check(bt, window=30, prefix=[5, 0, 17, 33])


def test_large_logits_and_a_zero_scale():
    bt = batch(19, [300, 40], qstd=1.0)
    bt.q[0] *= 64  # logits of hundreds: one token has all the weight
    got = run(bt, softcap=0.0)
    ref = attention_reference(bt, SCALE, per_row=False)
    # the largest logits, about 64 * 4, are off by up to 64 times the share above
    assert ((got.double() - ref).abs() <= 64 * F32).all()
    check(bt, softcap=2.0)
    check(bt, scale=0.0, softcap=2.0)
    check(bt, scale=0.0)
    check(bt, scale=-SCALE, softcap=3.0)
    bt.k[~bt.k.isnan()] *= 2.0 ** 60  # every score at its cap
    bt.k = bt.k.clone()
    check(bt, softcap=1.0)


def test_biases_far_away_and_of_the_other_sign():
    bt = batch(23, [500, 3])
    check(bt, slopes=torch.full((16,), -0.5))
    check(bt, slopes=torch.zeros(16))
    # only far tokens are seen: logits of hundreds whose differences count
    check(bt, slopes=torch.full((16,), 2.0), prefix=[30, 1], docs=[500, 3])


def test_many_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 120, 300)
    bt = batch(29, lens, hq=8, hkv=2)
    for split in (0, 32):
        check(bt, split=split, window=50, prefix=rng.integers(0, 30, 300), max_seq_len=128)


def test_none_of_the_scores_is_the_plain_step():
    bt = batch(31, [5, 700, 64])
    lens = up_i32(bt.lens)
    q, kc, vc, table = bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table)
    with DecodeAttention(16, 8, 3, 700, page_tokens=16, out_dtype=torch.bfloat16) as attn:
        a = attn.run_paged(q, kc, vc, table, lens, SCALE, torch.empty_like(q))
        b = attn.run_paged(q, kc, vc, table, lens, SCALE, torch.empty_like(q), scores=AttnScores())
        torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_refusals():
    bt = batch(37, [20, 5], hq=8, hkv=2)
    q, kc, vc = bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev())
    table, lens, out = up_i32(bt.table), up_i32(bt.lens), torch.empty((2, 8, D), device=dev())
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        call = lambda sc, **kw: attn.run_paged(q, kc, vc, table, lens, SCALE, out, scores=sc, **kw)  # noqa: E731
        call(AttnScores(softcap=1.0))
        for sc, status in ((AttnScores(softcap=-1.0), bd.CTX_ERR_INVALID_ARG),
                           (AttnScores(softcap=float("inf")), bd.CTX_ERR_INVALID_ARG),
                           (AttnScores(softcap=1e-45), bd.CTX_ERR_INVALID_ARG),
                           (AttnScores(window=-1), bd.CTX_ERR_INVALID_ARG)):
            with pytest.raises(CtxError) as e:
                call(sc)
            assert e.value.status == status
        with pytest.raises(ValueError):
            call(AttnScores(slopes=torch.ones(2, device=dev())))
        with pytest.raises(TypeError):
            call(AttnScores(prefix_lens=lens.long()))
        with pytest.raises(ValueError):
            call(AttnScores(doc_starts=lens.cpu()))
        with pytest.raises(ValueError):
            call(AttnScores(), k_new=kc[0, :2].contiguous(), v_new=vc[0, :2].contiguous())
        torch.cuda.synchronize()


def test_graph_replays_and_another_stream():
    from test_gpu_graphs import capture, replay_and_check

    bt = batch(41, [300, 33, 1000])
    q, kc, vc = bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev())
    table, lens, out = up_i32(bt.table), up_i32(bt.lens), torch.empty((3, 16, D), device=dev())
    sc = AttnScores(10.0, 200, slopes_of(16).to(dev()), up_i32([5, 6, 70]))
    attn = DecodeAttention(16, 8, 3, 1000, page_tokens=16)

    def call(stream=None):
        attn.run_paged(q, kc, vc, table, lens, SCALE, out, scores=sc, stream=stream)

    call()
    torch.cuda.synchronize()
    expected = out.clone()
    g = capture(call)
    replay_and_check(g, [out], [expected], lambda t: t.fill_(float("nan")), call)
    del g
    attn.close()
