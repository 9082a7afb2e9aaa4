"""ctx_prefill_attn_run_paged against a plain 64-bit form: caps, biases, windows,
prefixes and documents over shuffled pages, rows that see nothing, slots that no
query sees, and calls of both kinds of workgroup."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd import binding as bd
from paper_2609_36608_amd.binding import AttnScores, CtxError, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, attention_reference, randn

pytestmark = pytest.mark.gpu

SCALE = D ** -0.5

# fp32 outputs: logits of up to 30 and three-term weights as in the decode step's bound,
# 9e-5 (4.5 times 30 * 2^-21 of the logits and 2^-20 of the sums).
F32 = 9e-5
# bf16 outputs: a weight is rounded by at most u = 2^-8 of it and the row normalised by the
# sum of the rounded weights, which moves the output by at most 2 u / (1 - u) times the
# weighted mean of |value - output|; then half a step of the output.
U = 2.0 ** -8
ROUNDED = 2 * U / (1 - U)


def i32(t):
    return None if t is None else up_i32(t)


def up(t):
    return None if t is None else t.to(dev())


def run(bt, softcap=0.0, window=0, slopes=None, prefix=None, docs=None, out_dtype=torch.float32, scale=SCALE,
        max_q_len=None, scored=True, max_seq_len=None):
    buf = torch.full((bt.rows + 1, bt.hq, D), -777.0, dtype=out_dtype, device=dev())
    kc, vc = up(bt.k), up(bt.v)
    with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), max_seq_len or max(max(bt.lens), 1),
                         page_tokens=bt.page, out_dtype=out_dtype) as attn:
        attn.prefill_paged(up(bt.q), kc, vc, up_i32(bt.table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new),
                           max(bt.new) if max_q_len is None else max_q_len, scale, buf[:bt.rows],
                           scores=AttnScores(softcap, window, up(slopes), i32(prefix), i32(docs)) if scored else None)
        torch.cuda.synchronize()
    out = buf.cpu()
    assert (out[bt.rows] == -777.0).all()
    live = torch.tensor([at is not None for at in bt.row_of()])
    assert (out[:bt.rows][~live] == -777.0).all()
    assert torch.equal(kc.cpu().view(torch.int16), bt.k.view(torch.int16))
    return out[:bt.rows], live


def close(got, live, ref, spread, out_dtype, share=1.0):
    got, ref, spread = got[live], ref[live], spread[live]
    assert got.isfinite().all()
    bound = torch.full_like(ref, F32 * share)
    if out_dtype == torch.bfloat16:
        bound += ROUNDED * spread
        bound += U * (ref.abs() + bound)
    err = (got.double() - ref).abs()
    print(f"max-abs {err.max().item():.3e}, of the bound {(err / bound).max().item():.3f}", flush=True)
    assert (err <= bound).all(), f"worst {err.max().item():.3e}"


def check(bt, out_dtype=torch.float32, scale=SCALE, share=1.0, max_seq_len=None, **kw):
    got, live = run(bt, out_dtype=out_dtype, scale=scale, max_seq_len=max_seq_len, **kw)
    ref, spread = attention_reference(bt, scale, spread=True, **kw)
    close(got, live, ref, spread, out_dtype, share)
    return got, live


def kind_of(bt, out_dtype=torch.bfloat16, bound=None):
    """The workgroups that the call takes on 256 CUs: ("wide", tiles per wave) or ("narrow", waves)."""
    cols = max(bt.new) * (bt.hq // bt.hkv)
    most = 2 if out_dtype == torch.float32 else 3
    grid = lambda n: len(bt.lens) * bt.hkv * -(-cols // n)  # noqa: E731
    narrow = grid(16 * most)
    if (bound or max(bt.lens)) > 512 and narrow <= 512:
        return "narrow", 8 if narrow <= 256 else 4
    if grid(64) <= 768:
        return "wide", 1
    return "wide", 2 if most == 2 or grid(128) <= 576 else 3


def kind_batch(kind, gap=1):
    """A batch of 16 / 8 heads with odd and empty sequences that takes that kind with bf16 outputs,
    and the bound of its handle."""
    rng = np.random.default_rng(6)
    if kind == "wide3":
        new = rng.integers(1, 60, 40)
        lens = new + rng.integers(0, 200, 40)
        lens[:4], new[:4] = [300, 150, 33, 64], [300, 97, 33, 1]
    elif kind == "narrow8":
        lens, new = [150, 40, 0, 1, 300], [60, 40, 0, 1, 12]
    else:
        lens, new = [1, 40, 17, 33, 150, 300, 64, 0], [1, 40, 2, 1, 97, 12, 64, 0]
        if kind == "wide2":
            lens[4:6], new[4:6] = [480, 300], [450, 7]
    bound = 600 if kind.startswith("narrow") else None
    bt = Batch(3 + len(lens), lens, new, 16, 16, 8, gap=gap)
    assert kind_of(bt, bound=bound) == (kind[:-1], int(kind[-1]))
    return bt, bound


def slopes_of(hq):
    return 2.0 ** (-8.0 * torch.arange(1, hq + 1, dtype=torch.float32) / hq)


def docs_of(bt, rng, most=60):
    """Documents of 1..most tokens, and padding rows at the end of every other sequence."""
    docs = np.zeros(bt.rows, np.int32)
    for b, (n, m) in enumerate(zip(bt.lens, bt.new)):
        starts = np.cumsum(np.concatenate([[0], rng.integers(1, most, max(n, 1))]))
        for i in range(m):
            p = n - m + i
            docs[bt.starts[b] + i] = starts[starts <= p].max()
            if b % 2 and i >= m - 3:
                docs[bt.starts[b] + i] = 2 ** 31 - 1
    return docs


LENS = [1, 40, 17, 33, 150, 300, 64, 0]
NEW = [1, 40, 2, 1, 97, 12, 64, 0]
KINDS = ["none", "cap", "bias", "window", "prefix", "docs", "capbias", "all"]


def scores_of(kind, bt, rng):
    kw = {}
    if kind in ("cap", "capbias", "all"):
        kw["softcap"] = 5.0
    if kind in ("bias", "capbias", "all"):
        kw["slopes"] = slopes_of(bt.hq)
    if kind in ("window", "all"):
        kw["window"] = 37
    if kind in ("prefix", "all"):
        kw["prefix"] = rng.integers(0, 60, len(bt.lens))
    if kind in ("docs", "all"):
        kw["docs"] = docs_of(bt, rng)
    return kw


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scores", KINDS)
@pytest.mark.parametrize("kind", ["wide1", "wide2", "wide3", "narrow4", "narrow8"])
def test_scores_and_masks(kind, scores, out_dtype):
    bt, bound = kind_batch(kind)
    if scores == "cap":
        bt.q = randn(bt.g, bt.q.shape, 4.0)
    check(bt, out_dtype, max_seq_len=bound, **scores_of(scores, bt, np.random.default_rng(4)))


@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4), (16, 1), (5, 1), (9, 3), (7, 7), (30, 10), (1, 1)])
@pytest.mark.parametrize("page", [16, 48, 64])
def test_heads_and_pages(hq, hkv, page):
    bt = Batch(hq + page, [1, page, page + 1, 3 * page + 7, 100], [1, page, 5, page + 30, 33], page, hq, hkv, gap=1)
    kw = dict(softcap=20.0, window=50, slopes=slopes_of(hq), prefix=[0, 3, page, 17, 40])
    check(bt, torch.bfloat16, **kw)
    check(bt, torch.float32, max_seq_len=600, **kw)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 31, 32, 33, 1000])
@pytest.mark.parametrize("wide", [False, True])
def test_window_edges(window, wide):
    lens, new = ([900, 90], [850, 3]) if wide else (LENS, NEW)
    bt = Batch(window, lens, new, 16, 16, 8)
    assert kind_of(bt, bound=900) == (("wide", 1) if wide else ("narrow", 4))
    check(bt, torch.bfloat16, window=window, max_seq_len=900)


@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 33, 64, 65, 10 ** 6, -5])
@pytest.mark.parametrize("wide", [False, True])
def test_prefix_edges(prefix, wide):
    lens, new = ([900, 90], [850, 80]) if wide else (LENS, NEW)
    bt = Batch(prefix & 255, lens, new, 16, 16, 8)
    assert kind_of(bt, torch.float32, bound=900) == (("wide", 1) if wide else ("narrow", 4))
    got, live = run(bt, window=20, prefix=[prefix] * len(lens), max_seq_len=900)
    ref, spread = attention_reference(bt, SCALE, window=20, prefix=[min(max(prefix, 0), n) for n in lens], spread=True)
    close(got, live, ref, spread, torch.float32)


@pytest.mark.parametrize("wide", [False, True])
def test_rows_that_see_nothing_or_their_prefix_alone(wide):
    lens, new = ([900, 90, 50], [850, 90, 50]) if wide else ([100, 90, 50], [60, 90, 50])
    bt = Batch(11, lens, new, 16, 16, 8)
    kw = dict(max_seq_len=900)
    assert kind_of(bt, bound=900) == (("wide", 1) if wide else ("narrow", 8))
    docs = np.full(bt.rows, 2 ** 31 - 1, np.int64)
    got, live = run(bt, docs=docs, **kw)
    assert (got[live] == 0).all()
    docs[::2] = -7  # every other row sees all before it
    check(bt, docs=docs, **kw)
    check(bt, torch.bfloat16, docs=docs, prefix=[40, 0, 50], slopes=slopes_of(16) * 20, **kw)
    check(bt, docs=docs, prefix=[3, 33, 1], slopes=slopes_of(16) * 20, softcap=9.0, **kw)


@pytest.mark.parametrize("wide", [False, True])
def test_unseen_slots_may_hold_anything(wide):
    """NaN and infinities where no query of the sequence looks: between the prefix and the
    oldest window, and in the slots behind the sequence (NaN in every test here)."""
    lens, new = ([1500, 300], [850, 2]) if wide else ([600, 300], [40, 2])
    bt = Batch(13, lens, new, 16, 16, 8)
    assert kind_of(bt, torch.float32) == (("wide", 1) if wide else ("narrow", 8))
    kw = dict(window=45, prefix=[37, 3])
    clean, live = run(bt, **kw)
    for b, (n, m) in enumerate(zip(lens, new)):
        for t in range(kw["prefix"][b], n - m - 44):
            bt.k[bt.slot(b, t)] = float("nan")
            bt.v[bt.slot(b, t)] = float("inf") if t % 2 else float("nan")
    got, _ = run(bt, **kw)
    assert torch.equal(got, clean) and got[live].isfinite().all()


@pytest.mark.parametrize("kind", ["wide1", "wide2", "wide3", "narrow4", "narrow8"])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_padding_rows_between_documents_may_hold_anything(kind, out_dtype):
    """NaN and infinities at the positions of padding rows that no later row's document takes in,
    beside padding rows that a later row sees."""
    bt, bound = kind_batch(kind)
    rng = np.random.default_rng(9)
    docs = np.zeros(bt.rows, np.int64)
    prefix = rng.integers(0, 40, len(bt.lens))
    hidden = 0
    for b, (n, m) in enumerate(zip(bt.lens, bt.new)):
        seen = torch.arange(max(n, 0)) < int(prefix[b])
        first, i = 0, 0
        while i < m:
            for _ in range(min(int(rng.integers(1, 25)), m - i)):  # a document
                docs[bt.starts[b] + i] = first
                seen[first:n - m + i + 1] = True
                i += 1
            pads = min(int(rng.integers(0, 9)), m - i)
            docs[bt.starts[b] + i:bt.starts[b] + i + pads] = 2 ** 31 - 1
            i += pads
            first = n - m + i - int(rng.integers(0, 4) if rng.random() < 0.3 else 0)
        for t in torch.nonzero(~seen)[:, 0].tolist():
            bt.k[bt.slot(b, t)] = float("nan")
            bt.v[bt.slot(b, t)] = float("inf") if t % 2 else float("nan")
            hidden += 1
    assert hidden > 10
    got, live = run(bt, out_dtype=out_dtype, docs=docs, prefix=prefix, max_seq_len=bound)
    bt.k, bt.v = bt.k.nan_to_num(0.0, 0.0), bt.v.nan_to_num(0.0, 0.0)
    ref, spread = attention_reference(bt, SCALE, docs=docs, prefix=prefix, spread=True)
    close(got, live, ref, spread, out_dtype)


@pytest.mark.parametrize("wide", [False, True])
def test_pages_outside_the_cache_are_not_seen(wide):
    lens, new = ([700, 100, 90], [600, 50, 90]) if wide else ([200, 100, 90], [70, 50, 90])
    bt = Batch(17, lens, new, 16, 16, 8)
    kw = dict(max_seq_len=900)
    assert kind_of(bt, torch.float32, 900) == (("wide", 1) if wide else ("narrow", 8))
    bt.table[0, 3] = -1
    bt.table[0, 6] = bt.num_pages
    bt.table[1, :] = 2 ** 31 - 1  # nothing left
    bt.table[2, 0] = -2 ** 31
    got, live = check(bt, softcap=30.0, **kw)
    rows = [j for j, at in enumerate(bt.row_of()) if at is not None and at[0] == 1]
    assert (got[rows] == 0).all()
    check(bt, torch.bfloat16, window=60, prefix=[20, 0, 17], **kw)
    bt.table = np.ascontiguousarray(bt.table[:, :3])  # and tokens past the table
    check(bt, slopes=slopes_of(16), **kw)
    check(bt, torch.bfloat16, window=100, prefix=[20, 0, 17], **kw)


@pytest.mark.parametrize("hist", [1000, 1024, 2100])
@pytest.mark.parametrize("new", [4, 400])
def test_long_histories(hist, new):
    """More half blocks than a wave holds cache rows for, in calls of both kinds."""
    bt = Batch(hist + new, [hist + new, 70], [new, 30], 16, 32, 8)
    assert kind_of(bt) == (("wide", 1) if new == 400 else ("narrow", 8))
    check(bt, torch.bfloat16)
    check(bt, window=1100, prefix=[50, 70], softcap=8.0)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
def test_few_rows_over_contexts_shared_out(kind, out_dtype):
    """Handles whose bound lets several workgroups share a context: long ones, ones of a single
    block, empty ones, and rows of no sequence between them."""
    bt = Batch(53, [3000, 5, 33, 700, 0, 1200], [3, 5, 1, 2, 0, 4], 16, 16, 8, gap=1)
    kw = scores_of(kind, bt, np.random.default_rng(8))
    if kind in ("window", "all"):
        kw["window"] = 600
    check(bt, out_dtype, max_seq_len=30000, **kw)


def test_shared_out_with_few_heads_and_one_row():
    for hq, hkv in ((1, 1), (16, 1), (12, 2)):
        bt = Batch(59 + hq, [5000], [1], 48, hq, hkv)
        check(bt, torch.bfloat16, max_seq_len=1 << 20)
        check(bt, slopes=slopes_of(hq), prefix=[40], window=4000)
        bt.table[0, 30:] = -1  # the later shares see nothing
        check(bt, max_seq_len=1 << 20)


def test_large_logits_and_a_zero_scale():
    bt = Batch(19, [300, 40], [120, 40], 16, 16, 8)
    bt.q[:100] *= 64  # one token has all the weight
    check(bt, share=64.0)
    check(bt, softcap=2.0)
    check(bt, torch.bfloat16, softcap=2.0)
    check(bt, scale=0.0, softcap=2.0)
    check(bt, torch.bfloat16, scale=0.0)
    check(bt, torch.bfloat16, scale=-SCALE / 64, slopes=-slopes_of(16))
    bt.k[~bt.k.isnan()] *= 2.0 ** 60  # every score at its cap
    check(bt, torch.bfloat16, softcap=1.0)
    check(bt, softcap=1.0)


@pytest.mark.parametrize("softcap", [1e-3, 500.0, 600.0, 1e5, 1e38])
def test_caps_from_tiny_to_far_above_the_scores(softcap):
    bt = Batch(61, [300, 90], [120, 2], 16, 16, 8)
    bt.q[::3] *= 8
    for kw in (dict(), dict(slopes=slopes_of(16), window=70)):
        check(bt, torch.bfloat16, softcap=softcap, share=8.0, **kw)
        check(bt, softcap=softcap, share=8.0, **kw)


def test_rising_and_falling_scores():
    """Running maxima that move in every block, and rows whose first block is far below the rest."""
    bt = Batch(23, [600], [300], 16, 8, 8)
    check(bt, slopes=torch.full((8,), 1.5))
    check(bt, slopes=torch.full((8,), -1.5))
    check(bt, torch.bfloat16, slopes=torch.full((8,), 1.5), window=90)
    check(bt, slopes=torch.full((8,), 3.0), docs=np.full(300, 2 ** 31 - 1, np.int64), prefix=[100])


def test_many_sequences_of_one_token_and_none():
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 100, 300)
    bt = Batch(29, lens, np.minimum(lens, rng.integers(0, 4, 300)), 16, 4, 2)
    check(bt, torch.bfloat16, window=30, prefix=rng.integers(0, 20, 300))


def test_broken_batches_stay_in_bounds():
    """Rows past the arrays, more new tokens than tokens and negative lengths touch nothing outside."""
    bt = Batch(31, [50, 20, 30], [50, 20, 30], 16, 8, 2)
    q, kc, vc = up(bt.q), up(bt.k), up(bt.v)
    buf = torch.full((bt.rows + 64, 8, D), -777.0, device=dev())
    with DecodeAttention(8, 2, 3, 64, page_tokens=16) as attn:
        for lens, starts, new in (([50, 20, 30], [80, -10, 2 ** 31 - 40], [50, 20, 60]), ([-5, 3, 30], [0, 50, 70], [9, 20, 30])):
            attn.prefill_paged(q, kc, vc, up_i32(bt.table), up_i32(lens), up_i32(starts), up_i32(new), 60, SCALE,
                               buf[:bt.rows], scores=AttnScores(window=9))
            torch.cuda.synchronize()
        assert (buf[bt.rows:] == -777.0).all()


def test_a_bound_below_a_sequence_leaves_the_further_rows():
    bt = Batch(37, [50, 20], [50, 20], 16, 16, 8)
    got, _ = run(bt, max_q_len=33)
    ref = attention_reference(bt, SCALE)
    for j, (b, p) in enumerate(bt.row_of()):
        if p < 33:
            assert ((got[j].double() - ref[j]).abs() <= F32).all()
        else:
            assert (got[j] == -777.0).all()


def test_no_scores_equals_empty_scores_and_another_stream():
    bt = Batch(41, LENS, NEW, 16, 16, 8)
    a, _ = run(bt, scored=False)
    b, _ = run(bt)
    assert torch.equal(a, b)


def test_refusals():
    bt = Batch(43, [20, 5], [20, 5], 16, 8, 2)
    q, kc, vc = up(bt.q), up(bt.k), up(bt.v)
    table, lens, st, nl = up_i32(bt.table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new)
    out = torch.empty((bt.rows, 8, D), device=dev())
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        def call(scores=None, **kw):
            a = {**dict(q=q, k_pages=kc, v_pages=vc, block_tables=table, seq_lens=lens, q_starts=st, q_lens=nl,
                        max_q_len=20, scale=SCALE, out=out), **kw}
            return attn.prefill_paged(**a, scores=scores)

        call()
        for kw, status in ((dict(scores=AttnScores(softcap=-1.0)), bd.CTX_ERR_INVALID_ARG),
                           (dict(scores=AttnScores(softcap=2e38)), bd.CTX_ERR_INVALID_ARG),
                           (dict(scores=AttnScores(softcap=1e-40)), bd.CTX_ERR_INVALID_ARG),
                           (dict(scores=AttnScores(softcap=float("nan"))), bd.CTX_ERR_INVALID_ARG),
                           (dict(scores=AttnScores(window=-1)), bd.CTX_ERR_INVALID_ARG),
                           (dict(scale=float("nan")), bd.CTX_ERR_INVALID_ARG),
                           (dict(max_q_len=-1), bd.CTX_ERR_INVALID_ARG)):
            with pytest.raises(CtxError) as e:
                call(**kw)
            assert e.value.status == status
        with pytest.raises(ValueError):
            call(q=q[:, :4].contiguous())
        with pytest.raises(TypeError):
            call(out=out.bfloat16())
        with pytest.raises(ValueError):
            call(block_tables=table[:1])
        with pytest.raises(ValueError):
            call(scores=AttnScores(doc_starts=lens))  # one per row
        with pytest.raises(ValueError):
            call(scores=AttnScores(slopes=torch.ones(8)))
        with pytest.raises(ValueError):
            call(q_lens=nl[:1])
    with DecodeAttention(8, 2, 2, 32) as plain, pytest.raises(ValueError):
        plain.prefill_paged(q, kc, vc, table, lens, st, nl, 20, SCALE, out)


@pytest.mark.parametrize("wide", [False, True])
def test_graph_replays(wide):
    from test_gpu_graphs import capture, replay_and_check

    lens, new = ([900, 90], [850, 80]) if wide else ([300, 33], [60, 1])
    bt = Batch(47, lens, new, 16, 16, 8)
    assert kind_of(bt, bound=900) == (("wide", 1) if wide else ("narrow", 8))
    q, kc, vc = up(bt.q), up(bt.k), up(bt.v)
    args = [up_i32(x) for x in (bt.table, bt.lens, bt.starts, bt.new)]
    sc = AttnScores(10.0, 50, up(slopes_of(16)), up_i32([5, 40]))
    out = torch.empty((bt.rows, 16, D), dtype=torch.bfloat16, device=dev())
    attn = DecodeAttention(16, 8, 2, 900, page_tokens=16, out_dtype=torch.bfloat16)

    def call(stream=None):
        attn.prefill_paged(q, kc, vc, *args, max(new), SCALE, out, scores=sc, stream=stream)

    call()
    torch.cuda.synchronize()
    expected = out.clone()
    g = capture(call)
    replay_and_check(g, [out], [expected], lambda t: t.fill_(float("nan")), call)
    del g
    attn.close()
