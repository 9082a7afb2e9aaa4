"""Attention of drafted trees (ctx_tree_attn_run_paged) against a plain 64-bit form: trees of every
kind over shuffled pages, padding, windows, prefixes, caps and slopes by position, ranges that cut
items, and slots that no draft sees (NaN)."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import AttnScores, CtxError, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, randn

pytestmark = pytest.mark.gpu

SCALE = D ** -0.5
PADDING = 2 ** 31 - 1

# fp32 outputs: logits of up to 30 and three-term weights, as in the causal prefill's bound:
# 9e-5 (4.5 times 30 * 2^-21 of the logits and 2^-20 of the sums).
F32 = 9e-5
# bf16 outputs: a weight is rounded by at most u of it (2^-8, two terms 2^-16) and the row normalised
# by the sum of the rounded weights, which moves the output by at most 2 u / (1 - u) times the
# weighted mean of |value - output|; then half a step of the output, 2^-8.
U = 2.0 ** -8


def rounded(u):
    return 2 * u / (1 - u)


def tree_of(kind, n, rng):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "roots":
        return [-1] * n
    if kind == "binary":
        return [(i - 1) // 2 if i else -1 for i in range(n)]
    if kind == "padded":  # among the others, and with drafts below
        return [PADDING if rng.random() < 0.2 else int(rng.integers(-1, i)) if i else -1 for i in range(n)]
    if kind == "wrong":  # no parents: themselves, later ones, numbers below -1
        return [int(rng.choice([-1, i, i + 1, -2, max(i - 1, 0) if i else -1])) for i in range(n)]
    return [max(-1, i - int(rng.integers(1, 5))) for i in range(n)]


def paths_of(parents):
    paths = []
    for i, p in enumerate(parents):
        if p < -1 or p >= i:
            paths.append([])
        elif p == -1:
            paths.append([i])
        else:
            paths.append(paths[p] + [i] if paths[p] else [])
    return paths


class Trees:
    """A batch whose last new[b] tokens are drafts; padding rows hold NaN everywhere."""

    def __init__(self, seed, lens, new, kinds, page=16, hq=16, hkv=8, gap=1):
        self.bt = bt = Batch(seed, lens, new, page, hq, hkv, gap=gap)
        rng = np.random.default_rng(seed + 1)
        kinds = [kinds] * len(lens) if isinstance(kinds, str) else kinds
        self.trees = [tree_of(k, n, rng) for k, n in zip(kinds, new)]
        self.paths = [paths_of(t) for t in self.trees]
        self.parents = np.full(bt.rows, -77, np.int32)
        for b, tree in enumerate(self.trees):
            for i, p in enumerate(tree):
                self.parents[bt.starts[b] + i] = p
                if not self.paths[b][i]:
                    bt.q[bt.starts[b] + i] = float("nan")
                    slot = bt.slot(b, bt.lens[b] - bt.new[b] + i)
                    if slot is not None:
                        bt.k[slot] = bt.v[slot] = float("nan")

    def reference(self, scale=SCALE, softcap=0.0, window=0, slopes=None, prefix=None, max_q_len=None):
        bt = self.bt
        g = bt.hq // bt.hkv
        out = torch.full((bt.rows, bt.hq, D), float("nan"), dtype=torch.float64)
        spread = torch.zeros_like(out)
        for b, paths in enumerate(self.paths):
            n = max(bt.lens[b], 0)
            hist = n - bt.new[b]
            slots = [bt.slot(b, t) for t in range(n)]
            there = torch.tensor([s is not None for s in slots], dtype=torch.bool)
            kb, vb = torch.zeros((n, bt.hkv, D), dtype=torch.float64), torch.zeros((n, bt.hkv, D), dtype=torch.float64)
            if there.any():
                at = torch.tensor([s if s is not None else (0, 0) for s in slots])
                kb, vb = (x[at[:, 0], at[:, 1]].double() for x in (bt.k, bt.v))
            place = torch.arange(n)
            for i, path in enumerate(paths):
                place[hist + i] = hist + max(len(path) - 1, 0)
            for i, path in enumerate(paths):
                if max_q_len is not None and i >= max_q_len:
                    break
                row = bt.starts[b] + i
                out[row] = 0
                if not path:
                    continue
                p = hist + len(path) - 1
                see = torch.zeros(n, dtype=torch.bool)
                see[:hist] = True
                see[[hist + a for a in path]] = True
                if window:
                    see &= (p - place < window) | (torch.arange(n) < min(0 if prefix is None else prefix[b], hist))
                see &= there
                t = torch.nonzero(see)[:, 0]
                if len(t) == 0:
                    continue
                s = torch.einsum("hgd,thd->hgt", bt.q[row].double().view(bt.hkv, g, D), kb[t]) * scale
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                if slopes is not None:
                    s = s - slopes.double().view(bt.hkv, g, 1) * (p - place[t]).double()
                w = torch.softmax(s, -1)
                o = torch.einsum("hgt,thd->hgd", w, vb[t])
                out[row] = o.reshape(bt.hq, D)
                far = (vb[t].permute(1, 0, 2)[:, None] - o[:, :, None]).abs()
                spread[row] = (w[..., None] * far).sum(2).reshape(bt.hq, D)
        return out, spread

    def run(self, out_dtype=torch.float32, scale=SCALE, softcap=0.0, window=0, slopes=None, prefix=None, max_q_len=None,
            split_p=False, max_seq_len=None, scored=True):
        bt = self.bt
        buf = torch.full((bt.rows + 1, bt.hq, D), -777.0, dtype=out_dtype, device=dev())
        kc, vc = bt.k.to(dev()), bt.v.to(dev())
        scores = AttnScores(softcap, window, None if slopes is None else slopes.to(dev()),
                            None if prefix is None else up_i32(prefix), split_p=split_p)
        with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), max_seq_len or max(max(bt.lens), 1), page_tokens=bt.page,
                             out_dtype=out_dtype) as attn:
            attn.tree_paged(bt.q.to(dev()), kc, vc, up_i32(bt.table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new),
                            up_i32(self.parents), max(bt.new) if max_q_len is None else max_q_len, scale, buf[:bt.rows],
                            scores=scores if scored else None)
            torch.cuda.synchronize()
        out = buf.cpu()
        assert (out[bt.rows] == -777.0).all()
        assert torch.equal(kc.cpu().view(torch.int16), bt.k.view(torch.int16))
        return out[:bt.rows]

    def check(self, out_dtype=torch.float32, split_p=False, share=1.0, max_seq_len=None, scored=True, **kw):
        got = self.run(out_dtype=out_dtype, split_p=split_p, max_seq_len=max_seq_len, scored=scored, **kw)
        ref, spread = self.reference(**kw)
        live = ~torch.isnan(ref[:, 0, 0])
        assert (got[~live] == -777.0).all()
        got, ref, spread = got[live], ref[live], spread[live]
        assert got.isfinite().all()
        bound = torch.full_like(ref, F32 * share)
        if out_dtype == torch.bfloat16:
            bound += rounded(2.0 ** -16 if split_p else U) * spread
            bound += U * (ref.abs() + bound)
        err = (got.double() - ref).abs()
        print(f"max-abs {err.max().item():.3e}, of the bound {(err / bound).max().item():.3f}", flush=True)
        assert (err <= bound).all(), f"worst {err.max().item():.3e}"
        zero = (ref == 0).all(-1).all(-1)
        assert (got[zero] == 0).all()
        return got


DTYPES = pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
HEADS = [(16, 8), (32, 8), (28, 4), (16, 1), (5, 5), (64, 4)]


@DTYPES
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("kind", ["random", "chain", "padded"])
def test_ragged_batch(kind, hq, hkv, out_dtype):
    Trees(hq + hkv, [40, 300, 17, 64, 33, 0, 9, 700], [7, 16, 17, 1, 33, 0, 9, 30], kind, hq=hq, hkv=hkv).check(out_dtype)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 100, 128, 200, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (7, 1)])
def test_numbers_of_drafts(n, hq, hkv):
    """One to all words of the masks, every workgroup shape, tiles of columns."""
    rng = np.random.default_rng(n)
    lens = [n + int(h) for h in rng.integers(0, 150, 3)]
    Trees(n, lens, [n, max(1, n // 2), n], ["random", "binary", "chain"], hq=hq, hkv=hkv).check()


@DTYPES
@pytest.mark.parametrize("kind", ["roots", "binary", "wrong", "padded"])
def test_kinds_of_trees(kind, out_dtype):
    Trees(3, [130, 96, 64, 20], [40, 64, 64, 20], kind, page=48, hq=12, hkv=4).check(out_dtype)


def test_padding_alone():
    t = Trees(4, [90, 60, 33], [5, 60, 2], "random", hq=8, hkv=2)
    bt = t.bt
    for b in (0, 1):  # nothing of these sequences is seen: all of their caches may hold anything
        t.trees[b] = [PADDING] * bt.new[b]
        t.paths[b] = [[]] * bt.new[b]
        t.parents[bt.starts[b]:bt.starts[b] + bt.new[b]] = PADDING
        for x in range(bt.lens[b]):
            bt.k[bt.slot(b, x)] = bt.v[bt.slot(b, x)] = float("nan")
        bt.q[bt.starts[b]:bt.starts[b] + bt.new[b]] = float("nan")
    got = t.check()
    assert (got == 0).any()


@DTYPES
@pytest.mark.parametrize("window", [1, 2, 5, 33, 100, 10 ** 6])
@pytest.mark.parametrize("prefixed", [False, True])
def test_windows(window, prefixed, out_dtype):
    t = Trees(window, [200, 350, 64, 500], [20, 40, 64, 33], ["chain", "random", "chain", "padded"], hq=8, hkv=2)
    bt = t.bt
    prefix = [7, 0, 99, 70] if prefixed else None
    for b in range(4):  # tokens that no draft sees
        hist = bt.lens[b] - bt.new[b]
        for x in range(min(prefix[b], hist) if prefixed else 0, max(0, hist - window + 1)):
            bt.k[bt.slot(b, x)] = bt.v[bt.slot(b, x)] = float("nan")
    t.check(out_dtype, window=window, prefix=prefix)


@DTYPES
@pytest.mark.parametrize("hq,hkv,n", [(8, 8, 30), (28, 4, 61), (16, 1, 40)])
def test_scores(hq, hkv, n, out_dtype):
    t = Trees(hq, [900, 333, 70], [n, n // 2, n], ["random", "chain", "padded"], page=64, hq=hq, hkv=hkv)
    t.bt.q *= 4
    slopes = 2.0 ** (-8.0 * torch.arange(1, hq + 1) / hq)
    for kw in (dict(softcap=30.0), dict(slopes=slopes), dict(softcap=5.0, slopes=slopes, window=200, prefix=[20, 40, 9]),
               dict(slopes=-slopes / 4, window=300)):
        # a bias of up to 330 has steps of 2^-16 in fp32, two of them
        t.check(out_dtype, share=1.0 + (2 * 330 * 2.0 ** -24 / F32 if "slopes" in kw else 0), **kw)


def test_two_term_weights():
    t = Trees(6, [400, 90, 60], [30, 60, 33], "random", hq=32, hkv=8)
    t.check(torch.bfloat16, split_p=True)
    t.check(torch.bfloat16, scored=False)


@pytest.mark.parametrize("hq,hkv,lens,new", [
    (32, 8, [6000], [5]), (32, 8, [5000], [60]), (16, 2, [3000, 20, 4000], [64, 3, 17]),
    (8, 1, [100] * 70 + [3000] + [37] * 70, [3] * 141),
    (4, 4, list(range(1, 300)), [1 + n % 7 if n > 6 else 1 for n in range(1, 300)]),
])
def test_ranges_that_cut_items(hq, hkv, lens, new):
    Trees(len(lens), lens, new, "random", hq=hq, hkv=hkv, gap=0).check()
    t = Trees(len(lens), lens, new, "padded", hq=hq, hkv=hkv, gap=0)
    t.check(max_seq_len=64)  # fewer ranges than the lengths ask for


def test_a_chain_is_a_causal_prefill():
    t = Trees(8, [500, 80, 33], [40, 9, 33], "chain", hq=32, hkv=8)
    bt = t.bt
    got = t.run()
    out = torch.full((bt.rows, bt.hq, D), -777.0, device=dev())
    with DecodeAttention(bt.hq, bt.hkv, 3, 500, page_tokens=16) as attn:
        attn.prefill_paged(bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table), up_i32(bt.lens),
                           up_i32(bt.starts), up_i32(bt.new), 40, SCALE, out)
    assert (got - out.cpu()).abs().max() <= 2 * F32


def test_rows_past_the_bound_and_outside():
    t = Trees(9, [60, 70, 50], [20, 12, 30], "random", hq=8, hkv=2, gap=0)
    got = t.check(max_q_len=12)
    assert len(got) == 36
    bt = t.bt
    # rows before 0 and past total_q
    rows = bt.rows - 5
    starts = bt.starts.copy()
    first, last = int(np.argmin(starts)), int(np.argmax(starts))
    starts[first] -= 4
    buf = torch.full((bt.rows, 8, D), -777.0, device=dev())
    with DecodeAttention(8, 2, 3, 70, page_tokens=16) as attn:
        attn.tree_paged(bt.q[:rows].contiguous().to(dev()), bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table),
                        up_i32(bt.lens), up_i32(starts), up_i32(bt.new), up_i32(t.parents[:rows]), 30, SCALE, buf[:rows])
        torch.cuda.synchronize()
    assert (buf[rows:] == -777.0).all() and last != first
    middle = [b for b in range(3) if b not in (first, last)][0]
    ref, _ = t.reference()
    at = slice(bt.starts[middle], bt.starts[middle] + bt.new[middle])
    assert (buf[at].cpu().double() - ref[at]).abs().max() <= F32


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_pages_that_are_not_there(bad):
    t = Trees(10, [300, 200], [20, 33], "random", hq=8, hkv=2)
    t.bt.table[0, 4] = t.bt.table[0, 9] = bad
    t.bt.table[1, 12] = bad  # among the drafts
    t.check()
    t.bt.table = np.ascontiguousarray(t.bt.table[:, :11])  # tables that end early
    t.check()


def test_large_pages_far_into_the_caches():
    """Caches of more than 4 GiB each, pages at their ends."""
    page, hkv = 256, 8
    pages = (5 << 30) // (page * hkv * D * 2)
    t = Trees(11, [700, 300], [33, 12], "random", page=page, hq=32, hkv=hkv)
    bt = t.bt
    k = torch.zeros((pages, page, hkv, D), dtype=torch.bfloat16, device=dev())
    v = torch.zeros_like(k)
    table = bt.table.copy()
    for i, p in enumerate(sorted({int(x) for x in bt.table.ravel() if x >= 0})):
        to = pages - 1 - 3 * i
        k[to], v[to] = bt.k[p].to(dev()), bt.v[p].to(dev())
        table[bt.table == p] = to
    out = torch.full((bt.rows, 32, D), -777.0, device=dev())
    with DecodeAttention(32, hkv, 2, 700, page_tokens=page) as attn:
        attn.tree_paged(bt.q.to(dev()), k, v, up_i32(table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new),
                        up_i32(t.parents), 33, SCALE, out)
    ref, _ = t.reference()
    live = ~torch.isnan(ref[:, 0, 0])
    assert (out.cpu().double() - ref)[live].abs().max() <= F32


def device_args(t):
    bt = t.bt
    return dict(q=bt.q.to(dev()), k_pages=bt.k.to(dev()), v_pages=bt.v.to(dev()), block_tables=up_i32(bt.table),
                seq_lens=up_i32(bt.lens), q_starts=up_i32(bt.starts), q_lens=up_i32(bt.new), parents=up_i32(t.parents))


def test_graph_replays_and_streams():
    t = Trees(12, [2000, 300, 90], [30, 12, 20], "random", hq=16, hkv=8)
    a = device_args(t)
    outs = [torch.zeros((t.bt.rows, 16, D), device=dev()) for _ in range(3)]
    with DecodeAttention(16, 8, 3, 2000, page_tokens=16) as attn:
        want = attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=outs[0]).clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=outs[1])
        for _ in range(3):
            outs[1].zero_()
            graph.replay()
            attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=outs[0])  # between replays
            assert torch.equal(outs[1], want) and torch.equal(outs[0], want)
        # another state in the captured buffers
        a["q"].copy_(randn(torch.Generator().manual_seed(5), tuple(a["q"].shape)).to(dev()))
        graph.replay()
        eager = attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=outs[0])
        assert torch.equal(outs[1], eager) and not torch.equal(eager, want)
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(4):
            for s, o in zip(streams, outs[1:]):
                o.zero_()
                s.wait_stream(torch.cuda.current_stream())
                attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=o, stream=s)
            torch.cuda.synchronize()
            assert torch.equal(outs[1], eager) and torch.equal(outs[2], eager)
        size = attn.tree_workspace(3, 30)
        ws = torch.full((size,), 255, dtype=torch.uint8, device=dev())
        assert torch.equal(attn.tree_paged(**a, max_q_len=30, scale=SCALE, out=outs[0], workspace=ws), eager)


def test_refusals():
    t = Trees(13, [100, 60], [10, 12], "random", hq=8, hkv=2)
    a = device_args(t) | dict(max_q_len=12, scale=SCALE, out=torch.zeros((t.bt.rows, 8, D), device=dev()))
    with DecodeAttention(8, 2, 2, 100, page_tokens=16) as attn:
        attn.tree_paged(**a)
        for kw, error in ((dict(parents=a["parents"].long()), TypeError), (dict(parents=a["parents"][:-1].contiguous()), ValueError),
                          (dict(q=a["q"].float()), TypeError), (dict(out=a["out"].bfloat16()), TypeError),
                          (dict(scores=AttnScores(doc_starts=a["parents"])), ValueError), (dict(max_q_len=257), CtxError),
                          (dict(max_q_len=-1), CtxError), (dict(workspace=torch.empty(64, dtype=torch.uint8, device=dev())), CtxError),
                          (dict(scale=float("nan")), CtxError), (dict(scores=AttnScores(window=-1)), CtxError)):
            with pytest.raises(error):
                attn.tree_paged(**(a | kw))
        attn.tree_paged(**(a | dict(max_q_len=0)))
    with pytest.raises(RuntimeError):
        attn.tree_paged(**a)
