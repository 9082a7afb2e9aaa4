"""The operators over paged caches as a serving loop runs them: turns of new tokens appended,
prefilled and followed by decoded tokens, against attention computed from scratch; caches past
4 GiB; the loop's step in a captured graph."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import AttnScores, DecodeAttention, Rotary

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, append_reference, attention_reference, randn

pytestmark = pytest.mark.gpu

SCALE = D ** -0.5
HQ, HKV, PAGE = 16, 8, 16


def inv_freq():
    return (1e6 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float()


class Loop:
    """Sequences that grow, on the device and in a plain 64-bit form.  The plain form takes the
    rotated queries and keys as the device has rounded them to bf16 (checked by the append's own
    tests and here, to a rounding), so that the attention is compared by itself."""

    def __init__(self, seed, lens, room, out_dtype, scores):
        self.bt = Batch(seed, [n + room for n in lens], [0] * len(lens), PAGE, HQ, HKV)
        bt = self.bt
        bt.k.fill_(float("nan"))  # nothing is in the cache yet
        bt.v.fill_(float("nan"))
        bt.lens = [0] * len(lens)
        self.g, self.scores, self.out_dtype = bt.g, scores, out_dtype
        self.kc, self.vc, self.table = bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table)
        self.norm = 1 + randn(self.g, (D,), 0.2)
        self.rotary = Rotary(inv_freq().to(dev()), q_norm=self.norm.to(dev()), k_norm=self.norm.to(dev()))
        self.attn = DecodeAttention(HQ, HKV, len(lens), 4096, page_tokens=PAGE, out_dtype=out_dtype)

    def device_scores(self):
        s = self.scores
        up = lambda t: None if t is None else t.to(dev())  # noqa: E731
        return AttnScores(s.get("softcap", 0.0), s.get("window", 0), up(s.get("slopes")),
                          None if s.get("prefix") is None else up_i32(s["prefix"]))

    def turn(self, new):
        """new[b] more tokens of every sequence: appended, then attending."""
        bt, n = self.bt, len(new)
        bt.lens = [a + b for a, b in zip(bt.lens, new)]
        bt.new = list(new)
        bt.starts = np.concatenate([[0], np.cumsum(new)[:-1]]).astype(np.int32)
        bt.rows = int(sum(new))
        x = randn(self.g, (bt.rows, (HQ + 2 * HKV), D), 1.5)
        q, k, v = x.split([HQ, HKV, HKV], 1)
        rq, rk, rv, _, _ = append_reference(bt, q, k, v, inv_freq().tolist(), q_norm=self.norm, k_norm=self.norm)
        xd = x.to(dev())
        qd, kd, vd = xd.split([HQ, HKV, HKV], 1)
        lens = up_i32(bt.lens)
        single = all(m == 1 for m in new)
        rows = {} if single else dict(q_starts=up_i32(bt.starts), q_lens=up_i32(bt.new))
        qr = self.attn.append_paged(kd, vd, self.kc, self.vc, self.table, lens, q=qd, rotary=self.rotary, **rows)
        out = torch.full((bt.rows, HQ, D), -777.0, dtype=self.out_dtype, device=dev())
        sc = self.device_scores()
        if single:
            self.attn.run_paged(qr, self.kc, self.vc, self.table, lens, SCALE, out, scores=sc)
        else:
            self.attn.prefill_paged(qr, self.kc, self.vc, self.table, lens, rows["q_starts"], rows["q_lens"], max(new),
                                    SCALE, out, scores=sc)
        torch.cuda.synchronize()
        kc = self.kc.cpu()
        # one rounding to bf16, and fp32 arithmetic before it
        for got, ref in ((qr.cpu(), rq), (kc, rk)):
            ok = ~ref.isnan()
            assert torch.equal(ok, ~got.isnan())
            assert ((got.double() - ref)[ok].abs() <= 2.0 ** -8 * ref[ok].abs() + 2.0 ** -14).all()
        bt.k, bt.v, bt.q = kc, self.vc.cpu(), qr.cpu()
        there = ~rv.isnan()
        assert torch.equal(bt.v[there], rv[there].to(torch.bfloat16))
        ref, spread = attention_reference(bt, SCALE, spread=True, **self.scores)
        # the bounds of the attention's own tests
        bound = torch.full_like(ref, 9e-5)
        if self.out_dtype == torch.bfloat16:
            u = 2.0 ** -8
            bound += 2 * u / (1 - u) * spread
            bound += u * (ref.abs() + bound)
        got = out.cpu().double()
        assert got.isfinite().all() and ((got - ref).abs() <= bound).all(), (got - ref).abs().max().item()


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scores", [
    {},
    dict(softcap=8.0),
    dict(window=45, prefix=[10, 0, 33, 2]),
    dict(slopes=2.0 ** (-8.0 * torch.arange(1, HQ + 1, dtype=torch.float32) / HQ), softcap=20.0, window=100),
])
def test_turns_and_decoded_tokens(scores, out_dtype):
    loop = Loop(3, [60, 20, 300, 5], 200, out_dtype, scores)
    loop.turn([60, 20, 300, 5])
    for _ in range(3):
        loop.turn([1, 1, 1, 1])
    loop.turn([17, 1, 0, 40])
    loop.turn([0, 0, 64, 2])
    for _ in range(2):
        loop.turn([1, 1, 1, 1])
    loop.attn.close()


def test_caches_past_4_gib():
    """The same batch in a small cache and at the far end of one whose halves pass byte offset 2^32."""
    bt = Batch(5, [200, 40, 600], [33, 40, 1], PAGE, HQ, HKV, gap=1)
    small = [bt.k.to(dev()), bt.v.to(dev())]
    per_page = PAGE * HKV * D * 2
    far = (5 << 30) // per_page
    big = [torch.empty((far + bt.num_pages, PAGE, HKV, D), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    for b, s in zip(big, small):
        b[far:] = s
    q, k, v = (randn(bt.g, (bt.rows, h, D)).to(dev()) for h in (HQ, HKV, HKV))
    lens, starts, new = up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new)
    rotary = Rotary(inv_freq().to(dev()))
    sc = AttnScores(softcap=30.0, window=150, prefix_lens=up_i32([10, 0, 40]))
    results = []
    with DecodeAttention(HQ, HKV, 3, 600, page_tokens=PAGE) as attn:
        for (kc, vc), table in ((small, bt.table), (big, np.where(bt.table >= 0, bt.table + far, -1))):
            table = up_i32(table)
            qr = attn.append_paged(k, v, kc, vc, table, lens, q=q, q_out=torch.zeros_like(q), q_starts=starts, q_lens=new, rotary=rotary)
            out = torch.zeros((bt.rows, HQ, D), device=dev())
            attn.prefill_paged(qr, kc, vc, table, lens, starts, new, 40, SCALE, out, scores=sc)
            one = attn.run_paged(qr[1:4], kc, vc, table, lens, SCALE, torch.zeros((3, HQ, D), device=dev()), scores=sc)
            torch.cuda.synchronize()
            results.append((qr, out, one))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    for b, s in zip(big, small):
        assert torch.equal(b[far:].view(torch.int16), s.view(torch.int16))


def test_a_step_in_a_graph_follows_its_inputs():
    """Append and decode captured together and replayed as the sequences grow: lengths, tables and
    rows are read on the device."""
    from test_gpu_graphs import capture

    bt = Batch(7, [80, 33, 300], [1, 1, 1], PAGE, HQ, HKV)
    room = 40
    bt2 = Batch(7, [n + room for n in bt.lens], [1, 1, 1], PAGE, HQ, HKV)
    kc, vc, table = bt2.k.to(dev()), bt2.v.to(dev()), up_i32(bt2.table)
    lens = up_i32(bt.lens)
    k, v, q = (torch.empty((3, h, D), dtype=torch.bfloat16, device=dev()) for h in (HKV, HKV, HQ))
    qr, out = torch.empty_like(q), torch.empty((3, HQ, D), device=dev())
    rotary, sc = Rotary(inv_freq().to(dev())), AttnScores(softcap=15.0, window=64)
    attn = DecodeAttention(HQ, HKV, 3, 400, page_tokens=PAGE)

    def step(stream=None):
        attn.append_paged(k, v, kc, vc, table, lens, q=q, q_out=qr, rotary=rotary, stream=stream)
        attn.run_paged(qr, kc, vc, table, lens, SCALE, out, scores=sc, stream=stream)

    for t in (k, v, q):
        t.zero_()
    step()
    torch.cuda.synchronize()
    g = capture(step)
    for n in (0, 1, 15, 16, 17, 39):
        for t in (k, v, q):
            t.copy_(randn(bt.g, t.shape))
        lens.copy_(up_i32([x + n for x in bt.lens]))
        before = kc.clone(), vc.clone()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (qr, out, kc, vc)]
        kc.copy_(before[0])
        vc.copy_(before[1])
        for t in (qr, out):
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for got, ref in zip((qr, out, kc, vc), want):
            assert torch.equal(got.view(torch.int16), ref.view(torch.int16))
    del g
    attn.close()


def test_sequences_that_share_pages():
    """Pages of a common beginning in the tables of several sequences."""
    bt = Batch(11, [600, 90, 333, 64], [20, 3, 40, 1], PAGE, HQ, HKV, gap=1)
    bt.table[1, :4] = bt.table[0, :4]
    bt.table[2, :17] = bt.table[0, :17]
    bt.table[3, :4] = bt.table[2, :4]
    kc, vc, table, lens = bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table), up_i32(bt.lens)
    kw = dict(window=200, prefix=[48, 33, 64, 5], softcap=20.0)
    sc = AttnScores(20.0, 200, None, up_i32(kw["prefix"]))
    ref = attention_reference(bt, SCALE, **kw)
    live = torch.tensor([at is not None for at in bt.row_of()])
    with DecodeAttention(HQ, HKV, 4, 600, page_tokens=PAGE) as attn:
        out = torch.empty((bt.rows, HQ, D), device=dev())
        attn.prefill_paged(bt.q.to(dev()), kc, vc, table, lens, up_i32(bt.starts), up_i32(bt.new), 40, SCALE, out, scores=sc)
        torch.cuda.synchronize()
        assert ((out.cpu().double() - ref)[live].abs() <= 9e-5).all()
        newest = [int(s) + m - 1 for s, m in zip(bt.starts, bt.new)]
        step = torch.empty((4, HQ, D), device=dev())
        attn.run_paged(bt.q[newest].to(dev()), kc, vc, table, lens, SCALE, step, scores=sc)
        torch.cuda.synchronize()
        assert ((step.cpu().double() - ref[newest]).abs() <= 9e-5).all()


def calls_of_a_handle(seed):
    """A prefill whose rows share their context out and a decode step, both through the workspace."""
    bt = Batch(seed, [3000, 700, 33], [3, 5, 1], PAGE, HQ, HKV)
    kc, vc, q = bt.k.to(dev()), bt.v.to(dev()), bt.q.to(dev())
    table, lens, starts, new = (up_i32(x) for x in (bt.table, bt.lens, bt.starts, bt.new))
    out, step = torch.empty((bt.rows, HQ, D), device=dev()), torch.empty((3, HQ, D), device=dev())
    attn = DecodeAttention(HQ, HKV, 3, 30000, page_tokens=PAGE)
    sc = AttnScores(softcap=25.0, window=2500)

    def prefill(stream=None):
        attn.prefill_paged(q, kc, vc, table, lens, starts, new, 5, SCALE, out, scores=sc, stream=stream)

    def decode(stream=None):
        attn.run_paged(q[:3], kc, vc, table, lens, SCALE, step, scores=sc, stream=stream)

    return attn, prefill, decode, out, step


def test_two_handles_on_two_streams():
    handles = [calls_of_a_handle(seed) for seed in (21, 22)]
    want = []
    for _, prefill, decode, out, step in handles:
        prefill()
        decode()
        torch.cuda.synchronize()
        want.append((out.clone(), step.clone()))
    streams = [torch.cuda.Stream() for _ in handles]
    for _ in range(5):
        for _, _, _, out, step in handles:
            out.fill_(float("nan"))
            step.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(3):
            for s, (_, prefill, decode, _, _) in zip(streams, handles):
                prefill(s)
                decode(s)
        torch.cuda.synchronize()
        for (_, _, _, out, step), (o, d) in zip(handles, want):
            assert torch.equal(out, o) and torch.equal(step, d)
    for h in handles:
        h[0].close()


def test_two_graphs_share_a_handle():
    """Prefill and decode captured into graphs of their own, replayed in turn with eager calls between."""
    from test_gpu_graphs import capture

    attn, prefill, decode, out, step = calls_of_a_handle(23)
    prefill()
    decode()
    torch.cuda.synchronize()
    want = out.clone(), step.clone()
    graphs = capture(prefill), capture(decode)
    for order in ((0, 1), (1, 0), (0, 0, 1), (1, 1, 0)):
        out.fill_(float("nan"))
        step.fill_(float("nan"))
        for i in order:
            graphs[i].replay()
            if order[0]:
                prefill()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(step, want[1])
    del graphs
    attn.close()
