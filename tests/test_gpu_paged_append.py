"""ctx_kv_append_run_paged against a plain 64-bit form: norm, rotation, packed
rows, strides, pages outside the cache, and what must stay as it was."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd import binding as bd
from paper_2609_36608_amd.binding import CtxError, DecodeAttention, Rotary

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, append_reference, randn

pytestmark = pytest.mark.gpu

# One rounding to bf16 is off by at most 2^-8 of the value.  Before it, in fp32: the
# norm's sum of 128 squares (7 + 4 additions), its square root and two products are
# within 2^-19 of each value; cosine and sine carry the fp32 rounding of an angle of
# up to half a turn (2^-26 turns, 2^-23 absolute) and their own 2 ulp; two products and
# a sum.  Together below 2^-17 of the sizes that enter a value.
ROUND, BEFORE = 2.0 ** -8, 2.0 ** -17


def bits(t):
    """The values' bits: equal means identical, NaN included."""
    return t.contiguous().view(torch.int16)


def inv_freq(rot, theta=1e6):
    return (theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float() if rot else torch.zeros(0)


def close(got, ref, size):
    err = (got.double() - ref).abs()
    bound = ROUND * (ref.abs() + BEFORE * size) + BEFORE * size
    worst = (err - bound).max().item()
    assert worst <= 0, f"worst excess {worst:.3e}"


def run(bt, q, k, v, rot=128, interleaved=False, positions=None, q_norm=None, k_norm=None, rows_given=True,
        in_place=False, eps=1e-6, stream=None):
    """Runs the call and checks queries, caches and everything that must not change."""
    up = lambda t: None if t is None else t.to(dev())  # noqa: E731
    f = inv_freq(rot)
    kc, vc = up(bt.k), up(bt.v)
    kd, vd, qd = up(k), up(v), up(q)
    q_out = None
    if q is not None:
        q_out = qd if in_place else torch.full((bt.rows, bt.hq, D), -777.0, dtype=torch.bfloat16, device=dev())
    rotary = Rotary(up(f) if rot else None, interleaved=interleaved, positions=up(positions), q_norm=up(q_norm),
                    k_norm=up(k_norm), norm_eps=eps)
    rows = dict(q_starts=up_i32(bt.starts), q_lens=up_i32(bt.new)) if rows_given else {}
    with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), max(max(bt.lens), 1), page_tokens=bt.page) as attn:
        got = attn.append_paged(kd, vd, kc, vc, up_i32(bt.table), up_i32(bt.lens), q=qd, q_out=q_out, rotary=rotary,
                                **rows)
        torch.cuda.synchronize()
    assert got is q_out
    rq, rk, rv, sq, sk = append_reference(bt, q, k, v, f.tolist(), interleaved, positions, q_norm, k_norm, eps)
    written = torch.zeros((bt.num_pages, bt.page), dtype=torch.bool)
    live = torch.zeros(bt.rows, dtype=torch.bool)
    for j, at in enumerate(bt.row_of()):
        if at is None:
            continue
        live[j] = True
        slot = bt.slot(*at)
        if slot is not None:
            written[slot] = True
    kc, vc = kc.cpu(), vc.cpu()
    close(kc[written], rk[written], sk[written])
    assert torch.equal(bits(vc[written]), bits(rv[written].to(torch.bfloat16)))
    for new, old in ((kc, bt.k), (vc, bt.v)):
        assert torch.equal(bits(new[~written]), bits(old[~written]))
    if q is not None:
        g = got.cpu()
        close(g[live], rq[live], sq[live])
        rest = q if in_place else torch.full_like(g, -777.0)
        assert torch.equal(bits(g[~live]), bits(rest[~live]))
    return kc, vc, q_out


def fused(bt, extra=0):
    """q, k, v as slices of the rows of one projection."""
    x = randn(bt.g, (bt.rows, (bt.hq + 2 * bt.hkv) * D + extra), 2.0)
    q, k, v = x[:, :x.shape[1] - extra].reshape(bt.rows, -1, D).split([bt.hq, bt.hkv, bt.hkv], 1)
    return x, q, k, v


HEADS = [(16, 8), (32, 8), (28, 4), (5, 1), (9, 3), (64, 4), (1, 1)]


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (64, False), (96, True), (16, False), (0, False)])
def test_heads_and_rotary_dimensions(hq, hkv, rot, interleaved):
    bt = Batch(hq * 100 + rot, [40, 1, 17, 16, 33, 0], [9, 1, 0, 16, 2, 0], 16, hq, hkv, gap=1)
    q, k, v = (randn(bt.g, (bt.rows, h, D), 2.0) for h in (hq, hkv, hkv))
    w = [1 + randn(bt.g, (D,), 0.2) for _ in range(2)]
    run(bt, q, k, v, rot, interleaved, q_norm=w[0], k_norm=w[1])


@pytest.mark.parametrize("norms", ["none", "q", "k", "both"])
@pytest.mark.parametrize("page", [16, 48, 64])
def test_norms_and_pages(norms, page):
    bt = Batch(7 + page, [page + 5, 3 * page, 2, 130], [page + 5, page + 1, 1, 70], page, 12, 2)
    q, k, v = (randn(bt.g, (bt.rows, h, D), 2.0) for h in (12, 2, 2))
    w = [1 + randn(bt.g, (D,), 0.2) for _ in range(2)]
    run(bt, q, k, v, 64, q_norm=w[0] if norms in ("q", "both") else None,
        k_norm=w[1] if norms in ("k", "both") else None, eps=1e-5)


def test_zero_rows_of_a_norm_and_large_ones():
    bt = Batch(3, [4], [4], 16, 8, 8)
    q, k, v = (randn(bt.g, (4, 8, D)) for _ in range(3))
    q[0] = 0
    k[1] = 0
    k[2] *= 2.0 ** 40
    q[3] *= 2.0 ** -30
    w = 1 + randn(bt.g, (D,), 0.2)
    run(bt, q, k, v, q_norm=w, k_norm=w, eps=1e-6)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    bt = Batch(11, [20, 30], [20, 30], 16, 16, 8)
    q, k, v = (randn(bt.g, (bt.rows, h, D)) for h in (16, 8, 8))
    pos = torch.randint(0, 1 << 24, (bt.rows,), generator=bt.g, dtype=torch.int32)
    pos[:4] = torch.tensor([0, 1, -5, 1 << 20])
    run(bt, q, k, v, positions=pos, interleaved=interleaved)


def test_single_token_form_and_slices_of_one_projection():
    lens = [1, 16, 17, 0, 300, 31, 33, 64, 5]
    for hq, hkv in ((32, 8), (7, 7)):
        bt = Batch(5, lens, [1 if n else 0 for n in lens], 16, hq, hkv)
        bt.starts = np.arange(len(lens), dtype=np.int32)
        bt.rows = len(lens)
        x, q, k, v = fused(bt, extra=8)
        w = 1 + randn(bt.g, (D,), 0.2)
        xd = x.to(dev())
        views = [xd.as_strided((bt.rows, h, D), (x.shape[1], D, 1), at * D)
                 for h, at in ((hq, 0), (hkv, hq), (hkv, hq + hkv))]
        run_views(bt, (q, k, v), views, w)


def run_views(bt, host, device, w):
    q, k, v = host
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    f = inv_freq(128)
    with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), max(bt.lens), page_tokens=bt.page) as attn:
        out = attn.append_paged(device[1], device[2], kc, vc, up_i32(bt.table), up_i32(bt.lens), q=device[0],
                                rotary=Rotary(f.to(dev()), q_norm=w.to(dev()), k_norm=w.to(dev())))
        torch.cuda.synchronize()
    rq, rk, rv, sq, sk = append_reference(bt, q, k, v, f.tolist(), q_norm=w, k_norm=w)
    ok = ~rk.isnan()
    close(kc.cpu()[ok], rk[ok], sk[ok])
    ok = ~rv.isnan()  # the slots that hold a token
    assert torch.equal(vc.cpu()[ok], rv[ok].to(torch.bfloat16)) and vc.cpu()[~ok].isnan().all()
    live = torch.tensor([n > 0 for n in bt.lens])
    close(out.cpu()[live], rq[live], sq[live])


def test_many_rows_and_many_sequences():
    """Enough rows for a wave per row, and more sequences than a wave has lanes."""
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 60, 300)
    new = np.minimum(lens, rng.integers(0, 60, 300))
    bt = Batch(17, lens, new, 16, 6, 2, gap=1)
    assert bt.rows > 4096
    _, q, k, v = fused(bt)
    w = 1 + randn(bt.g, (D,), 0.2)
    run(bt, q.contiguous(), k.contiguous(), v.contiguous(), q_norm=w, k_norm=w)


def test_in_place_queries_and_no_queries():
    bt = Batch(23, [50, 20], [33, 7], 16, 16, 8, gap=2)
    q, k, v = (randn(bt.g, (bt.rows, h, D)) for h in (16, 8, 8))
    run(bt, q, k, v, in_place=True)
    run(bt, None, k, v)
    kc, _, _ = run(bt, q, k, v, rot=0)  # neither norm nor rotation: copies
    for j, at in enumerate(bt.row_of()):
        if at is not None:
            assert torch.equal(bits(kc[bt.slot(*at)]), bits(k[j]))


def test_pages_outside_the_cache_take_nothing():
    bt = Batch(29, [70, 40, 100], [70, 40, 100], 16, 8, 2)
    bt.table[0, 1] = -1
    bt.table[0, 2] = bt.num_pages
    bt.table[1, 0] = 2 ** 31 - 1
    bt.table = np.ascontiguousarray(bt.table[:, :5])  # and tokens past the table
    q, k, v = (randn(bt.g, (bt.rows, h, D)) for h in (8, 2, 2))
    run(bt, q, k, v)


def test_more_new_tokens_than_tokens_or_rows_stays_in_bounds():
    """Broken batches: rows before position 0 and rows past the arrays are not touched."""
    bt = Batch(31, [3, 20], [3, 20], 16, 8, 2)
    k, v = (randn(bt.g, (bt.rows, 2, D)).to(dev()) for _ in range(2))
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        attn.append_paged(k, v, kc, vc, up_i32(bt.table), up_i32([3, 20]), q_starts=up_i32([0, 15]),
                          q_lens=up_i32([10, 100]))
        torch.cuda.synchronize()
    assert kc.isfinite().any()


def test_other_stream_and_refusals():
    bt = Batch(37, [20, 5], [2, 1], 16, 8, 2)
    q, k, v = (randn(bt.g, (bt.rows, h, D)).to(dev()) for h in (8, 2, 2))
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    table, lens, st, nl = up_i32(bt.table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new)
    f = inv_freq(128).to(dev())
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        rows = dict(q_starts=st, q_lens=nl)
        a = attn.append_paged(k, v, kc, vc, table, lens, q=q, rotary=Rotary(f), **rows)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        k2, v2 = bt.k.to(dev()), bt.v.to(dev())
        b = torch.empty_like(q)
        s.wait_stream(torch.cuda.current_stream())
        attn.append_paged(k, v, k2, v2, table, lens, q=q, q_out=b, rotary=Rotary(f), stream=s, **rows)
        torch.cuda.synchronize()
        assert torch.equal(bits(a), bits(b)) and torch.equal(bits(kc), bits(k2))
        call = lambda **kw: attn.append_paged(**{**dict(k=k, v=v, k_pages=kc, v_pages=vc, block_tables=table, seq_lens=lens, q=q, **rows), **kw})  # noqa: E731,E501
        with pytest.raises(TypeError):
            call(k=k.float())
        with pytest.raises(ValueError):
            call(v=v.cpu())
        with pytest.raises(ValueError):
            call(q=q[:, :4])
        with pytest.raises(ValueError):
            call(q_lens=None)
        with pytest.raises(ValueError):
            call(q_starts=None, q_lens=None)  # as many rows as sequences then
        with pytest.raises(ValueError):
            call(k_pages=kc[:, :8].contiguous())
        with pytest.raises(ValueError):
            call(q=None, q_out=torch.empty_like(q))
        with pytest.raises(ValueError):
            call(k=k.transpose(1, 2).contiguous().transpose(1, 2))
        with pytest.raises(ValueError):
            call(rotary=Rotary(f, positions=lens[:1]))
        for kw, status in ((dict(inv_freq=f[:7].clone()), bd.CTX_ERR_UNSUPPORTED),
                           (dict(inv_freq=inv_freq(160).to(dev())), bd.CTX_ERR_UNSUPPORTED),
                           (dict(q_norm=bits(q[0, 0]).view(torch.bfloat16), norm_eps=float("nan")), bd.CTX_ERR_INVALID_ARG)):
            with pytest.raises(CtxError) as e:
                call(rotary=Rotary(**kw))
            assert e.value.status == status
    with DecodeAttention(8, 2, 2, 32) as plain, pytest.raises(ValueError):
        plain.append_paged(k, v, kc, vc, table, lens, **rows)


def test_graph_replays():
    from test_gpu_graphs import capture, replay_and_check

    bt = Batch(41, [80, 33], [50, 1], 16, 16, 8)
    q, k, v = (randn(bt.g, (bt.rows, h, D)).to(dev()) for h in (16, 8, 8))
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    table, lens, st, nl, f = up_i32(bt.table), up_i32(bt.lens), up_i32(bt.starts), up_i32(bt.new), inv_freq(128).to(dev())
    out = torch.empty_like(q)
    attn = DecodeAttention(16, 8, 2, 80, page_tokens=16)

    def call(stream=None):
        attn.append_paged(k, v, kc, vc, table, lens, q=q, q_out=out, q_starts=st, q_lens=nl, rotary=Rotary(f), stream=stream)

    call()
    torch.cuda.synchronize()
    expected = [out.clone(), kc.clone(), vc.clone()]
    g = capture(call)
    replay_and_check(g, [out], expected[:1], lambda t: t.fill_(float("nan")), call)
    assert torch.equal(bits(kc), bits(expected[1])) and torch.equal(bits(vc), bits(expected[2]))
    del g
    attn.close()
