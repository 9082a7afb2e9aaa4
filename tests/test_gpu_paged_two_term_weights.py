"""The paged prefill with bf16 outputs and CTX_SCORES_SPLIT_P: softmax weights as two bf16 terms, in
every kind of workgroup and with every kind of score."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import AttnScores, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, attention_reference, randn
from test_gpu_paged_prefill import F32, KINDS, SCALE, kind_batch, kind_of, scores_of, slopes_of

pytestmark = pytest.mark.gpu

# Each bf16 rounding is off by at most u = 2^-8: the second term's is u of what the first left,
# u^2 of the weight together.  The row sum adds the unrounded weights, so an output moves by at
# most u^2 times the weighted mean of |value| <= spread + |output|, beside F32 (logits and sums
# of the fp32 outputs' tests); then half a step of the output.
U = 2.0 ** -8


def run(bt, split_p=True, max_seq_len=None, softcap=0.0, window=0, slopes=None, prefix=None, docs=None):
    up = lambda t: None if t is None else up_i32(t)  # noqa: E731
    out = torch.full((bt.rows, bt.hq, D), -777.0, dtype=torch.bfloat16, device=dev())
    scores = AttnScores(softcap, window, None if slopes is None else slopes.to(dev()), up(prefix), up(docs),
                        split_p=split_p)
    with DecodeAttention(bt.hq, bt.hkv, len(bt.lens), max_seq_len or max(max(bt.lens), 1), page_tokens=bt.page,
                         out_dtype=torch.bfloat16) as attn:
        attn.prefill_paged(bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table), up_i32(bt.lens),
                           up_i32(bt.starts), up_i32(bt.new), max(bt.new), SCALE, out, scores=scores)
        torch.cuda.synchronize()
    live = torch.tensor([at is not None for at in bt.row_of()])
    assert (out.cpu()[~live] == -777.0).all()
    return out.cpu()[live].double(), live


def excess(got, ref, spread):
    """The largest error less its bound."""
    bound = F32 + U * U * (spread + ref.abs())
    return ((got - ref).abs() - (bound + U * (ref.abs() + bound))).max().item()


def check(bt, max_seq_len=None, **kw):
    got, live = run(bt, max_seq_len=max_seq_len, **kw)
    ref, spread = attention_reference(bt, SCALE, spread=True, **kw)
    assert got.isfinite().all()
    assert excess(got, ref[live], spread[live]) <= 0
    return got, ref[live], spread[live]


# two column tiles per wave at most, as with fp32 outputs
TWO_TERMS = {"wide1": ("wide", 1), "wide2": ("wide", 2), "wide3": ("wide", 2), "narrow4": ("narrow", 4),
             "narrow8": ("narrow", 8)}


@pytest.mark.parametrize("scores", KINDS)
@pytest.mark.parametrize("kind", list(TWO_TERMS))
def test_scores_and_masks(kind, scores):
    bt, bound = kind_batch(kind)
    assert kind_of(bt, torch.float32, bound) == TWO_TERMS[kind]
    if scores == "cap":
        bt.q = randn(bt.g, bt.q.shape, 4.0)
    kw = scores_of(scores, bt, np.random.default_rng(4))
    got, ref, spread = check(bt, bound, **kw)
    if scores == "none":  # which weights of one term do not keep to
        one, _ = run(bt, split_p=False, max_seq_len=bound)
        assert excess(one, ref, spread) > 0


@pytest.mark.parametrize("scores", ["none", "capbias", "prefix"])
def test_contexts_shared_out(scores):
    bt = Batch(53, [3000, 5, 33, 700, 0, 1200], [3, 5, 1, 2, 0, 4], 16, 16, 8, gap=1)
    check(bt, 30000, **scores_of(scores, bt, np.random.default_rng(8)))


@pytest.mark.parametrize("hq,hkv", [(28, 4), (16, 1), (9, 3), (1, 1)])
def test_heads_and_pages(hq, hkv):
    bt = Batch(hq, [1, 48, 49, 151, 100], [1, 48, 5, 78, 33], 48, hq, hkv, gap=1)
    check(bt, softcap=20.0, window=50, slopes=slopes_of(hq), prefix=[0, 3, 48, 17, 40])
    check(bt, 600)


def test_fp32_outputs_and_decode_steps_do_not_change():
    bt = Batch(61, [300, 40, 9], [40, 40, 1], 16, 16, 8)
    args = [t.to(dev()) for t in (bt.q, bt.k, bt.v)] + [up_i32(t) for t in (bt.table, bt.lens)]
    with DecodeAttention(16, 8, 3, 300, page_tokens=16) as attn:
        outs = [attn.prefill_paged(*args, up_i32(bt.starts), up_i32(bt.new), 40, SCALE,
                                   torch.empty((bt.rows, 16, D), device=dev()), scores=AttnScores(split_p=s))
                for s in (False, True)]
        steps = [attn.run_paged(args[0][:3].contiguous(), *args[1:], SCALE, torch.empty((3, 16, D), device=dev()),
                                scores=AttnScores(split_p=s)) for s in (False, True)]
        torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(steps[0], steps[1])


@pytest.mark.parametrize("softcap", [512.5, 1e5])
@pytest.mark.parametrize("biased", [False, True])
def test_large_caps_take_two_terms_in_every_kind_of_call(softcap, biased):
    """Few rows over a long context, shared out, and many over a short one."""
    for bt, bound in ((Batch(67, [1500, 700], [5, 33], 16, 16, 8), 20000), kind_batch("wide1"), kind_batch("narrow4")):
        kw = dict(softcap=softcap, slopes=slopes_of(16) if biased else None)
        ref, spread = attention_reference(bt, SCALE, spread=True, **kw)
        got, live = run(bt, split_p=False, max_seq_len=bound, **kw)
        assert excess(got, ref[live], spread[live]) <= 0
        assert torch.equal(got, run(bt, max_seq_len=bound, **kw)[0])
