"""Bounds that do not fit the C interface's 32 bits: refused, not wrapped round to another call."""
import pytest
import torch

from paper_2609_36608_amd.binding import AttnScores, DecodeAttention

from _gpu_util import dev, up_i32
from _paged_util import D, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bound", [2 ** 31, 2 ** 32, 2 ** 32 + 3])
def test_numbers_past_32_bits(bound):
    bt = Batch(3, [20, 5], [20, 5], 16, 8, 2)
    q, kc, vc = bt.q.to(dev()), bt.k.to(dev()), bt.v.to(dev())
    table, lens, st, nl = (up_i32(x) for x in (bt.table, bt.lens, bt.starts, bt.new))
    out = torch.empty((bt.rows, 8, D), device=dev())
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        with pytest.raises(ValueError):
            attn.prefill_paged(q, kc, vc, table, lens, st, nl, bound, 0.1, out)
        with pytest.raises(ValueError):
            attn.prefill_paged(q, kc, vc, table, lens, st, nl, 20, 0.1, out, scores=AttnScores(window=bound))
        with pytest.raises(ValueError):
            attn.run_paged(q[:2], kc, vc, table, lens, 0.1, out[:2], scores=AttnScores(window=bound))
        with pytest.raises(ValueError):
            attn.prefill(q, kc[0], vc[0], lens, lens, st, nl, bound, 0.1, out)
        torch.cuda.synchronize()
