"""More of ctx_kv_append_run_paged: lengths below zero."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import DecodeAttention, Rotary

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, randn
from test_gpu_paged_append import bits, inv_freq

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
