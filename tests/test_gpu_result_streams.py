"""Results that a call allocates belong to the stream that it runs on: dropped before that stream
is done, their memory is not given to another one."""
import pytest
import torch

from paper_2609_36608_amd.binding import DecodeAttention, opd_loss

from _gpu_util import dev, up_i32
from _paged_util import D, Batch, randn

pytestmark = pytest.mark.gpu


def given_away(make):
    """Whether a tensor of the current stream gets the memory of make()'s result, dropped just before."""
    t = make()
    torch.cuda.synchronize()
    at, like = t.data_ptr(), t.shape
    del t
    return torch.empty(like, dtype=torch.bfloat16, device=dev()).data_ptr() == at


@pytest.mark.parametrize("raw", [False, True])
def test_append(raw):
    bt = Batch(3, [20, 5], [20, 5], 16, 8, 2)
    q, k, v = (randn(bt.g, (bt.rows, h, D)).to(dev()) for h in (8, 2, 2))
    kc, vc = bt.k.to(dev()), bt.v.to(dev())
    args = k, v, kc, vc, up_i32(bt.table), up_i32(bt.lens)
    rows = dict(q_starts=up_i32(bt.starts), q_lens=up_i32(bt.new))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        here = attn.append_paged(*args, q=q, **rows)
        there = attn.append_paged(*args, q=q, stream=s.cuda_stream if raw else s, **rows)
        torch.cuda.synchronize()
        assert torch.equal(here, there)
        del there
        assert not given_away(lambda: attn.append_paged(*args, q=q, stream=s.cuda_stream if raw else s, **rows))
        assert given_away(lambda: attn.append_paged(*args, q=q, **rows))  # its own stream's, in order


def test_the_default_stream_by_its_handle():
    bt = Batch(5, [20, 5], [20, 5], 16, 8, 2)
    q, k, v = (randn(bt.g, (bt.rows, h, D)).to(dev()) for h in (8, 2, 2))
    args = k, v, bt.k.to(dev()), bt.v.to(dev()), up_i32(bt.table), up_i32(bt.lens)
    rows = dict(q_starts=up_i32(bt.starts), q_lens=up_i32(bt.new))
    assert torch.cuda.default_stream().cuda_stream == 0
    torch.cuda.synchronize()
    with DecodeAttention(8, 2, 2, 32, page_tokens=16) as attn:
        assert given_away(lambda: attn.append_paged(*args, q=q, stream=0, **rows))
        with torch.cuda.stream(torch.cuda.Stream()):
            assert not given_away(lambda: attn.append_paged(*args, q=q, stream=0, **rows))


def test_opd_loss():
    n, vocab = 64, 40000  # a gradient too large for a block of the allocator's small ones
    logits = torch.randn((n, vocab), device=dev()).to(torch.bfloat16)
    args = (logits, torch.arange(n, dtype=torch.int32, device=dev()), torch.full((n,), -12.0, device=dev()),
            torch.full((n,), -11.0, device=dev()), torch.ones(n, dtype=torch.uint8, device=dev()), up_i32([0, 20, n]))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert not given_away(lambda: opd_loss(*args, stream=s)["grad_logits"])
    assert given_away(lambda: opd_loss(*args)["grad_logits"])
    here, there = opd_loss(*args), opd_loss(*args, stream=s)
    torch.cuda.synchronize()
    for name in here:
        assert torch.equal(here[name], there[name])
