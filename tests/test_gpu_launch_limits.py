"""The largest launches: as many rows as a launch has workgroups of 256 threads for."""
import pytest
import torch

from paper_2609_36608_amd import token_logprobs, token_logprobs_grad

pytestmark = pytest.mark.gpu


def test_the_most_rows_of_log_probabilities():
    rows, vocab = 2 ** 24 - 1, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((rows, vocab), generator=g, device="cuda", dtype=torch.bfloat16)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    r = token_logprobs(z, tokens)
    grad = token_logprobs_grad(z, tokens, r, torch.ones(rows, device="cuda"))
    u = 2.0 ** -24  # of sums of 8, each within a few roundings; values up to 2^4
    for part in torch.arange(rows, device="cuda").split(1 << 21):
        logp = torch.log_softmax(z[part].double(), -1)
        at = tokens[part].long()[:, None]
        assert (r["token_logp"][part].double() - logp.gather(1, at)[:, 0]).abs().max() <= 16 * 64 * u
        assert (r["entropy"][part].double() + (logp.exp() * logp).sum(-1)).abs().max() <= 16 * 64 * u
        want = -logp.exp()
        want.scatter_add_(1, at, torch.ones_like(want[:, :1]))
        # bf16's half step of the value and of what it was rounded from
        assert ((grad[part].double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 16 * 64 * u).all()
    with pytest.raises(Exception, match="num_rows"):
        token_logprobs(z[:1].expand(rows + 1, vocab).contiguous())
