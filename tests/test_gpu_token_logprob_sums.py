"""The running sums of the token log probabilities where many tiles of a row meet and the largest logit
times the scale is far from 0: neither may drift with the number of tiles nor with the offset.

Tolerances, with u = 2^-24 (fp32's half step).  d = (x - max) log2 e of an entry is off by 3 u (|d| + 1/2): the
scale, its factor in log2 units and the one rounding of the difference, whose origin is the largest product
rounded, half a step of at most 2^24 off.  A sum is rounded once for each of a tile's 4 chunks of E logits, once
for each of a lane's K tiles and at most 16 times in the joins of lanes, waves and shares; at each of K + 3 raises of
the maximum the sums are scaled by an exp2 (2 u, and u x 2^-x < u of the whole for a difference of x) and rounded:
4 u.  That is c = 4 E + K + 16 + 4 (K + 3).  With D1 = sum p (|d| + 1/2) and D2 = sum p (|d| + 1/2)^2:
  log s     c u + 3 u D1 + 4 u, and 2 u (|log s| + 1/2) for the logarithm
  logp      that, and 3 u (|d_t| + 1/2) + 2 u |logp|
  entropy   that of log s, and (c + 8) u D1 + 4 u D2 + 2 u H
  p         that of log s and 3 u (|d| + 1/2) + 6 u, relative
None of them grows with the offset.
"""
import math

import pytest
import torch

from paper_2609_36608_amd import token_logprobs, token_logprobs_grad

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
VOCAB = 151936
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Exact:
    """In 64 bits, on the device, of the logits as they are."""

    def __init__(self, logits, temperature):
        z = logits.double()
        z = torch.where(z <= -1e38, -math.inf, z) / temperature
        self.temperature = temperature
        self.logp = torch.log_softmax(z, -1)
        self.p = self.logp.exp()
        self.lp = self.logp.clamp(min=-200)
        self.h = -(self.p * self.lp).sum(-1)
        self.d = ((z - z.amax(-1, keepdim=True)) / math.log(2)).abs().clamp(max=1e30) + 0.5
        near = self.d.clamp(max=1100)  # beyond, p is 0
        self.d1, self.d2 = (self.p * near).sum(-1), (self.p * near * near).sum(-1)
        self.s = (z - z.amax(-1, keepdim=True)).exp().sum(-1)
        e = 16 // logits.element_size()
        k = -(-z.shape[1] // (4 * 4 * 64 * e))
        c = 4 * e + k + 16 + 4 * (k + 3)
        self.log_tol = U * (c + 3 * self.d1 + 4 + 2 * (self.s.log().abs() + 0.5))
        self.h_tol = self.log_tol + U * ((c + 8) * self.d1 + 4 * self.d2 + 2 * self.h)

    def logp_of(self, tokens):
        """Values and tolerances."""
        lp, d = self.logp.gather(1, tokens), self.d.gather(1, tokens)
        return lp, self.log_tol[:, None] + U * (3 * d + 2 * lp.abs())

    def grad(self, tokens, by, by_h):
        a, b = by.double(), by_h.double()[:, None]
        p_tol = self.log_tol[:, None] + U * (3 * self.d.clamp(max=1100) + 6)
        inner = a.sum(1, keepdim=True) + b * (self.lp + self.h[:, None])
        size = a.abs().sum(1, keepdim=True) + b.abs() * (self.lp.abs() + self.h[:, None])
        g = -self.p * inner
        g.scatter_add_(1, tokens, a)
        off = self.p * (size * (p_tol + 8 * U) + b.abs() * (p_tol + self.h_tol[:, None]))
        off = off + 4 * U * (self.p * size + g.abs()) + 2.0 ** -126 * size  # smaller powers of 2 are 0
        return g / self.temperature, off / self.temperature


def within(got, want, tol, what):
    err = torch.where(got.double() == want, 0.0, (got.double() - want).abs())
    worst = (err / tol.clamp(min=1e-300)).max().item()
    print(f"{what}: error {err.max().item():.3e}, {worst:.3f} of the tolerance", flush=True)
    assert (err <= tol).all(), what


def check(z, copies, temperature):
    """Rows z, each `copies` times in the call: few rows are cut into shares, many are not."""
    rows, vocab = z.shape
    wide = z.repeat(copies, 1)
    e = Exact(z, temperature)
    g = torch.Generator().manual_seed(5)
    # a largest one, the smallest and two others
    tokens = torch.cat([z.double().argmax(1, keepdim=True), z.double().argmin(1, keepdim=True),
                        torch.randint(0, vocab, (rows, 2), generator=g).cuda()], 1)
    given = tokens.int().repeat(copies, 1).contiguous()
    r = token_logprobs(wide, given, temperature=temperature, top=3)
    for name, x in r.items():  # a row's results are those of its copies
        assert torch.equal(x, x[:rows].repeat(*([copies] + [1] * (x.dim() - 1)))), name
    part = {k: x[:rows] for k, x in r.items()}
    within(part["token_logp"], *e.logp_of(tokens), "logp")
    within(part["top_logp"], *e.logp_of(part["top_tokens"].long()), "top logp")
    within(part["entropy"], e.h, e.h_tol, "entropy")
    assert torch.equal(z.gather(1, part["top_tokens"][:, :1].long()), z.gather(1, tokens[:, :1]))
    by, by_h = torch.randn(rows, 4, generator=g).cuda(), torch.randn(rows, generator=g).cuda()
    for with_h in (True, False):
        h = by_h if with_h else torch.zeros_like(by_h)
        grad = token_logprobs_grad(wide, given, r, by.repeat(copies, 1), temperature=temperature,
                                   grad_entropy=h.repeat(copies) if with_h else None)[:rows]
        want, off = e.grad(tokens, by, h)
        eps = torch.finfo(z.dtype).eps / 2
        within(grad, want, off + eps * (want.abs() + off) + torch.finfo(z.dtype).tiny, "gradient")


CASES = [("f32", 0.0, 0.05), ("f32", 0.0, 1e-3), ("f32", 0.0, 1e-5), ("f32", 1e3, 1.0), ("f32", -1e3, 1.0),
         ("f32", 1e5, 1.0), ("f32", -1e5, 0.7), ("f32", 1e7, 1.0), ("f32", -1e7, 1.0), ("f32", 1e9, 1.0),
         ("bf16", 0.0, 0.05), ("bf16", 0.0, 1e-3), ("bf16", 3000.0, 0.7), ("bf16", -1e5, 1.0)]


@pytest.mark.parametrize("copies", [1, 700], ids=["shares", "whole rows"])
@pytest.mark.parametrize("dtype,offset,temperature", CASES)
def test_many_tiles(dtype, offset, temperature, copies):
    g = torch.Generator().manual_seed(17)
    std = max(2.5, abs(offset) / (2e7 if dtype == "f32" else 200))
    z = (torch.randn(3, VOCAB, generator=g) * std + offset).to(DTYPES[dtype]).cuda()
    check(z, copies, temperature)


@pytest.mark.parametrize("dtype,offset", [("f32", 1e7), ("f32", -1e7), ("f32", 1e5), ("bf16", 3000.0)])
@pytest.mark.parametrize("copies", [1, 700], ids=["shares", "whole rows"])
@pytest.mark.parametrize("vocab", [16384, VOCAB])
def test_lanes_with_masked_logits_alone(vocab, copies, dtype, offset):
    """Lanes whose every logit is masked, beside others of the same wave: each lane's terms, and what is
    taken from their sums, count from the same number."""
    g = torch.Generator().manual_seed(18)
    std = max(2.5, abs(offset) / (2e7 if dtype == "f32" else 200))
    z = torch.randn(3, vocab, generator=g) * std + offset
    lane = torch.arange(vocab) // (16 // DTYPES[dtype].itemsize) % 64
    z[0, lane % 2 == 0] = -math.inf
    z[1, lane != 5] = torch.finfo(torch.bfloat16).min
    z[2, lane == 63] = -1e38 * 1.01
    z[2, :vocab // 2] = -math.inf
    check(z.to(DTYPES[dtype]).cuda(), copies, 1.0)


def test_products_either_side_of_the_large_ones():
    """Lanes whose largest products lie on either side of 2^24, where differences to them are taken
    in another way, in one wave and in one lane's tiles."""
    g = torch.Generator().manual_seed(19)
    at = 2.0 ** 24 * math.log(2)
    for sign in (1, -1):
        z = (sign * at + torch.randn(3, VOCAB, generator=g) * 8).float()
        z[1] = sign * at + (torch.arange(VOCAB) % 64 - 32).float() * 0.5
        z[2] = sign * at + (torch.arange(VOCAB) // 4096 - 18).float()
        check(z.cuda(), 1, 1.0)
        check(z.cuda(), 700, 1.0)


def test_masked_logits_near_the_others():
    """The least scale and logits just above the masked ones."""
    z = torch.full((3, 4100), -1e38)
    z[:, 7] = torch.nextafter(torch.tensor(-1e38), torch.tensor(0.0))
    z[1, 9] = z[1, 7]
    z[2, 4099] = -9.9e37
    z = z.cuda()
    r = token_logprobs(z, torch.tensor([7, 9, 3], dtype=torch.int32).cuda(), temperature=1e30, top=3)
    assert r["top_tokens"].tolist() == [[7, -1, -1], [7, 9, -1], [4099, 7, -1]]
    ln2 = math.log(2)
    # [2]: column 7 is 1e36 below, 1e6 in scaled units
    assert abs(r["token_logp"][0].item()) <= 4 * U and abs(r["token_logp"][1].item() + ln2) <= 8 * U
    assert r["token_logp"][2] == -math.inf
    assert abs(r["entropy"][0].item()) <= 4 * U and abs(r["entropy"][1].item() - ln2) <= 8 * U and r["entropy"][2] == 0
    by = torch.ones(3).cuda()
    grad = token_logprobs_grad(z, torch.tensor([7, 7, 4099], dtype=torch.int32).cuda(), r, by, temperature=1e30)
    grad = grad.double().cpu() * 1e30
    want = torch.zeros(3, 4100, dtype=torch.float64)
    want[1, 7], want[1, 9] = 0.5, -0.5
    assert ((grad - want).abs() <= 16 * U).all()


@pytest.mark.parametrize("copies", [1, 700], ids=["shares", "whole rows"])
@pytest.mark.parametrize("dtype,offset,temperature", CASES)
def test_stats(dtype, offset, temperature, copies):
    """The largest logit, and the sum of exp(x - scale * that) of the row."""
    g = torch.Generator().manual_seed(20)
    std = max(2.5, abs(offset) / (2e7 if dtype == "f32" else 200))
    z = (torch.randn(3, VOCAB, generator=g) * std + offset).to(DTYPES[dtype]).cuda()
    e = Exact(z, temperature)
    stats = token_logprobs(z.repeat(copies, 1), temperature=temperature)["stats"][:3]
    assert torch.equal(stats[:, 0], z.float().amax(1))
    # its logarithm is off as log s is, and by an exp2 and a product more
    within(stats[:, 1].double().log(), e.s.log(), e.log_tol + 4 * U, "log of the sum")
    # a row's log sum exp follows from them
    x = z.double() / temperature
    lse = stats[:, 0].double() / temperature + stats[:, 1].double().log()
    within(lse - x.amax(1), torch.logsumexp(x - x.amax(1, keepdim=True), 1), e.log_tol + 4 * U, "log sum exp")
