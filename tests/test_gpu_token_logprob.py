"""Token log probabilities, entropy, alternatives and their gradient against 64 bits.

Tolerances, with u = 2^-24 (fp32's half step) and d = (x - max) log2 e of an entry: the difference, the
factor and the product put d off by 3 u |d|, so 2^d by 3 u |d| ln 2 + 2 u of itself (exp2 is good to a
step); a lane adds V / 256 terms and at most 64 more on its way (the tile's ends, the joins), each sum
off by u.  With n = V / 256 + 64 and the means D1 = sum p |d|, D2 = sum p d^2:
  log s       n u + 3 u D1 + 4 u               (natural units, and 2 u |log s| for the logarithm itself)
  logp        that, and 3 u |d_t| + 2 u |logp|
  entropy     that, (n + 6) u H-like from t / s: (n + 8) u D1 + 4 u D2
  gradient    of p: (3 |d| + n + 3 D1 + 10) u relative; half a step of the type once rounded
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_36608_amd import token_logprobs, token_logprobs_grad
from paper_2609_36608_amd import binding as bd

pytestmark = pytest.mark.gpu
U = 2.0 ** -24  # and 2^-8 in bf16, which has 8 significant bits


def logits_of(seed, rows, vocab, dtype, std=2.5, wide=None):
    """Rows apart by a multiple of 16 bytes, NaN behind them."""
    g = torch.Generator().manual_seed(seed)
    wide = (vocab + 7) // 8 * 8 if wide is None else wide
    z = torch.full((rows, wide), float("nan"))
    z[:, :vocab] = torch.randn(rows, vocab, generator=g) * std
    return z.to(dtype).cuda()[:, :vocab]


class Exact:
    def __init__(self, logits, temperature=1.0):
        z = logits.double().cpu()
        z = torch.where(z <= -1e38, -math.inf, z) / temperature
        self.logp = torch.log_softmax(z, -1)
        self.p = self.logp.exp()
        plogp = torch.where(self.p > 0, self.p * self.logp, 0.0)
        self.h = -plogp.sum(-1)
        d = ((z - z.amax(-1, keepdim=True)) / math.log(2)).clamp(min=-200)
        self.d = d
        self.d1, self.d2 = (self.p * d.abs()).sum(-1), (self.p * d * d).sum(-1)
        n = z.shape[1] / 256 + 64
        log_s = (-(self.d[..., :1]) * 0)[..., 0] + torch.exp2(d).sum(-1).log()
        self.log_tol = U * (n + 3 * self.d1 + 4 + 2 * log_s.abs())
        self.h_tol = self.log_tol + U * ((n + 8) * self.d1 + 4 * self.d2 + 2 * self.h)
        self.p_tol = U * (3 * d.abs() + n + 3 * self.d1[:, None] + 10)

    def logp_tol(self, tokens):
        d, lp = self.d.gather(1, tokens).abs(), self.logp.gather(1, tokens).abs()
        return self.log_tol[:, None] + U * (3 * d + 2 * lp)

    def grad(self, tokens, by, by_h, temperature, mask=None):
        """Value and what it may be off by, before the rounding to the logits' type."""
        a = by.double().cpu() if by is not None else torch.zeros(self.p.shape[0], 1, dtype=torch.float64)
        b = by_h.double().cpu()[:, None] if by_h is not None else torch.zeros(self.p.shape[0], 1, dtype=torch.float64)
        lp = self.logp.clamp(min=-200)
        inner = a.sum(1, keepdim=True) + b * (lp + self.h[:, None])
        size = a.abs().sum(1, keepdim=True) + b.abs() * (lp.abs() + self.h[:, None])
        g = -self.p * inner
        if by is not None:
            g.scatter_add_(1, tokens, a)
        off = self.p * size * (self.p_tol + 70 * U) + self.p * b.abs() * (self.h_tol + self.log_tol)[:, None]
        off += U * 2 * g.abs() + (U * 4 * a.abs().sum(1, keepdim=True) if by is not None and tokens.shape[1] > 1 else 0)
        g, off = g / temperature, off / temperature
        if mask is not None:
            off = off * (mask.cpu() != 0)[:, None]
            g = g * (mask.cpu() != 0)[:, None]
        return g, off


def check_top(logits, r, top, rows=None):
    """Columns are those of a stable sort, by value and then by column."""
    z = logits.double().cpu() + 0.0
    want = z.sort(dim=-1, descending=True, stable=True).indices[:, :top].int()
    got = r["top_tokens"].cpu()
    k = want.shape[1]
    rows = range(z.shape[0]) if rows is None else rows
    for j in rows:
        assert torch.equal(got[j, :k], want[j]), (j, got[j], want[j])
        assert (got[j, k:] == -1).all() and (r["top_logp"][j, k:].cpu() == -math.inf).all()


def within(got, want, tol, what):
    err = (got.double().cpu() - want).abs()
    worst = (err / tol.clamp(min=1e-300)).max().item() if err.numel() else 0.0
    print(f"{what}: error {err.max().item() if err.numel() else 0:.3e}, {worst:.3f} of the tolerance", flush=True)
    assert (err <= tol).all(), what


SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (2, 255), (9, 1000), (3, 2049), (2, 8191), (3, 50257), (2, 151936), (130, 4099),
          (1100, 517), (1030, 12944)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_against_64_bits(rows, vocab, dtype):
    temperature, m, top = [(1.0, 1, 5), (0.7, 3, 64), (1.5, 64, 1)][vocab % 3]
    z = logits_of(vocab, rows, vocab, dtype)
    g = torch.Generator().manual_seed(rows)
    tokens = torch.randint(0, vocab, (rows, m), generator=g)
    given = tokens.int().cuda()
    r = token_logprobs(z, given if m > 1 else given[:, 0].contiguous(), temperature=temperature, top=top)
    e = Exact(z, temperature)
    within(r["token_logp"].view(rows, m), e.logp.gather(1, tokens), e.logp_tol(tokens), "logp")
    within(r["entropy"], e.h, e.h_tol, "entropy")
    check_top(z, r, top)
    at = r["top_tokens"].long().cpu().clamp(min=0)
    k = min(top, vocab)
    within(r["top_logp"][:, :k], e.logp.gather(1, at)[:, :k], e.logp_tol(at)[:, :k], "top logp")

    by = torch.randn(rows, m, generator=g).cuda()
    by_h = torch.randn(rows, generator=g).cuda() if vocab % 2 else None
    shaped = by if m > 1 else by[:, 0].contiguous()
    grad = token_logprobs_grad(z, given if m > 1 else given[:, 0].contiguous(), r, shaped, grad_entropy=by_h,
                               temperature=temperature)
    assert grad.dtype == dtype and grad.shape == z.shape
    want, off = e.grad(tokens, by, by_h, temperature)
    eps = torch.finfo(dtype).eps / 2
    within(grad, want, off + eps * (want.abs() + off) + torch.finfo(dtype).tiny, "gradient")


@pytest.mark.parametrize("rows", [2, 1200])
def test_parts_of_a_call(rows):
    """Without tokens, entropy or alternatives; each part has the same bits as in a whole call."""
    z = logits_of(3, rows, 9001, torch.bfloat16)
    tokens = torch.arange(rows, dtype=torch.int32).cuda()
    whole = token_logprobs(z, tokens, top=7)
    for kw in (dict(top=7), dict(top=0), dict(top=0, entropy=False), dict(top=7, entropy=False)):
        for given in (tokens, None):
            r = token_logprobs(z, given, **kw)
            names = {"stats"} | ({"token_logp"} if given is not None else set())
            names |= ({"entropy"} if kw.get("entropy", True) else set()) | ({"top_tokens", "top_logp"} if kw["top"] else set())
            assert set(r) == names
            for name in names:
                assert torch.equal(r[name], whole[name]), (kw, name)
    none = token_logprobs(z, torch.zeros((rows, 0), dtype=torch.int32).cuda())
    assert "token_logp" not in none and torch.equal(none["entropy"], whole["entropy"])


@pytest.mark.parametrize("rows,vocab", [(1, 60000), (7, 151936), (1500, 20000)])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "coarse", "one wave", "zeros"])
def test_alternatives_wherever_they_lie(kind, rows, vocab):
    if kind == "rising":  # every value passes what was met before
        z = torch.arange(vocab).float().expand(rows, -1) * 1e-3
    elif kind == "falling":
        z = -torch.arange(vocab).float().expand(rows, -1) * 1e-3
    elif kind == "equal":
        z = torch.full((rows, vocab), -3.0)
    elif kind == "coarse":
        z = torch.randint(-3, 4, (rows, vocab), generator=torch.Generator().manual_seed(1)).float()
    elif kind == "one wave":
        z = torch.zeros(rows, vocab)
        z[:, 5000:5100] = torch.arange(100).float()
    else:  # of both signs, which are equal
        z = torch.zeros(rows, vocab)
        z[:, ::3] = -0.0
        z[:, 17] = -1.0
    wide = torch.zeros(rows, (vocab + 7) // 8 * 8)
    wide[:, :vocab] = z
    wide = wide.cuda()[:, :vocab]
    for top in (1, 20, 64):
        r = token_logprobs(wide, top=top, entropy=False)
        check_top(wide, r, top, rows=[0, rows - 1])
        assert torch.equal(r["top_tokens"], r["top_tokens"][:1].expand(rows, -1)) or kind == "coarse"


LOWEST = {torch.bfloat16: torch.finfo(torch.bfloat16).min, torch.float32: torch.finfo(torch.float32).min}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(12, 700), (12, 40000), (1212, 700)])
def test_masked_logits_and_rows(rows, vocab, dtype):
    inf, low = math.inf, LOWEST[dtype]
    z = logits_of(5, rows, vocab, dtype)
    z[0, 3:] = -inf                 # three alternatives
    z[1, 5:] = low
    z[2] = -inf                     # none
    z[3] = low
    z[4, 600] = math.nan
    z[5, 699] = inf
    z[6, ::2] = -inf
    z[7] = low
    z[7, 123] = -2.0                # one
    z[8, :] = -inf
    z[8, 9] = low
    tokens = torch.full((rows, 3), 4, dtype=torch.int32)
    tokens[:, 1] = -1
    tokens[:, 2] = vocab + 5
    tokens[7, 0] = 123
    mask = torch.ones(rows, dtype=torch.uint8)
    mask[9] = 0
    z[9] = math.nan                 # not read
    tokens, mask = tokens.cuda(), mask.cuda()
    r = {k: v.cpu() for k, v in token_logprobs(z, tokens, mask=mask, top=6).items()}
    lp, h, at, alt = r["token_logp"], r["entropy"], r["top_tokens"], r["top_logp"]
    assert (lp[:, 1] == 0).all()
    assert torch.isnan(lp[torch.arange(rows) != 9, 2]).all() and (lp[9] == 0).all()
    e = Exact(z.cpu()[:, :])
    for j in (0, 1, 6, 7, 10, 11):
        assert (h[j].double() - e.h[j]).abs() <= e.h_tol[j], j
        want = e.logp[j, tokens[j, 0].item()]
        assert lp[j, 0] == -inf if want == -inf else abs(lp[j, 0].double() - want) <= 1e-5, j
    assert lp[0, 0] == -inf and lp[1, 0] == (-inf if vocab > 4 and z[1, 4] == low else lp[1, 0])
    for j, n in ((0, 3), (1, 5), (7, 1)):
        assert (at[j, :n] >= 0).all() and (at[j, n:] == -1).all() and (alt[j, n:] == -inf).all()
    assert at[7, 0] == 123 and alt[7, 0] == 0.0 and h[7] == 0.0 and lp[7, 0] == 0.0
    for j in (2, 3, 8):
        assert lp[j, 0] == -inf and h[j] == 0 and (at[j] == -1).all() and (alt[j] == -inf).all(), j
    for j in (4, 5):
        assert torch.isnan(lp[j, 0]) and torch.isnan(h[j]) and (at[j] == -1).all() and torch.isnan(alt[j]).all(), j
    assert h[9] == 0 and (at[9] == -1).all() and (alt[9] == 0).all()

    res = token_logprobs(z, tokens, mask=mask, top=6)
    by = torch.ones(rows, 3).cuda()
    by[11] = 0
    grad = token_logprobs_grad(z, tokens, res, by, grad_entropy=torch.zeros(rows).cuda(), mask=mask).double().cpu()
    for j in (2, 3, 8, 9, 11):
        assert (grad[j] == 0).all(), j
    for j in (4, 5):
        assert torch.isnan(grad[j]).all(), j
    eps = torch.finfo(dtype).eps / 2
    for j in (0, 1, 6, 7, 10):
        want = -e.p[j]
        want[tokens[j, 0].item()] += 1
        assert ((grad[j] - want).abs() <= eps * want.abs() + 1e-5).all(), j
    # an entropy's gradient over masked logits is finite
    grad = token_logprobs_grad(z, None, res, None, grad_entropy=torch.ones(rows).cuda(), mask=mask).double().cpu()
    for j in (0, 1, 6, 7, 10):
        want = -e.p[j] * (e.logp[j].clamp(min=-200) + e.h[j])
        assert ((grad[j] - want).abs() <= eps * want.abs() + 1e-5).all(), j
    assert (grad[9] == 0).all()


@pytest.mark.parametrize("temperature", [1e-3, 0.05, 30.0, 1e4])
def test_temperatures(temperature):
    z = logits_of(8, 6, 3001, torch.float32)
    tokens = torch.randint(0, 3001, (6, 1), generator=torch.Generator().manual_seed(2))
    r = token_logprobs(z, tokens[:, 0].int().cuda(), temperature=temperature, top=3)
    e = Exact(z, temperature)
    within(r["token_logp"][:, None], e.logp.gather(1, tokens), e.logp_tol(tokens), "logp")
    within(r["entropy"], e.h, e.h_tol, "entropy")
    check_top(z, r, 3)


def test_large_logits():
    """Logits near the ends of the range, and differences past it."""
    z = torch.zeros(5, 64)
    z[0], z[0, 1] = 1e37, 1.0001e37
    z[1, :32] = -5e37
    z[2] = -9.9e37
    z[3, 7] = 3e38
    z[4, :5] = -1.01e38  # masked
    r = {k: v.cpu() for k, v in token_logprobs(z.cuda(), torch.ones(5, dtype=torch.int32).cuda(), top=1).items()}
    assert r["token_logp"][0] == 0 and r["entropy"][0] == 0 and r["top_tokens"][0, 0] == 1
    assert abs(r["entropy"][1].item() - math.log(32)) < 1e-5 and r["token_logp"][1] < -1e37
    assert abs(r["entropy"][2].item() - math.log(64)) < 1e-5
    assert r["token_logp"][3] == torch.tensor(-3e38) and r["entropy"][3] == 0 and r["top_tokens"][3, 0] == 7
    assert r["token_logp"][4] == -math.inf and abs(r["entropy"][4].item() - math.log(59)) < 1e-5


def test_same_token_twice():
    z = logits_of(9, 3, 400, torch.float32)
    tokens = torch.tensor([[5, 5, 9], [0, 0, 0], [399, 5, 399]], dtype=torch.int32).cuda()
    r = token_logprobs(z, tokens)
    by = torch.tensor([[1.0, 2.0, -1.0], [0.5, 0.25, 0.125], [-2.0, 1.0, 3.0]]).cuda()
    grad = token_logprobs_grad(z, tokens, r, by)
    e = Exact(z)
    want, off = e.grad(tokens.long().cpu(), by, None, 1.0)
    within(grad, want, off + U * want.abs(), "gradient")


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_gradient_against_differences(temperature):
    vocab, h = 37, 1e-5
    z = logits_of(10, 3, vocab, torch.float32)
    tokens = torch.tensor([[3, 17], [36, 36], [0, -1]], dtype=torch.int32)
    by, by_h = torch.tensor([[1.0, -0.5], [0.75, 0.5], [2.0, 9.0]]), torch.tensor([0.5, -1.5, 1.0])

    def value(x):
        lp = torch.log_softmax(x / temperature, -1)
        given = torch.where(tokens >= 0, lp.gather(1, tokens.long().clamp(min=0)), 0.0)
        return (given * by).sum(1) - by_h * (lp.exp() * lp).sum(-1)

    x = z.double().cpu()
    want = torch.empty_like(x)
    for v in range(vocab):
        step = torch.zeros_like(x)
        step[:, v] = h
        want[:, v] = (value(x + step) - value(x - step)) / (2 * h)
    r = token_logprobs(z, tokens.cuda(), temperature=temperature)
    grad = token_logprobs_grad(z, tokens.cuda(), r, by.cuda(), grad_entropy=by_h.cuda(), temperature=temperature)
    # h^2 / 6 times the third derivative, below 20 / T^3 here, and 64-bit rounding over h
    assert ((grad.double().cpu() - want).abs() <= 20 / temperature ** 3 * h * h + 1e-9 + 1e-5 * want.abs() + 2e-6).all()


def test_gradient_of_alternatives():
    """The top alternatives as given tokens, -1 among them."""
    z = logits_of(11, 5, 900, torch.bfloat16)
    z[2, 4:] = -math.inf
    r = token_logprobs(z, top=10)
    by = torch.randn(5, 10, generator=torch.Generator().manual_seed(4)).cuda()
    grad = token_logprobs_grad(z, r["top_tokens"], r, by)
    e = Exact(z)
    at = r["top_tokens"].long().cpu()
    live = torch.where(at >= 0, by.cpu(), 0.0)
    want, off = e.grad(at.clamp(min=0), live, None, 1.0)
    within(grad, want, off + 2.0 ** -8 * (want.abs() + off) + 2.0 ** -133, "gradient")


def test_outputs_and_what_lies_behind_them():
    rows, vocab = 6, 1003
    z = logits_of(12, rows, vocab, torch.bfloat16, wide=1040)
    tokens = torch.arange(rows, dtype=torch.int32).cuda()
    want = token_logprobs(z, tokens, top=4)
    out = {k: torch.full_like(v, 7) for k, v in want.items()}
    size = (4 << 20)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    got = token_logprobs(z, tokens, top=4, out=out, workspace=ws)
    for k in want:
        assert got[k] is out[k] and torch.equal(got[k], want[k]), k
    grads = torch.full((rows, 1024), 5.0, dtype=torch.bfloat16, device="cuda")
    by = torch.ones(rows).cuda()
    g = token_logprobs_grad(z, tokens, want, by, out=grads[:, :vocab])
    assert (grads[:, vocab:] == 5.0).all()
    assert torch.equal(g, token_logprobs_grad(z, tokens, want, by))
    # of one row alone, and of views
    one = token_logprobs(z[3:4], tokens[3:4], top=4)
    for k in want:
        assert torch.allclose(one[k].float(), want[k][3:4].float(), rtol=1e-5, atol=1e-5), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_gradients_between_the_logits(dtype):
    """Logits and gradients are column slices of the same rows."""
    rows, vocab = 5, 1003
    z = logits_of(14, rows, vocab, dtype, wide=2048)
    tokens = torch.arange(rows, dtype=torch.int32).cuda()
    result, by = token_logprobs(z, tokens), torch.ones(rows).cuda()
    want = token_logprobs_grad(z, tokens, result, by)
    both = torch.full((rows, 2048), 5.0, dtype=dtype, device="cuda")
    both[:, :vocab] = z
    token_logprobs_grad(both[:, :vocab], tokens, result, by, out=both[:, 1008:1008 + vocab])
    assert torch.equal(both[:, 1008:1008 + vocab], want) and torch.equal(both[:, :vocab], z)
    assert (both[:, vocab:1008] == 5.0).all() and (both[:, 1008 + vocab:] == 5.0).all()
    with pytest.raises(bd.CtxError, match="overlaps"):
        token_logprobs_grad(both[:, :vocab], tokens, result, by, out=both[:, 1000:1000 + vocab])


def test_refusals():
    z = logits_of(1, 4, 96, torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int32).cuda()
    r = token_logprobs(z, t)
    by = torch.zeros(4).cuda()
    with pytest.raises(TypeError):
        token_logprobs(z, t.long())
    with pytest.raises(ValueError):
        token_logprobs(z, t[:3])
    with pytest.raises(ValueError):
        token_logprobs(z, t, mask=torch.ones(5, dtype=torch.uint8).cuda())
    with pytest.raises(TypeError):
        token_logprobs(z, t, mask=torch.ones(4, dtype=torch.bool).cuda())
    with pytest.raises(ValueError):
        token_logprobs(z.t(), t)
    with pytest.raises(ValueError):
        token_logprobs(z, t, temperature=0.0)
    with pytest.raises(bd.CtxError, match="top"):
        token_logprobs(z, t, top=65)
    with pytest.raises(ValueError):
        token_logprobs(z, t, out={"entropy": torch.empty(5).cuda()})
    with pytest.raises(bd.CtxError, match="workspace"):
        token_logprobs(logits_of(1, 2, 100000, torch.bfloat16), workspace=torch.empty(16, dtype=torch.uint8).cuda())
    with pytest.raises(bd.CtxError, match="row_stride"):
        token_logprobs(torch.zeros(4, 97, dtype=torch.bfloat16).cuda())
    with pytest.raises(bd.CtxError, match="aligned"):
        token_logprobs(torch.zeros(4, 104, dtype=torch.bfloat16).cuda()[:, 4:])
    with pytest.raises(ValueError):
        token_logprobs_grad(z, t, r, None)
    with pytest.raises(ValueError):
        token_logprobs_grad(z, t, {"stats": r["stats"]}, by, grad_entropy=by)
    with pytest.raises(ValueError):
        token_logprobs_grad(z, t, r, by[:3].contiguous())
    with pytest.raises(ValueError):
        token_logprobs_grad(z, t, r, by, out=torch.empty(4, 96).cuda())


@pytest.mark.parametrize("rows", [3, 1100])
def test_graph_replays(rows):
    vocab = 20011
    z = logits_of(13, rows, vocab, torch.bfloat16)
    tokens = torch.randint(0, vocab, (rows,), dtype=torch.int32).cuda()
    by, by_h = torch.randn(rows).cuda(), torch.randn(rows).cuda()
    token_logprobs(z, tokens, top=5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = token_logprobs(z, tokens, top=5)
        g = token_logprobs_grad(z, tokens, r, by, grad_entropy=by_h)
    for seed in (14, 15, 16):
        z.copy_(logits_of(seed, rows, vocab, torch.bfloat16))
        graph.replay()
        got = {k: v.clone() for k, v in r.items()} | {"grad": g.clone()}
        torch.cuda.synchronize()
        want = token_logprobs(z, tokens, top=5)
        want["grad"] = token_logprobs_grad(z, tokens, want, by, grad_entropy=by_h)
        for k in want:
            assert torch.equal(got[k], want[k]), k


def test_two_streams_at_once():
    z = [logits_of(20 + i, 4, 100003 + 8 * i, torch.bfloat16, wide=100032) for i in range(2)]
    want = [token_logprobs(x, top=9) for x in z]
    streams = [torch.cuda.Stream() for _ in z]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for x, s in zip(z, streams):
            got.append(token_logprobs(x, top=9, stream=s))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for k in r:
            assert torch.equal(r[k], want[i % 2][k]), k


def test_log_probabilities_for_the_distillation_loss():
    """The sampler's and the teacher's log probabilities of a batch go into the OPD loss, whose own
    log probability of the student is the same."""
    from paper_2609_36608_amd import opd_loss

    rows, vocab = 40, 5000
    student, teacher = (logits_of(s, rows, vocab, torch.bfloat16) for s in (30, 31))
    tokens = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1)).int().cuda()
    mask = (torch.arange(rows) % 5 != 0).to(torch.uint8).cuda()
    old = token_logprobs(student, tokens, mask=mask)["token_logp"]
    tea = token_logprobs(teacher, tokens, mask=mask, entropy=False)["token_logp"]
    starts = torch.tensor([0, 13, rows], dtype=torch.int32).cuda()
    r = opd_loss(student, tokens, old, tea, mask, starts)
    e = Exact(student)
    at = tokens.long().cpu()[:, None]
    tol = 2 * e.logp_tol(at)[:, 0]
    assert ((r["token_logp"] - old).double().cpu().abs() <= tol).all()
    # on policy the ratio is 1: the gradient is the advantage's, by the log probability
    e_t = Exact(teacher)
    adv = (e_t.logp - e.logp).gather(1, at)[:, 0] * (mask.cpu() != 0)
    weight = r["token_weight"].double().cpu()
    res = token_logprobs(student, tokens, mask=mask)
    g = token_logprobs_grad(student, tokens, res, (-weight * adv).float().cuda(), mask=mask)
    diff = (g.float() - r["grad_logits"].float()).abs().cpu()
    assert (diff <= 2 * 2.0 ** -8 * r["grad_logits"].float().abs().cpu() + 1e-6).all()
