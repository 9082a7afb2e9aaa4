"""Operators over paged key-value caches, measured: the append of new keys and values with the norm
and the rotation of positions applied on the way, and the causal prefill and the decode step whose
scores are capped by a tanh, biased by distance or masked by a window, a prefix or documents.

`listed()` holds fixed cases, `draw()` gives others of the same ranges.  A case's context lengths,
documents and page placement come from its own `lens_seed`, so that every seed has the same work;
queries, keys, values and caches come from the seed given to `prepare`.

The operators, for the row j that is the i-th of the n new rows of sequence b, whose cache holds
L tokens, the new ones included (p = L - n + i is the row's position):

  append   normed(x) = x * w / sqrt(mean(x^2) + eps) over a head; rotated(x): pairs (a, c) of the
           rotary dimensions become (a cos - c sin, c cos + a sin) with the angle position * inv_freq
           q_out[j] = rotated(normed(q[j]));  K of token p = rotated(normed(k[j]));  V of token p = v[j]
  prefill  s = q.k / sqrt(128);  s = cap * tanh(s / cap);  s -= slope[head] * |p - t|
           token t is visible if t < prefix[b] or max(doc[j], p - window + 1) <= t <= p
           out[j] = softmax(s over the visible tokens) . V, zeros where none is visible
  decode   the same for the one row of each sequence, p = L - 1
"""
import math
import random

import torch

own = False  # True: the framework's operators; False: their plain form

HEAD_DIM = 128
SCALE = 1.0 / math.sqrt(HEAD_DIM)
ROPE_THETA = 1e6
NORM_EPS = 1e-6
PEAKY_FRAC, PEAKY_GAIN = 0.05, 4.0
EMPTY_ROW = 2**31 - 1  # the document start of a padding row, which sees nothing

_APPEND = dict(op="append", page=16, hist_lo=0, hist_hi=0, norm=True, interleaved=False, rot=128, positions=False)
_ATTEND = dict(page=16, new_lo=1, new_hi=1, out="bf16", softcap=0.0, window=0, prefix=0, slopes=False, doc_lo=0,
               doc_hi=0, pad=0, qstd=1.0, peaky=False)


def listed():
    return [
        # one new token each of a few requests of a small student: latency alone
        dict(_APPEND, name="append_step_few", hq=16, hkv=8, batch=4, hist_lo=256, hist_hi=1024, new_lo=1, new_hi=1,
             lens_seed=1),
        # one decode step of the largest batch
        dict(_APPEND, name="append_step_batch", hq=32, hkv=8, batch=256, hist_lo=512, hist_hi=1536, new_lo=1, new_hi=1,
             lens_seed=2),
        # the reference observations of a burst, rows of a fused projection
        dict(_APPEND, name="append_burst", hq=32, hkv=8, batch=96, hist_lo=128, hist_hi=1024, new_lo=128, new_hi=512,
             lens_seed=3),
        # one long prompt, half of each head rotated, pairs side by side, positions given
        dict(_APPEND, name="append_prompt", page=64, hq=28, hkv=4, batch=1, new_lo=20479, new_hi=20479, norm=False,
             interleaved=True, rot=64, positions=True, lens_seed=4),
        # a few short contexts in flight, capped scores: latency
        dict(_ATTEND, name="decode_cap_few", op="decode", hq=16, hkv=8, batch=4, hist_lo=255, hist_hi=1023,
             softcap=30.0, qstd=4.0, lens_seed=5),
        # long ragged contexts of which a step sees the prompt and the last 4,096 tokens
        dict(_ATTEND, name="decode_window_ragged", op="decode", hq=32, hkv=8, batch=32, hist_lo=512, hist_hi=32767,
             window=4096, prefix=100, lens_seed=6),
        # a student of another kind: scores fall with the distance, 32-bit outputs
        dict(_ATTEND, name="decode_bias_batch", op="decode", hq=32, hkv=8, batch=64, hist_lo=2048, hist_hi=8191,
             slopes=True, out="f32", lens_seed=7),
        # one request takes in its reference observation, capped scores
        dict(_ATTEND, name="prefill_cap_single", op="prefill", hq=32, hkv=8, batch=1, hist_lo=8000, hist_hi=8000,
             new_lo=301, new_hi=301, softcap=50.0, qstd=4.0, peaky=True, lens_seed=8),
        # fresh prompts of which the task description is seen from everywhere
        dict(_ATTEND, name="prefill_prefix_prompts", op="prefill", hq=16, hkv=8, batch=12, hist_lo=0, hist_hi=0,
             new_lo=200, new_hi=2000, prefix=150, lens_seed=9),
        # turns packed into one row of tokens, each seeing itself and the shared prompt; padding behind them
        dict(_ATTEND, name="prefill_documents", op="prefill", page=32, hq=32, hkv=8, batch=1, hist_lo=0, hist_hi=0,
             new_lo=10240, new_hi=10240, prefix=333, doc_lo=100, doc_hi=1500, pad=37, lens_seed=10),
        # a chunk of a long context under a window, scores falling with the distance, 32-bit outputs
        dict(_ATTEND, name="prefill_window_chunk", op="prefill", page=64, hq=28, hkv=4, batch=1, hist_lo=16001,
             hist_hi=16001, new_lo=1024, new_hi=1024, window=4096, slopes=True, out="f32", lens_seed=11),
        # reference observations over long contexts, plainly causal
        dict(_ATTEND, name="prefill_burst", op="prefill", hq=32, hkv=8, batch=16, hist_lo=4096, hist_hi=12288,
             new_lo=128, new_hi=512, lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill"])
    while True:
        case = {"append": _draw_append, "decode": _draw_decode, "prefill": _draw_prefill}[op](rng)
        # no more than the largest listed case of its kind, also in the memory of the plain form
        w = work(case)
        rows, tokens = max(_lengths(case)[1]), max(_lengths(case)[0])
        scores = case["batch"] * case["hq"] * rows * tokens if op != "append" else 0
        if w["bytes"] <= 1.1e9 and w["flops"] <= 6e11 and scores <= 2.5e9 and case["batch"] * tokens <= 1.1e6:
            return case


def _draw_append(rng):
    hq, hkv = rng.choice([(16, 8), (32, 8), (64, 8), (16, 16), (28, 4), (12, 2), (16, 1)])
    step = rng.random() < 0.4
    new_lo = 1 if step else _log_int(rng, 2, 4096)
    return dict(op="append", page=rng.choice([16, 16, 32, 64, 48]), hq=hq, hkv=hkv, batch=_log_int(rng, 1, 256),
                hist_lo=(lo := _log_int(rng, 1, 1024)), hist_hi=lo + rng.randrange(1024), new_lo=new_lo,
                new_hi=1 if step else int(new_lo * rng.uniform(1.0, 4.0)), norm=rng.random() < 0.5,
                interleaved=rng.random() < 0.3, rot=rng.choice([128, 128, 64, 32, 96]), positions=rng.random() < 0.3,
                lens_seed=rng.randrange(1 << 30))


def _draw_scores(rng, batch):
    kind = rng.choice(["cap", "bias", "window", "prefix", "docs", "mixed", "causal"])
    mixed = kind == "mixed"
    docs = kind == "docs" or (mixed and rng.random() < 0.3)
    doc_lo = _log_int(rng, 20, 1000) if docs else 0
    return dict(softcap=rng.choice([20.0, 30.0, 50.0]) if kind == "cap" or (mixed and rng.random() < 0.6) else 0.0,
                slopes=kind == "bias" or (mixed and rng.random() < 0.5),
                window=_log_int(rng, 16, 8192) if kind == "window" or (mixed and rng.random() < 0.5) else 0,
                prefix=_log_int(rng, 1, 2000) if kind == "prefix" or (kind != "causal" and rng.random() < 0.3) else 0,
                doc_lo=doc_lo, doc_hi=doc_lo * 4, pad=rng.randrange(8) if docs else 0,
                qstd=rng.choice([1.0, 1.0, 2.0, 4.0]), peaky=rng.random() < 0.3)


def _draw_decode(rng):
    hq, hkv = rng.choice([(16, 8), (32, 8), (32, 8), (64, 8), (16, 16), (28, 4), (12, 2), (16, 1)])
    batch = _log_int(rng, 1, 256)
    lo = _log_int(rng, 32, 16384)
    return dict(op="decode", page=rng.choice([16, 16, 32, 64, 48]), hq=hq, hkv=hkv, batch=batch, hist_lo=lo,
                hist_hi=min(32767, int(lo * rng.uniform(1.0, 16.0))), new_lo=1, new_hi=1,
                out=rng.choice(["bf16", "bf16", "f32"]), lens_seed=rng.randrange(1 << 30), **_draw_scores(rng, batch))


def _draw_prefill(rng):
    hq, hkv = rng.choice([(16, 8), (32, 8), (32, 8), (64, 8), (16, 16), (28, 4), (12, 2)])
    batch = _log_int(rng, 1, 64)
    hist_lo = 0 if rng.random() < 0.4 else _log_int(rng, 64, 12288)
    new_lo = _log_int(rng, 16, 2048)
    return dict(op="prefill", page=rng.choice([16, 16, 32, 64, 48]), hq=hq, hkv=hkv, batch=batch, hist_lo=hist_lo,
                hist_hi=int(hist_lo * rng.uniform(1.0, 2.0)), new_lo=new_lo,
                new_hi=int(new_lo * rng.uniform(1.0, 3.0)), out=rng.choice(["bf16", "bf16", "f32"]),
                lens_seed=rng.randrange(1 << 30), **_draw_scores(rng, batch))


# ------------------------------------------------------------------ shapes of a case (no seed)

def _lengths(case):
    """Tokens in the cache, the new ones included, and new tokens of every sequence."""
    rng = random.Random(case["lens_seed"])
    if case["op"] == "decode" and case["hist_hi"] > 8 * case["hist_lo"]:  # widely ragged: spread over the logarithm
        a, b = math.log(case["hist_lo"]), math.log(case["hist_hi"])
        hist = [int(math.exp(rng.uniform(a, b))) for _ in range(case["batch"])]
    else:
        hist = [rng.randint(case["hist_lo"], case["hist_hi"]) for _ in range(case["batch"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    return [h + n for h, n in zip(hist, new)], new


def _prefixes(case):
    return [min(case["prefix"], n) for n in _lengths(case)[0]]


def _documents(case):
    """The document start of every new row: documents follow the prefix; the last rows of a sequence are padding."""
    rng = random.Random(case["lens_seed"] + 1)
    starts = []
    for length, new, prefix in zip(*_lengths(case), _prefixes(case)):
        at, row = prefix, []
        end = at + rng.randint(case["doc_lo"], case["doc_hi"])
        for p in range(length - new, length):
            while p >= end:
                at, end = end, end + rng.randint(case["doc_lo"], case["doc_hi"])
            row.append(at)
        pad = min(case["pad"], new - 1)
        starts.extend(row[:new - pad] + [EMPTY_ROW] * pad)
    return starts


def _first_seen(case):
    """The first token past the prefix that each new row sees, by sequence."""
    lens, new = _lengths(case)
    docs = _documents(case) if case["doc_lo"] else [0] * sum(new)
    window, at, seen = case["window"], 0, []
    for length, n in zip(lens, new):
        rows = []
        for i in range(n):
            p = length - n + i
            rows.append(max(docs[at + i], p - window + 1 if window else 0, 0))
        at += n
        seen.append(rows)
    return seen


def work(case):
    lens, new = _lengths(case)
    rows, hq, hkv = sum(new), case["hq"], case["hkv"]
    if case["op"] == "append":
        values = rows * (hq + 2 * hkv) * HEAD_DIM
        return {"bytes": values * 2 * 2 + rows * 4, "flops": rows * (hq + hkv) * HEAD_DIM * (7 if case["norm"] else 3)}
    pairs = tokens = 0
    for length, n, prefix, first in zip(lens, new, _prefixes(case), _first_seen(case)):
        for i in range(n):
            pairs += prefix + max(0, length - n + i + 1 - max(first[i], prefix))
        tokens += length - max(0, min(min(first), length) - prefix)
    out = 4 if case["out"] == "f32" else 2
    return {"bytes": tokens * hkv * HEAD_DIM * 2 * 2 + rows * hq * HEAD_DIM * (2 + out),
            "flops": pairs * hq * HEAD_DIM * 4}


# ------------------------------------------------------------------ inputs

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(g, shape, std=1.0):
    """bf16 N(0, std^2)."""
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = t.view(-1)
    for s in range(0, flat.numel(), 1 << 28):
        flat[s:s + (1 << 28)].normal_(0.0, std, generator=g)
    return t


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lens, new = _lengths(case)
    rows, batch, hq, hkv = sum(new), case["batch"], case["hq"], case["hkv"]
    pages = [-(-n // case["page"]) for n in lens]
    order = list(range(sum(pages) + 4))
    random.Random(seed).shuffle(order)
    table, at = [], 0
    for n in pages:
        table.append(order[at:at + n] + [0] * (max(pages) - n))
        at += n
    starts = [sum(new[:b]) for b in range(batch)]
    shape = (len(order), case["page"], hkv, HEAD_DIM)
    s = {"case": case, "lens": _i32(lens), "new": _i32(new), "starts": _i32(starts), "table": _i32(table),
         "max_new": max(new), "max_len": max(lens), "rows": rows, "k": _normal(g, shape), "v": _normal(g, shape)}
    if case["op"] == "append":
        # rows of one fused projection: queries, then keys, then values
        s["qkv"] = _normal(g, (rows, (hq + 2 * hkv) * HEAD_DIM), 2.0)
        rot = case["rot"]
        s["inv_freq"] = (ROPE_THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)).float()
        if case["norm"]:
            s["q_norm"], s["k_norm"] = (1 + 0.2 * _normal(g, (HEAD_DIM,)) for _ in range(2))
        if case["positions"]:  # far positions too
            s["positions"] = torch.randint(0, 1 << 17, (rows,), generator=g, device="cuda", dtype=torch.int32)
        return s
    if case["peaky"]:
        gain = torch.ones(shape[:2], dtype=torch.bfloat16, device="cuda")
        gain.masked_fill_(torch.rand(shape[:2], generator=g, device="cuda") < PEAKY_FRAC, PEAKY_GAIN)
        s["k"].mul_(gain[:, :, None, None])
    s["q"] = _normal(g, (rows, hq, HEAD_DIM), case["qstd"])
    if case["slopes"]:
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda", dtype=torch.float32) / hq)
    if case["prefix"]:
        s["prefix"] = _i32(_prefixes(case))
    if case["doc_lo"]:
        s["docs"] = _i32(_documents(case))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    dtype = torch.float32 if case.get("out") == "f32" else torch.bfloat16
    s["out"] = torch.empty((s["rows"], case["hq"], HEAD_DIM), dtype=dtype, device="cuda")
    if own:  # a serving program keeps its handle
        from paper_2609_36608_amd import DecodeAttention

        s["attn"] = DecodeAttention(case["hq"], case["hkv"], case["batch"], s["max_len"], out_dtype=dtype,
                                    page_tokens=case["page"])
    return s


# ------------------------------------------------------------------ the plain forms

def _split(s):
    case = s["case"]
    q, k, v = s["qkv"].view(s["rows"], -1, HEAD_DIM).split([case["hq"], case["hkv"], case["hkv"]], dim=1)
    return q, k, v


def _rows(s):
    """Sequence and position of every new row."""
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["starts"].long(), row, right=True) - 1
    return seq, (s["lens"] - s["new"] - s["starts"]).long()[seq] + row


def _normed(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + NORM_EPS) * weight.float()


def _rotated(x, angle, interleaved):
    x, cos, sin = x.float(), angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = angle.shape[1]
    if interleaved:
        a, c, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
        turned = torch.stack([a * cos - c * sin, c * cos + a * sin], -1).flatten(-2)
    else:
        a, c, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        turned = torch.cat([a * cos - c * sin, c * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _plain_append(s):
    case = s["case"]
    q, k, v = _split(s)
    if case["norm"]:
        q, k = _normed(q, s["q_norm"]), _normed(k, s["k_norm"])
    seq, p = _rows(s)
    angle = (s["positions"] if case["positions"] else p).double()[:, None] * s["inv_freq"].double()
    slot = s["table"].long()[seq, p // case["page"]] * case["page"] + p % case["page"]
    s["out"].copy_(_rotated(q, angle, case["interleaved"]))
    s["k"].view(-1, case["hkv"], HEAD_DIM)[slot] = _rotated(k, angle, case["interleaved"]).to(torch.bfloat16)
    s["v"].view(-1, case["hkv"], HEAD_DIM)[slot] = v


def _plain_attention(s):
    """Every sequence padded to the longest: scores [batch, KV head, row, head of the group, token]."""
    case, rows, tokens = s["case"], s["max_new"], s["max_len"]
    batch, hkv, g = case["batch"], case["hkv"], case["hq"] // case["hkv"]
    # from projected rows to padded sequences
    seq, p = _rows(s)
    i = torch.arange(rows, device="cuda")
    at = (s["starts"].long()[:, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"][at].float().view(batch, rows, hkv, g, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(batch, hkv, rows * g, HEAD_DIM)
    k = s["k"][s["table"].long()].flatten(1, 2)[:, :tokens].permute(0, 2, 3, 1).float().contiguous()
    x = (q @ k).mul_(SCALE).view(batch, hkv, rows, g, tokens)
    if case["softcap"]:
        x = x.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    t = torch.arange(tokens, device="cuda")
    pos = (s["lens"] - s["new"]).long()[:, None] + i  # [batch, row]
    if case["slopes"]:
        x.sub_(s["slopes"].view(1, hkv, 1, g, 1) * (pos[:, :, None] - t).abs().float()[:, None, :, None])
    first = torch.zeros_like(pos)
    if case["window"]:
        first = pos - case["window"] + 1
    if case["doc_lo"]:
        first = torch.maximum(first, s["docs"].long()[at])
    seen = (t >= first[:, :, None]) & (t <= pos[:, :, None])
    if case["prefix"]:
        seen |= t < s["prefix"][:, None, None]
    seen &= t < s["lens"][:, None, None]
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)).exp_()
    total = x.sum(-1, keepdim=True).view(batch, hkv, rows * g, 1)
    v = s["v"][s["table"].long()].flatten(1, 2)[:, :tokens].permute(0, 2, 1, 3).float().contiguous()
    o = (x.view(batch, hkv, rows * g, tokens) @ v) / torch.where(total > 0, total, 1.0)
    o = o.view(batch, hkv, rows, g, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(batch, rows, case["hq"], HEAD_DIM)
    s["out"].copy_(o[seq, torch.arange(s["rows"], device="cuda") - s["starts"].long()[seq]])


# ------------------------------------------------------------------ the framework's calls

def _own_append(s):
    from paper_2609_36608_amd import Rotary

    case = s["case"]
    q, k, v = _split(s)
    rotary = Rotary(s["inv_freq"], interleaved=case["interleaved"], positions=s.get("positions"),
                    q_norm=s.get("q_norm"), k_norm=s.get("k_norm"), norm_eps=NORM_EPS)
    rows = {} if case["new_hi"] == 1 else dict(q_starts=s["starts"], q_lens=s["new"])
    s["attn"].append_paged(k, v, s["k"], s["v"], s["table"], s["lens"], q=q, q_out=s["out"], rotary=rotary, **rows)


def _own_attention(s):
    from paper_2609_36608_amd import AttnScores

    case = s["case"]
    scores = AttnScores(softcap=case["softcap"], window=case["window"], slopes=s.get("slopes"),
                        prefix_lens=s.get("prefix"), doc_starts=s.get("docs"))
    if case["op"] == "decode":
        s["attn"].run_paged(s["q"], s["k"], s["v"], s["table"], s["lens"], SCALE, s["out"], scores=scores)
    else:
        s["attn"].prefill_paged(s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], s["new"], s["max_new"],
                                SCALE, s["out"], scores=scores)


def run(s):
    if s["case"]["op"] == "append":
        if own:
            _own_append(s)
        else:
            _plain_append(s)
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    if own:
        _own_attention(s)
    else:
        _plain_attention(s)
    return {"out": s["out"]}


# ------------------------------------------------------------------ 64-bit results

def _exact_append(s):
    case = s["case"]
    lens, new = _lengths(case)
    x = s["qkv"].double().view(s["rows"], -1, HEAD_DIM)
    hq, hkv, rot = case["hq"], case["hkv"], case["rot"]
    k, v = (s[name].double() for name in ("k", "v"))
    heads = x[:, :hq + hkv]
    if case["norm"]:
        w = torch.cat([s["q_norm"].expand(hq, -1), s["k_norm"].expand(hkv, -1)]).double()
        heads = heads / (heads.pow(2).mean(-1, keepdim=True) + NORM_EPS).sqrt() * w
    pos = s["positions"].tolist() if case["positions"] else [t for n, m in zip(lens, new) for t in range(n - m, n)]
    turn = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, None] * s["inv_freq"].double()
    # the pairs as complex numbers
    if case["interleaved"]:
        z = torch.view_as_complex(heads[..., :rot].reshape(s["rows"], -1, rot // 2, 2).contiguous())
    else:
        z = torch.complex(heads[..., :rot // 2].contiguous(), heads[..., rot // 2:rot].contiguous())
    z = z * torch.polar(torch.ones_like(turn), turn)[:, None]
    done = torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
    heads = torch.cat([done, heads[..., rot:]], -1)
    table, at = s["table"].tolist(), 0
    for b, (n, m) in enumerate(zip(lens, new)):
        slots = [table[b][t // case["page"]] * case["page"] + t % case["page"] for t in range(n - m, n)]
        slots = torch.tensor(slots, device="cuda")
        k.view(-1, hkv, HEAD_DIM)[slots] = heads[at:at + m, hq:]
        v.view(-1, hkv, HEAD_DIM)[slots] = x[at:at + m, hq + hkv:]
        at += m
    return {"q": heads[:, :hq].contiguous(), "k": k, "v": v}


def _exact_attention(s):
    case = s["case"]
    lens, new = _lengths(case)
    g = case["hq"] // case["hkv"]
    out = torch.empty((s["rows"], case["hq"], HEAD_DIM), dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m, prefix, first) in enumerate(zip(lens, new, _prefixes(case), _first_seen(case))):
        pages = s["table"][b, :-(-n // case["page"])].long()
        kb, vb = (s[name][pages].flatten(0, 1)[:n] for name in ("k", "v"))
        t = torch.arange(n, device="cuda")
        for r in range(0, m, 512):  # some rows at a time
            c = min(512, m - r)
            p = torch.arange(n - m + r, n - m + r + c, device="cuda")
            low = torch.tensor(first[r:r + c], device="cuda")
            hidden = ((t < low[:, None]) | (t > p[:, None])) & (t >= prefix)
            far = (p[:, None] - t).abs().double()
            for h in range(case["hkv"]):
                heads = slice(h * g, (h + 1) * g)
                q = s["q"][at + r:at + r + c, heads].double().transpose(0, 1).reshape(g * c, HEAD_DIM)
                x = (q @ kb[:, h].double().t().contiguous()).view(g, c, n) / math.sqrt(HEAD_DIM)
                if case["softcap"]:
                    x = torch.tanh(x / case["softcap"]) * case["softcap"]
                if case["slopes"]:
                    x = x - s["slopes"][heads].double()[:, None, None] * far
                weight = torch.softmax(x.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
                o = weight.view(g * c, n) @ vb[:, h].double().contiguous()
                out[at + r:at + r + c, heads] = o.view(g, c, HEAD_DIM).transpose(0, 1)
        at += m
    return {"out": out}


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)
