"""More operators, measured: attention of a tree of drafted tokens over paged caches, the caches' pages
(forked, grown and trimmed; kept tokens moved together), and log probabilities of given tokens with
their entropy, the top alternatives and the gradient of the logits.

`listed()` holds fixed cases, `draw()` gives others of the same ranges.  A case's lengths, trees, kept
tokens and masks come from its own `lens_seed`, so that every seed has the same work; queries, keys,
values, caches, logits and page placement come from the seed given to `prepare`.

The operators:

  tree      sequence b holds L tokens, the last n of them drafted; draft i has a parent among the drafts
            before it, or none (-1), or is padding.  Its position is p = L - n + its depth.  It sees the
            tokens before the drafts, if p - position < window or token < prefix, and itself and its
            ancestors by the same rule.  s = q.k / sqrt(128); s = cap * tanh(s / cap);
            s -= slope[head] * (p - position);  out = softmax(s) . V, zeros for padding
  cycle     rows of the block table become copies of other rows, whose pages they share (every page
            counts its rows); every row then gets room for drafted tokens: the lowest free pages, by
            row, and a copy of its last page where that is shared and not full; then it is trimmed again
  compact   of a sequence's last n tokens those listed, in order, are moved together
  logprobs  x = logits / temperature;  lp = x[token] - log sum exp x;  H = -sum p log p;  the largest
            logits, the lowest index first among equal ones
  grad      the gradient of sum_j (a_j . lp_j + b_j H_j) by the logits
"""
import math
import random

import torch

own = False  # True: the framework's operators; False: their plain form

HEAD_DIM = 128
SCALE = 1.0 / math.sqrt(HEAD_DIM)
PEAKY_FRAC, PEAKY_GAIN = 0.05, 4.0
PADDING = 2**31 - 1  # the parent of a padding row

_TREE = dict(op="tree", page=16, out="bf16", softcap=0.0, window=0, prefix=0, slopes=False, pad=0, qstd=1.0, peaky=False)
_LOGITS = dict(dtype="bf16", mask=1.0, given=1, top=0, entropy=True, temperature=1.0)


def listed():
    return [
        # drafts of a few requests of a small student: latency
        dict(_TREE, name="tree_few", hq=16, hkv=8, batch=4, hist_lo=256, hist_hi=1024, new_lo=8, new_hi=16, lens_seed=1),
        # drafts of a batch in the middle of its episodes
        dict(_TREE, name="tree_batch", hq=32, hkv=8, batch=64, hist_lo=2048, hist_hi=8191, new_lo=12, new_hi=31,
             lens_seed=2),
        # large trees over long ragged contexts
        dict(_TREE, name="tree_long_ragged", hq=32, hkv=8, batch=32, hist_lo=512, hist_hi=32767, new_lo=64, new_hi=64,
             peaky=True, lens_seed=3),
        # a student of another kind: capped scores that fall with the distance under a window, 32-bit outputs,
        # drafts padded to one size
        dict(_TREE, name="tree_scores", page=64, hq=28, hkv=4, batch=16, hist_lo=3000, hist_hi=16000, new_lo=33,
             new_hi=61, softcap=30.0, window=4096, prefix=100, slopes=True, pad=5, out="f32", qstd=4.0, lens_seed=4),
        # a few requests fork their contexts and get room for their next tokens: latency
        dict(op="cycle", name="fork_few", page=16, hkv=8, parents=4, forks=1, free=200, len_lo=300, len_hi=1000, new=8,
             lens_seed=5),
        # every request of a batch forks into three branches
        dict(op="cycle", name="fork_batch", page=16, hkv=8, parents=64, forks=3, free=3000, len_lo=2048, len_hi=8191,
             new=64, lens_seed=6),
        # the accepted path of each request's drafts
        dict(op="compact", name="compact_accepted", page=16, hkv=8, batch=64, len_lo=1024, len_hi=8191, new_lo=32,
             new_hi=64, keep="path", lens_seed=7),
        # turns dropped from the middle of long contexts
        dict(op="compact", name="compact_dropped", page=64, hkv=8, batch=12, len_lo=8192, len_hi=16384, new_lo=0,
             new_hi=0, keep="runs", lens_seed=8),
        # one serving step: the sampled tokens' log probabilities and 20 alternatives
        dict(_LOGITS, op="logprobs", name="logprobs_step", rows=8, vocab=151936, top=20, entropy=False, lens_seed=9),
        # a teacher scores a batch of responses, a part of whose tokens count
        dict(_LOGITS, op="logprobs", name="logprobs_batch", rows=4301, vocab=151936, mask=0.8, top=1, lens_seed=10),
        # a step of training by log probabilities and entropy
        dict(_LOGITS, op="grad", name="grad_batch", rows=2057, vocab=151936, mask=0.9, lens_seed=11),
        # a student drawn to a teacher's alternatives: 20 given tokens per row, 32-bit logits
        dict(_LOGITS, op="grad", name="grad_lists", rows=777, vocab=50257, dtype="f32", given=20, temperature=1.5,
             lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "cycle", "compact", "logprobs", "grad"])
    while True:
        case = {"tree": _draw_tree, "cycle": _draw_cycle, "compact": _draw_compact, "logprobs": _draw_logits,
                "grad": _draw_logits}[op](rng, op)
        w = work(case)
        if op == "tree":
            # no more than the largest listed case, also in the memory of the plain form
            lens, new = _lengths(case)
            if case["batch"] * case["hq"] * max(new) * max(lens) > 2.2e9 or case["batch"] * max(lens) > 1.1e6:
                continue
        if w["bytes"] <= {"tree": 1.3e9, "cycle": 6e7, "compact": 1e9, "logprobs": 1.1e9, "grad": 1.7e9}[op]:
            return case


def _draw_tree(rng, op):
    hq, hkv = rng.choice([(16, 8), (32, 8), (32, 8), (64, 8), (16, 16), (28, 4), (12, 2), (16, 1)])
    lo, new_lo = _log_int(rng, 16, 16384), _log_int(rng, 1, 96)
    kind = rng.choice(["plain", "plain", "cap", "bias", "window", "mixed"])
    mixed = kind == "mixed"
    return dict(op=op, page=rng.choice([16, 16, 32, 64, 48]), hq=hq, hkv=hkv, batch=_log_int(rng, 1, 128), hist_lo=lo,
                hist_hi=min(32767, int(lo * rng.uniform(1.0, 12.0))), new_lo=new_lo,
                new_hi=min(128, int(new_lo * rng.uniform(1.0, 2.0))), out=rng.choice(["bf16", "bf16", "f32"]),
                softcap=rng.choice([20.0, 30.0, 50.0]) if kind == "cap" or mixed else 0.0,
                window=_log_int(rng, 16, 8192) if kind == "window" or mixed else 0,
                prefix=_log_int(rng, 1, 2000) if kind in ("window", "mixed") and rng.random() < 0.5 else 0,
                slopes=kind == "bias" or mixed, pad=rng.choice([0, 0, 3]), qstd=rng.choice([1.0, 1.0, 2.0, 4.0]),
                peaky=rng.random() < 0.3, lens_seed=rng.randrange(1 << 30))


def _draw_cycle(rng, op):
    lo = _log_int(rng, 16, 6000)
    return dict(op=op, page=rng.choice([16, 16, 32, 64, 48]), hkv=rng.choice([8, 8, 4, 2, 16]),
                parents=_log_int(rng, 1, 64), forks=rng.choice([1, 1, 2, 3]), free=3000, len_lo=lo,
                len_hi=int(lo * rng.uniform(1.0, 1.4)), new=_log_int(rng, 1, 100), lens_seed=rng.randrange(1 << 30))


def _draw_compact(rng, op):
    keep = rng.choice(["path", "runs"])
    lo = _log_int(rng, 200, 12000)
    new_lo = _log_int(rng, 2, 96) if keep == "path" else 0
    return dict(op=op, page=rng.choice([16, 16, 32, 64, 48]), hkv=rng.choice([8, 8, 4, 2, 16]),
                batch=_log_int(rng, 1, 128 if keep == "path" else 24), len_lo=lo, len_hi=int(lo * rng.uniform(1.0, 1.5)),
                new_lo=new_lo, new_hi=min(128, 2 * new_lo), keep=keep, lens_seed=rng.randrange(1 << 30))


def _draw_logits(rng, op):
    given = rng.choice([1, 1, 1, 5, 20])
    return dict(op=op, rows=_log_int(rng, 1, 4096), vocab=_log_int(rng, 1000, 155000), dtype=rng.choice(["bf16", "bf16", "f32"]),
                mask=rng.choice([1.0, 0.9, 0.5]), given=given, top=rng.choice([0, 1, 5, 20]) if op == "logprobs" else 0,
                entropy=rng.random() < 0.7, temperature=rng.choice([1.0, 1.0, 0.7, 1.5]), lens_seed=rng.randrange(1 << 30))


# ------------------------------------------------------------------ shapes of a case (no seed)

def _lengths(case):
    """Tokens in the cache, the new ones included, and new tokens of every sequence."""
    rng = random.Random(case["lens_seed"])
    if case["op"] != "tree":
        lens = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
        return lens, [rng.randint(case["new_lo"], case["new_hi"]) or n for n in lens]
    if case["hist_hi"] > 8 * case["hist_lo"]:  # widely ragged: spread over the logarithm
        a, b = math.log(case["hist_lo"]), math.log(case["hist_hi"])
        hist = [int(math.exp(rng.uniform(a, b))) for _ in range(case["batch"])]
    else:
        hist = [rng.randint(case["hist_lo"], case["hist_hi"]) for _ in range(case["batch"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    return [h + n for h, n in zip(hist, new)], new


def _trees(case):
    """The parent of every draft, by sequence: most hang on one of the last few before them."""
    rng = random.Random(case["lens_seed"] + 1)
    trees = []
    for n in _lengths(case)[1]:
        pad = min(case["pad"], n - 1)
        row = [-1 if i == 0 or rng.random() < 0.1 else max(0, i - rng.randint(1, 6)) for i in range(n - pad)]
        trees.append(row + [PADDING] * pad)
    return trees


def _paths(row):
    """Every draft's ancestors and itself, the first first; none for padding."""
    paths = []
    for i, parent in enumerate(row):
        paths.append([] if parent == PADDING else ([] if parent < 0 else paths[parent]) + [i])
    return paths


def _prefixes(case):
    return [min(case["prefix"], n - m) for n, m in zip(*_lengths(case))]


def _kept(case):
    """Which of a sequence's last tokens stay: a path through its drafts, or what dropping turns leaves."""
    rng = random.Random(case["lens_seed"] + 1)
    kept = []
    for n in _lengths(case)[1]:
        row, at = [], 0
        while at < n:
            if case["keep"] == "path":
                row.append(at)
                if rng.random() < 0.2:
                    break
                at += rng.randint(1, 6)
            else:
                stay = rng.randint(200, 2000)
                row += range(at, min(n, at + stay))
                at += stay + rng.randint(20, 600)
        kept.append(row)
    return kept


def _supervised(case):
    rng = random.Random(case["lens_seed"])
    return [rng.random() < case["mask"] for _ in range(case["rows"])]


def _contexts(case):
    """The lengths of the forked rows."""
    rng = random.Random(case["lens_seed"])
    return [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["parents"])]


def work(case):
    op = case["op"]
    if op == "tree":
        lens, new = _lengths(case)
        pairs = tokens = 0
        for n, m, prefix, row in zip(lens, new, _prefixes(case), _trees(case)):
            hist, window = n - m, case["window"] or n
            for path in _paths(row):
                if path:
                    low = max(hist + len(path) - window, 0)
                    pairs += prefix + max(0, hist - max(low, prefix)) + min(len(path), window)
            tokens += m - row.count(PADDING) + prefix + max(0, hist - max(hist - window + 1, prefix))
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": tokens * case["hkv"] * HEAD_DIM * 2 * 2 + sum(new) * case["hq"] * HEAD_DIM * (2 + out),
                "flops": pairs * case["hq"] * HEAD_DIM * 4}
    if op == "cycle":
        lens, page, forks = _contexts(case), case["page"], case["forks"]
        pages = [-(-n // page) for n in lens]
        partial = sum(n % page > 0 for n in lens) * (1 + forks)
        fresh = sum(-(-(n + case["new"]) // page) - p for n, p in zip(lens, pages)) * (1 + forks)
        # shared entries read and written and their counts changed; pages taken and given back; pages copied
        return {"bytes": sum(pages) * forks * 12 + (fresh + partial) * 24 + partial * page * case["hkv"] * HEAD_DIM * 8,
                "flops": 0}
    if op == "compact":
        moved = sum(i != t for row in _kept(case) for i, t in enumerate(row))
        listed_tokens = sum(len(row) for row in _kept(case))
        return {"bytes": moved * case["hkv"] * HEAD_DIM * 2 * 2 * 2 + listed_tokens * 4 + case["batch"] * 24, "flops": 0}
    rows, size = sum(_supervised(case)), 2 if case["dtype"] == "bf16" else 4
    logits = rows * case["vocab"] * size
    small = rows * (case["given"] * 8 + case["top"] * 8 + 12)
    if op == "logprobs":
        return {"bytes": logits + small, "flops": rows * case["vocab"] * 4}
    # forward, and the gradient, which is written for every row
    return {"bytes": 2 * logits + case["rows"] * case["vocab"] * size + 2 * small, "flops": rows * case["vocab"] * 8}


# ------------------------------------------------------------------ inputs

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    for s in range(0, flat.numel(), 1 << 28):
        flat[s:s + (1 << 28)].normal_(0.0, std, generator=g)
    return t


def _table(pages, spare, seed):
    """Shuffled pages of every row, padded with -1, and how many there are with `spare` free ones."""
    order = list(range(sum(pages) + spare))
    random.Random(seed).shuffle(order)
    table, at = [], 0
    for n in pages:
        table.append(order[at:at + n] + [-1] * (max(pages) - n))
        at += n
    return table, len(order)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"tree": _tree_inputs, "cycle": _cycle_inputs, "compact": _compact_inputs, "logprobs": _logits_inputs,
            "grad": _logits_inputs}[case["op"]](case, seed, g)


def _caches(case, g, num_pages):
    shape = (num_pages, case["page"], case["hkv"], HEAD_DIM)
    return {"k": _normal(g, shape), "v": _normal(g, shape)}


def _tree_inputs(case, seed, g):
    lens, new = _lengths(case)
    rows = sum(new)
    table, num_pages = _table([-(-n // case["page"]) for n in lens], 4, seed)
    s = {"case": case, "lens": _i32(lens), "new": _i32(new), "starts": _i32([sum(new[:b]) for b in range(len(new))]),
         "table": _i32(table), "parents": _i32([p for row in _trees(case) for p in row]), "max_new": max(new),
         "max_len": max(lens), "rows": rows, **_caches(case, g, num_pages)}
    if case["peaky"]:
        gain = torch.ones((num_pages, case["page"]), dtype=torch.bfloat16, device="cuda")
        gain.masked_fill_(torch.rand(gain.shape, generator=g, device="cuda") < PEAKY_FRAC, PEAKY_GAIN)
        s["k"].mul_(gain[:, :, None, None])
    s["q"] = _normal(g, (rows, case["hq"], HEAD_DIM), case["qstd"])
    if case["slopes"]:
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["hq"] + 1, device="cuda", dtype=torch.float32) / case["hq"])
    if case["prefix"]:
        s["prefix"] = _i32(_prefixes(case))
    return s


def _cycle_inputs(case, seed, g):
    lens, forks, page = _contexts(case), case["forks"], case["page"]
    children = len(lens) * forks
    room = -(-(max(lens) + case["new"]) // page)
    pages = [-(-n // page) for n in lens]
    table, num_pages = _table(pages, case["free"], seed)
    table = [row + [-1] * (room - len(row)) for row in table] + [[-1] * room] * children
    refs = [0] * num_pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] = 1
    total = lens + [lens[c % len(lens)] for c in range(children)]  # after the fork
    return {"case": case, "table": _i32(table), "lens": _i32(lens + [0] * children), "refs": _i32(refs),
            "parents": _i32([-1] * len(lens) + [c % len(lens) for c in range(children)]),
            "want": _i32([n + case["new"] for n in total]), "longest": room, **_caches(case, g, num_pages)}


def _compact_inputs(case, seed, g):
    lens, new = _lengths(case)
    table, num_pages = _table([-(-n // case["page"]) for n in lens], 4, seed)
    kept = _kept(case)
    keep = [t for row, n in zip(kept, new) for t in row + [0] * (n - len(row))]
    return {"case": case, "lens": _i32(lens), "new": _i32(new), "starts": _i32([sum(new[:b]) for b in range(len(new))]),
            "table": _i32(table), "keep": _i32(keep), "keep_lens": _i32([len(row) for row in kept]), "rows": sum(new),
            **_caches(case, g, num_pages)}


def _logits_inputs(case, seed, g):
    rows, vocab = case["rows"], case["vocab"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    wide = -(-vocab // 8) * 8
    s = {"case": case, "logits": _normal(g, (rows, wide), 2.5, dtype)[:, :vocab],
         "mask": torch.tensor(_supervised(case), device="cuda").to(torch.uint8)}
    shape = (rows, case["given"]) if case["given"] > 1 else (rows,)
    s["tokens"] = torch.randint(0, vocab, shape, generator=g, device="cuda", dtype=torch.int32)
    # a sampled token is a likely one
    at = s["tokens"].view(rows, -1)[:, :1].long()
    s["logits"].scatter_add_(1, at, torch.rand(at.shape, generator=g, device="cuda").mul_(12.0).to(dtype))
    if case["op"] == "grad":
        s["by_logp"] = torch.randn(shape, generator=g, device="cuda") / rows
        if case["entropy"]:
            s["by_entropy"] = torch.randn((rows,), generator=g, device="cuda") / rows
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "tree":
        dtype = torch.float32 if case["out"] == "f32" else torch.bfloat16
        s["out"] = torch.empty((s["rows"], case["hq"], HEAD_DIM), dtype=dtype, device="cuda")
    if own and case["op"] in ("tree", "cycle", "compact"):  # a serving program keeps its handle
        from paper_2609_36608_amd import DecodeAttention

        hq = case.get("hq", case["hkv"])
        most = s["max_len"] if case["op"] == "tree" else s["table"].shape[1] * case["page"]
        s["attn"] = DecodeAttention(hq, case["hkv"], s["lens"].shape[0], most,
                                    out_dtype=s["out"].dtype if "out" in s else torch.bfloat16, page_tokens=case["page"])
    return s


# ------------------------------------------------------------------ the plain forms

def _plain_tree(s):
    """Every sequence padded to the longest: scores [batch, KV head, draft, head of the group, token]."""
    case, rows, tokens = s["case"], s["max_new"], s["max_len"]
    batch, hkv, g = case["batch"], case["hkv"], case["hq"] // case["hkv"]
    i = torch.arange(rows, device="cuda")
    starts, lens, new = (s[k].long() for k in ("starts", "lens", "new"))
    at = (starts[:, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"][at].float().view(batch, rows, hkv, g, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(batch, hkv, rows * g, HEAD_DIM)
    table = s["table"].long().clamp(min=0)
    k = s["k"][table].flatten(1, 2)[:, :tokens].permute(0, 2, 3, 1).float().contiguous()
    x = (q @ k).mul_(SCALE).view(batch, hkv, rows, g, tokens)
    if case["softcap"]:
        x = x.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    # ancestors: the powers of identity and parents count the ways from a draft to another, one or none
    parent = s["parents"].long()[at]
    padding = (parent >= i) | (i >= new[:, None])
    step = (parent[:, :, None] == i).double()  # padding rows' parents are none of these
    above = torch.linalg.matrix_power(torch.eye(rows, dtype=torch.float64, device="cuda") + step, rows) > 0
    above &= ~padding[:, :, None]
    pos = (lens - new)[:, None] + above.sum(-1) - 1
    t = torch.arange(tokens, device="cuda")
    draft = t - (lens - new)[:, None]  # of each token, below 0 before the drafts
    there = draft.clamp(0, rows - 1)
    token_pos = torch.where(draft < 0, t, pos.gather(1, there))
    far = pos[:, :, None] - token_pos[:, None, :]
    if case["slopes"]:
        x.sub_(s["slopes"].view(1, hkv, 1, g, 1) * far.float()[:, None, :, None])
    seen = torch.where(draft[:, None] < 0, ~padding[:, :, None], above.gather(2, there[:, None].expand(-1, rows, -1)))
    seen &= (draft < new[:, None])[:, None]
    if case["window"]:
        near = far < case["window"]
        if case["prefix"]:
            near |= t < s["prefix"][:, None, None]
        seen &= near
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)).exp_()
    total = x.sum(-1, keepdim=True).view(batch, hkv, rows * g, 1)
    v = s["v"][table].flatten(1, 2)[:, :tokens].permute(0, 2, 1, 3).float().contiguous()
    o = (x.view(batch, hkv, rows * g, tokens) @ v) / torch.where(total > 0, total, 1.0)
    o = o.view(batch, hkv, rows, g, HEAD_DIM).permute(0, 2, 1, 3, 4).reshape(batch, rows, case["hq"], HEAD_DIM)
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    s["out"].copy_(o[seq, row - starts[seq]])


def _count(refs, table, changed, by):
    """refs += by for the pages that `changed` entries of the table name."""
    named = changed & (table >= 0)
    refs.scatter_add_(0, table.clamp(min=0).flatten().long(), (named * by).flatten().int())


def _plain_fork(s, j):
    table, lens, refs, page = s["table"], s["lens"], s["refs"], s["case"]["page"]
    forked = (s["parents"] >= 0)[:, None]
    parent = s["parents"].long().clamp(min=0)
    _count(refs, table, forked & (j < (lens[:, None] + page - 1) // page), -1)
    lens.copy_(torch.where(forked[:, 0], lens[parent], lens))
    held = j < (lens[:, None] + page - 1) // page
    table.copy_(torch.where(forked, torch.where(held, table[parent], -1), table))
    _count(refs, table, forked & held, 1)


def _plain_resize(s, j, lens, want):
    """Rows that hold `lens` tokens get room for `want`: that or `lens`, and pages to copy."""
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    had, get = (lens + page - 1) // page, (want + page - 1) // page
    gone = (j >= get[:, None]) & (j < had[:, None])
    _count(refs, table, gone, -1)
    table.masked_fill_(gone, -1)
    last = table.gather(1, (had - 1).clamp(min=0).long()[:, None])[:, 0]
    copied = (want > lens) & (lens % page > 0) & (refs[last.clamp(min=0).long()] > 1) & (last >= 0)
    need = (get - had).clamp(min=0) + copied
    free = torch.cumsum(refs <= 0, 0)
    upto = torch.cumsum(need, 0)
    ok = ((upto <= free[-1]) | (need == 0)) & (get <= table.shape[1])
    rank = (upto - need)[:, None] + copied[:, None] + j - had[:, None]  # of an added page among the free ones
    added = ok[:, None] & (j >= had[:, None]) & (j < get[:, None])
    second = ok[:, None] & copied[:, None] & (j == had[:, None] - 1)
    rank = torch.where(second, (upto - need)[:, None], rank)
    fresh = torch.searchsorted(free, rank.clamp(min=0) + 1).int()
    _count(refs, table, second, -1)
    copies = torch.stack([torch.where(ok & copied, last, -1),
                          torch.where(second, fresh, -1).amax(1).int()], 1)
    table.copy_(torch.where(added | second, fresh, table))
    _count(refs, table, added | second, 1)
    return torch.where(ok, want, lens), copies


def _plain_copy(s, copies):
    src, dst = copies.long().unbind(1)
    # where nothing is copied, one of the copies again (page 0 to itself where there is none)
    some, there = dst.argmax(), dst >= 0
    src, dst = (torch.where(there, x, x[some].clamp(min=0)) for x in (src, dst))
    for name in ("k", "v"):
        s[name][dst] = s[name][src]


def _plain_cycle(s):
    j = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    _plain_fork(s, j)
    granted, copies = _plain_resize(s, j, s["lens"], s["want"])
    _plain_copy(s, copies)
    _plain_resize(s, j, granted, s["lens"])
    return granted


def _plain_compact(s):
    case, page = s["case"], s["case"]["page"]
    row = torch.arange(s["rows"], device="cuda")
    starts, lens, new = (s[k].long() for k in ("starts", "lens", "new"))
    seq = torch.searchsorted(starts, row, right=True) - 1
    i = row - starts[seq]
    hist = (lens - new)[seq]
    # tokens that are not kept stay where they are, in places that no kept one goes to
    stays = i >= s["keep_lens"].long()[seq]
    src = torch.where(stays, i, s["keep"].long())
    table = s["table"].long()
    place = lambda t: table[seq, t // page] * page + t % page  # noqa: E731
    src, dst = place(hist + src), place(hist + i)
    for name in ("k", "v"):
        flat = s[name].view(-1, case["hkv"], HEAD_DIM)
        flat[dst] = flat[src]
    return (lens - new).int() + s["keep_lens"]


def _plain_logprobs(s):
    case, live = s["case"], s["mask"][:, None] != 0
    x = s["logits"].float()
    tokens = s["tokens"].view(case["rows"], -1).long()
    res = {}
    if case["top"]:
        bits = (x + 0.0).view(torch.int32)  # without a negative zero
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
        order += (1 << 32) - 1 - torch.arange(case["vocab"], device="cuda")
        best = torch.topk(order, case["top"], dim=1).values
        del bits, order
        at = (1 << 32) - 1 - (best & 0xFFFFFFFF)
        res["top_tokens"] = torch.where(live, at, -1).int()
    scaled = x * (1.0 / case["temperature"])
    top = scaled.amax(1, keepdim=True)
    d = scaled.sub_(top)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    res["logp"] = torch.where(live, d.gather(1, tokens) - log_total, 0.0).view(s["tokens"].shape)
    if case["top"]:
        res["top_logp"] = torch.where(live, d.gather(1, at) - log_total, 0.0)
    if case["entropy"]:
        h = log_total - (e * d).sum(1, keepdim=True) / total
        res["entropy"] = torch.where(live, h, 0.0)[:, 0]
    return res, (d, e, total, log_total)


def _plain_grad(s):
    case, live = s["case"], s["mask"][:, None] != 0
    res, (d, e, total, log_total) = _plain_logprobs(s)
    p = e.div_(total)
    by = s["by_logp"].view(case["rows"], -1)
    grad = p * -by.sum(1, keepdim=True)
    if case["entropy"]:
        grad.sub_(d.sub_(log_total).add_(res["entropy"][:, None]).mul_(p).mul_(s["by_entropy"][:, None]))
    grad.scatter_add_(1, s["tokens"].view(case["rows"], -1).long(), by)
    grad.mul_(1.0 / case["temperature"])
    res["grad"] = torch.where(live, grad, 0.0).to(s["logits"].dtype)
    return res


# ------------------------------------------------------------------ the framework's calls

def _own_tree(s):
    from paper_2609_36608_amd import AttnScores

    case = s["case"]
    scores = AttnScores(softcap=case["softcap"], window=case["window"], slopes=s.get("slopes"),
                        prefix_lens=s.get("prefix"))
    s["attn"].tree_paged(s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], s["new"], s["parents"], s["max_new"],
                         SCALE, s["out"], scores=scores)


def _own_cycle(s):
    attn = s["attn"]
    attn.fork_pages(s["table"], s["lens"], s["refs"], s["parents"])
    granted, copies = attn.resize_pages(s["table"], s["lens"], s["want"], s["refs"])
    attn.copy_pages(s["k"], s["v"], copies)
    attn.resize_pages(s["table"], granted, s["lens"], s["refs"])
    return granted


def _own_compact(s):
    return s["attn"].compact_paged(s["k"], s["v"], s["table"], s["lens"], s["starts"], s["new"], s["keep"], s["keep_lens"])


def _own_logprobs(s):
    from paper_2609_36608_amd import token_logprobs

    case = s["case"]
    r = token_logprobs(s["logits"], s["tokens"], mask=s["mask"], temperature=case["temperature"], top=case["top"],
                       entropy=case["entropy"])
    res = {"logp": r["token_logp"]}
    if case["top"]:
        res["top_tokens"], res["top_logp"] = r["top_tokens"], r["top_logp"]
    if case["entropy"]:
        res["entropy"] = r["entropy"]
    return res, r


def _own_grad(s):
    from paper_2609_36608_amd import token_logprobs_grad

    res, r = _own_logprobs(s)
    res["grad"] = token_logprobs_grad(s["logits"], s["tokens"], r, s["by_logp"], grad_entropy=s.get("by_entropy"),
                                      mask=s["mask"], temperature=s["case"]["temperature"])
    return res


def run(s):
    op = s["case"]["op"]
    if op == "tree":
        _own_tree(s) if own else _plain_tree(s)
        return {"out": s["out"]}
    if op == "cycle":
        granted = _own_cycle(s) if own else _plain_cycle(s)
        return {"granted": granted, "k": s["k"], "lens": s["lens"], "refs": s["refs"], "table": s["table"], "v": s["v"]}
    if op == "compact":
        lens = _own_compact(s) if own else _plain_compact(s)
        return {"k": s["k"], "lens": lens, "v": s["v"]}
    if op == "logprobs":
        return (_own_logprobs(s) if own else _plain_logprobs(s))[0]
    return _own_grad(s) if own else _plain_grad(s)


# ------------------------------------------------------------------ 64-bit results

def _exact_tree(s):
    case = s["case"]
    lens, new = _lengths(case)
    g = case["hq"] // case["hkv"]
    out = torch.zeros((s["rows"], case["hq"], HEAD_DIM), dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m, prefix, row) in enumerate(zip(lens, new, _prefixes(case), _trees(case))):
        pages = s["table"][b, :-(-n // case["page"])].long()
        kb, vb = (s[name][pages].flatten(0, 1)[:n] for name in ("k", "v"))
        paths = _paths(row)
        place = torch.arange(n, dtype=torch.float64)
        seen = torch.zeros((m, n), dtype=torch.bool)
        for i, path in enumerate(paths):
            place[n - m + i] = n - m + len(path) - 1
        for i, path in enumerate(paths):
            if path:
                seen[i, :n - m] = True
                seen[i, [n - m + a for a in path]] = True
        far = place[n - m:, None] - place
        if case["window"]:
            seen &= (far < case["window"]) | (torch.arange(n) < prefix)
        hidden, far = ~seen.cuda(), far.cuda()
        for h in range(case["hkv"]):
            heads = slice(h * g, (h + 1) * g)
            q = s["q"][at:at + m, heads].double().transpose(0, 1).reshape(g * m, HEAD_DIM)
            x = (q @ kb[:, h].double().t().contiguous()).view(g, m, n) / math.sqrt(HEAD_DIM)
            if case["softcap"]:
                x = torch.tanh(x / case["softcap"]) * case["softcap"]
            if case["slopes"]:
                x = x - s["slopes"][heads].double()[:, None, None] * far
            weight = torch.softmax(x.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
            o = weight.view(g * m, n) @ vb[:, h].double().contiguous()
            out[at:at + m, heads] = o.view(g, m, HEAD_DIM).transpose(0, 1)
        at += m
    return {"out": out}


def _exact_cycle(s):
    """The same by lists: what every page of the caches holds at the end."""
    case, page = s["case"], s["case"]["page"]
    table, lens, refs = s["table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    source = list(range(len(refs)))
    for b, parent in enumerate(s["parents"].tolist()):
        if parent >= 0:
            lens[b], table[b] = lens[parent], list(table[parent])
            for p in table[b]:
                if p >= 0:
                    refs[p] += 1
    free = [p for p, n in enumerate(refs) if n == 0]
    granted, shared = list(lens), list(refs)
    for b, n in enumerate(lens):
        had, get = -(-n // page), -(-(n + case["new"]) // page)
        again = n % page > 0 and shared[table[b][had - 1]] > 1
        if len(free) < get - had + again:
            free = []
            continue
        if again:
            source[free.pop(0)] = table[b][had - 1]
        del free[:get - had]
        granted[b] = n + case["new"]
    k, v = (s[name].double()[torch.tensor(source, device="cuda")] for name in ("k", "v"))
    return {"granted": None, "k": k, "lens": None, "refs": None, "table": None, "v": v}


def _exact_compact(s):
    case, page = s["case"], s["case"]["page"]
    k, v = (s[name].double() for name in ("k", "v"))
    table = s["table"].tolist()
    src, dst = [], []
    for b, (n, m, row) in enumerate(zip(*_lengths(case), _kept(case))):
        for i, t in enumerate(row):
            src.append(table[b][(n - m + t) // page] * page + (n - m + t) % page)
            dst.append(table[b][(n - m + i) // page] * page + (n - m + i) % page)
    src, dst = (torch.tensor(x, device="cuda") for x in (src, dst))
    for x in (k, v):
        flat = x.view(-1, case["hkv"], HEAD_DIM)
        flat[dst] = flat[src].clone()
    return {"k": k, "lens": None, "v": v}


def _exact_logits(s):
    case, rows = s["case"], s["case"]["rows"]
    live = s["mask"] != 0
    tokens = s["tokens"].view(rows, -1).long()
    res = {"logp": torch.zeros(tokens.shape, dtype=torch.float64, device="cuda")}
    if case["entropy"]:
        res["entropy"] = torch.zeros((rows,), dtype=torch.float64, device="cuda")
    if case["top"]:
        res["top_logp"] = torch.zeros((rows, case["top"]), dtype=torch.float64, device="cuda")
        res["top_tokens"] = None
    if case["op"] == "grad":
        res["grad"] = torch.zeros((rows, case["vocab"]), dtype=torch.float64, device="cuda")
    for r in range(0, rows, 256):  # some rows at a time
        part = slice(r, r + 256)
        on = live[part, None].double()
        logp = torch.log_softmax(s["logits"][part].double() / case["temperature"], -1)
        p = logp.exp()
        h = -(p * logp).sum(-1)
        res["logp"][part] = logp.gather(1, tokens[part]) * on
        if case["entropy"]:
            res["entropy"][part] = h * on[:, 0]
        if case["top"]:
            res["top_logp"][part] = logp.sort(-1, descending=True).values[:, :case["top"]] * on
        if case["op"] == "grad":
            by = s["by_logp"].view(rows, -1)[part].double()
            grad = torch.zeros_like(p).scatter_add_(1, tokens[part], by) - p * by.sum(1, keepdim=True)
            if case["entropy"]:
                grad -= s["by_entropy"][part, None].double() * p * (logp + h[:, None])
            res["grad"][part] = grad / case["temperature"] * on
    res["logp"] = res["logp"].view(s["tokens"].shape)
    return res


def exact(case, seed):
    s = _inputs(case, seed)
    return {"tree": _exact_tree, "cycle": _exact_cycle, "compact": _exact_compact, "logprobs": _exact_logits,
            "grad": _exact_logits}[case["op"]](s)
