"""Drafted decoding with the operators as they are used together: forks of two contexts grow by a tree
of drafts a step (pages taken, shared ones copied, drafts appended with their rotations and attended),
the log probabilities choose the accepted path, its tokens are compacted and the pages past them given back.
What it emits and leaves in the caches has to be what decoding a token a step gives."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd.binding import DecodeAttention, Rotary, token_logprobs

from _gpu_util import dev, up_i32
from _paged_util import D, randn

pytestmark = pytest.mark.gpu

HQ, HKV, PAGE, WIDTH = 8, 2, 16, 16
VOCAB = HQ * D  # the outputs of a token's attention are its logits
SCALE = 0.2  # scores of up to 12 or so
NODES, LEVELS = 7, 3  # a binary tree below the token that was emitted last
CONTEXTS, FORKS = [37, 80], [-1, -1, 0, 1, 0]  # 80: its pages are full
FIRST = [3, 500, 77, 1000, 640]
STEPS = 10

# an fp32 output of either attention is off by 9e-5 at most (outputs of this size, scores below 30)
F32 = 9e-5


class Model:
    def __init__(self):
        g = torch.Generator().manual_seed(71)
        self.q, self.k, self.v = (randn(g, (VOCAB, h, D)).to(dev()) for h in (HQ, HKV, HKV))
        self.contexts = [torch.randint(0, VOCAB, (n,), generator=g) for n in CONTEXTS]
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2) / D)).float().to(dev())

    def append(self, attn, caches, tokens, table, lens, starts, new, positions=None):
        return attn.append_paged(self.k[tokens], self.v[tokens], *caches, table, lens, q=self.q[tokens], q_starts=starts,
                                 q_lens=new, rotary=Rotary(self.inv_freq, positions=positions))


def empty_caches(pages):
    return [torch.full((pages, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device=dev()) for _ in range(2)]


def one_by_one(model, steps):
    """Tokens, their log probabilities and the caches' rows of every sequence, a token a step."""
    seqs = len(FORKS)
    caches = empty_caches(seqs * WIDTH)
    table = torch.arange(seqs * WIDTH, dtype=torch.int32, device=dev()).view(seqs, WIDTH)
    origin = [b if p < 0 else p for b, p in enumerate(FORKS)]
    lens = [len(model.contexts[b]) for b in origin]
    tokens = torch.cat([model.contexts[b] for b in origin]).to(dev())
    starts = np.concatenate([[0], np.cumsum(lens)[:-1]])
    out = torch.empty((seqs, HQ, D), device=dev())
    streams, logps = [], []
    with DecodeAttention(HQ, HKV, seqs, WIDTH * PAGE, page_tokens=PAGE) as attn:
        model.append(attn, caches, tokens, table, up_i32(lens), up_i32(starts), up_i32(lens))
        pending, lens = torch.tensor(FIRST, device=dev()), up_i32(lens)
        for _ in range(steps):
            lens = lens + 1
            q = model.append(attn, caches, pending, table, lens, None, None)
            attn.run_paged(q, *caches, table, lens, SCALE, out)
            res = token_logprobs(out.view(seqs, VOCAB), top=2)
            # no near ties: the two attentions differ by 2 F32 in each logit at most
            assert (res["top_logp"][:, 0] - res["top_logp"][:, 1] > 5 * F32).all()
            pending = res["top_tokens"][:, 0].long()
            streams.append(pending)
            logps.append(res["top_logp"][:, 0])
        torch.cuda.synchronize()
    return torch.stack(streams, 1).cpu(), torch.stack(logps, 1).cpu(), [c.view(seqs, WIDTH * PAGE, HKV, D) for c in caches]


def guesses(streams):
    """Two drafts after each token: many of the first ones what follows it, others not."""
    rng = np.random.default_rng(72)
    guess = rng.integers(0, VOCAB, (VOCAB, 2))
    for first, row in zip(FIRST, streams.tolist()):
        for a, b in zip([first] + row, row):
            if rng.random() < 0.75:
                guess[a, rng.integers(0, 2)] = b
    return torch.from_numpy(guess).to(dev())


class Drafted:
    def __init__(self, model, guess, pages):
        self.model, self.guess = model, guess
        seqs = self.seqs = len(FORKS)
        i32 = dict(dtype=torch.int32, device=dev())
        self.attn = DecodeAttention(HQ, HKV, seqs, WIDTH * PAGE, page_tokens=PAGE)
        self.caches = empty_caches(pages)
        self.table = torch.full((seqs, WIDTH), -1, **i32)
        self.refs, self.lens = torch.zeros(pages, **i32), torch.zeros(seqs, **i32)
        self.pending = torch.zeros(seqs, dtype=torch.int64, device=dev())
        self.starts = torch.arange(seqs, **i32) * NODES
        self.parents = up_i32([-1, 0, 0, 1, 1, 2, 2] * seqs)
        self.depths = up_i32([0, 1, 1, 2, 2, 2, 2])
        self.out = torch.zeros((seqs * NODES, HQ, D), device=dev())
        self.start()

    def start(self):
        """The contexts and their forks, in place."""
        m, seqs = self.model, self.seqs
        self.refs.zero_(), self.lens.zero_(), self.table.fill_(-1)
        for c in self.caches:
            c.fill_(float("nan"))
        lens = CONTEXTS + [0] * (seqs - len(CONTEXTS))
        self.attn.resize_pages(self.table, self.lens, up_i32(lens), self.refs, granted=self.lens)
        starts = np.concatenate([[0], np.cumsum(lens)[:-1]])
        m.append(self.attn, self.caches, torch.cat(m.contexts).to(dev()), self.table, self.lens, up_i32(starts), up_i32(lens))
        self.attn.fork_pages(self.table, self.lens, self.refs, up_i32(FORKS))
        self.pending.copy_(torch.tensor(FIRST))

    def step(self):
        """One step, with nothing read on the host: what each sequence emitted (-1 past it), with the
        log probabilities."""
        attn, guess = self.attn, self.guess
        grown, copies = attn.resize_pages(self.table, self.lens, self.lens + NODES, self.refs)
        attn.copy_pages(*self.caches, copies)
        new = grown - self.lens  # none without room
        tokens = [self.pending]
        for i in range(NODES // 2):
            tokens += [guess[tokens[i], 0], guess[tokens[i], 1]]
        tokens = torch.stack(tokens, 1)
        positions = (self.lens[:, None] + self.depths).view(-1)
        q = self.model.append(attn, self.caches, tokens.view(-1), self.table, grown, self.starts, new, positions)
        attn.tree_paged(q, *self.caches, self.table, grown, self.starts, new, self.parents, NODES, SCALE, self.out)
        live = new > 0
        mask = live[:, None].expand(-1, NODES).reshape(-1).to(torch.uint8)
        res = token_logprobs(self.out.view(-1, VOCAB), mask=mask, top=1)
        best = res["top_tokens"].view(-1, NODES).long()
        logp = res["top_logp"].view(-1, NODES)
        node = torch.zeros_like(self.pending)
        count = live.int()
        keep = torch.zeros((self.seqs, NODES), dtype=torch.int32, device=dev())
        said, at = [], lambda x: x.gather(1, node[:, None])[:, 0]  # noqa: E731
        for level in range(LEVELS):
            said.append((torch.where(live, at(best), -1), torch.where(live, at(logp), 0.0)))
            if level == LEVELS - 1:
                break
            left = torch.clamp(2 * node + 1, max=NODES - 2)
            hit = [live & (tokens.gather(1, (left + i)[:, None])[:, 0] == at(best)) for i in range(2)]
            child = torch.where(hit[0], left, left + 1)
            live = hit[0] | hit[1]
            self.pending.copy_(torch.where(new > 0, at(best), self.pending))
            node = torch.where(live, child, node)
            keep[:, level + 1] = torch.where(live, node, 0).int()
            count = count + live.int()
        self.pending.copy_(torch.where(new > 0, at(best), self.pending))
        short = attn.compact_paged(*self.caches, self.table, grown, self.starts, new, keep.view(-1), count)
        attn.resize_pages(self.table, grown, short, self.refs, granted=self.lens)
        return torch.stack([s[0] for s in said], 1), torch.stack([s[1] for s in said], 1)


@pytest.mark.parametrize("pages", [40, 16], ids=["room", "few_pages"])
def test_drafts_are_what_one_by_one_gives(pages):
    model = Model()
    streams, logps, plain = one_by_one(model, STEPS * LEVELS)
    drafted = Drafted(model, guesses(streams), pages)
    emitted, sizes, eager = [[] for _ in FORKS], [[] for _ in FORKS], []
    for _ in range(STEPS):
        said, lp = drafted.step()
        eager.append((said.clone(), lp.clone(), drafted.table.clone(), drafted.lens.clone(), drafted.refs.clone()))
        for b, (row, rlp) in enumerate(zip(said.tolist(), lp.tolist())):
            emitted[b] += [t for t in row if t >= 0]
            sizes[b] += [x for t, x in zip(row, rlp) if t >= 0]
    counts = [len(e) for e in emitted]
    print("emitted", counts, flush=True)
    if pages == 40:
        assert all(STEPS < n for n in counts) and any(n < STEPS * LEVELS for n in counts)
    else:
        assert any((said < 0).all(1).any() for said, *_ in eager)  # rows that found no room
    base = [len(model.contexts[b if p < 0 else p]) for b, p in enumerate(FORKS)]
    assert drafted.lens.tolist() == [n + m for n, m in zip(base, counts)]
    table = drafted.table.cpu()
    held = np.zeros(pages, int)
    for b, n in enumerate(counts):
        assert emitted[b] == streams[b, :n].tolist(), b
        # each logit within 2 F32, and so their log-sum-exp
        assert np.allclose(sizes[b], logps[b, :n], rtol=0, atol=4 * F32 + 1e-5)
        length = base[b] + n
        for t in range(length):
            p = int(table[b, t // PAGE])
            for mine, theirs in zip(drafted.caches, plain):
                assert torch.equal(mine[p, t % PAGE], theirs[b, t]), (b, t)
        rows = table[b, :-(-length // PAGE)]
        held[rows.numpy()] += 1
        assert (table[b, len(rows):] == -1).all()
    assert drafted.refs.tolist() == held.tolist()
    # the step captured once, from the start again
    drafted.start()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        said, lp = drafted.step()
    for i, want in enumerate(eager):
        graph.replay()
        got = (said, lp, drafted.table, drafted.lens, drafted.refs)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i
    drafted.attn.close()
