"""Pages of paged caches: forks, resizes, copies and compaction against plain loops over lists.  All
results are whole numbers or moved bits, compared exactly."""
import numpy as np
import pytest
import torch

from paper_2609_36608_amd import CtxError, DecodeAttention

pytestmark = pytest.mark.gpu
D = 128


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Pool:
    """Tables, lengths and counts as lists."""

    def __init__(self, seqs, width, page, pages):
        self.page, self.width = page, width
        self.table = [[-1] * width for _ in range(seqs)]
        self.lens = [0] * seqs
        self.refs = [0] * pages

    def held(self, n):
        return -(-max(min(n, self.width * self.page), 0) // self.page)

    def count(self, page, by):
        if 0 <= page < len(self.refs):
            self.refs[page] += by

    def fork(self, parents):
        n = len(self.lens)
        forked = lambda b: 0 <= parents[b] < n and parents[b] != b  # noqa: E731
        for b in [b for b in range(n) if forked(b) and not forked(parents[b])]:
            for j in range(self.held(self.lens[b])):
                self.count(self.table[b][j], -1)
            self.lens[b] = self.lens[parents[b]]
            m = self.held(self.lens[b])
            self.table[b] = self.table[parents[b]][:m] + [-1] * (self.width - m)
            for p in self.table[b][:m]:
                self.count(p, 1)

    def resize(self, new):
        copies = [[-1, -1] for _ in new]
        for b, n in enumerate(new):
            for j in range(self.held(n), self.held(self.lens[b])):
                self.count(self.table[b][j], -1)
                self.table[b][j] = -1
        free = [p for p, c in enumerate(self.refs) if c <= 0]
        shared = list(self.refs)
        for b, n in enumerate(new):
            n, old = max(n, 0), max(min(self.lens[b], self.width * self.page), 0)
            self.lens[b] = old
            if n <= old:
                self.lens[b] = n
                continue
            if n > self.width * self.page:
                continue
            had, get = self.held(old), self.held(n)
            last = self.table[b][had - 1] if old % self.page else -1
            again = 0 <= last < len(shared) and shared[last] > 1
            need = get - had + again
            if need > len(free):
                free = []
                continue
            if again:
                copies[b] = [last, free[0]]
                self.count(last, -1)
                self.table[b][had - 1] = free.pop(0)
                self.refs[copies[b][1]] = 1
            for j in range(had, get):
                self.table[b][j] = free.pop(0)
                self.refs[self.table[b][j]] = 1
            self.lens[b] = n
        return copies


class OnDevice:
    def __init__(self, pool, hkv=2):
        self.table, self.lens, self.refs = i32(pool.table), i32(pool.lens), i32(pool.refs)
        self.attn = DecodeAttention(hkv, hkv, len(pool.lens), pool.width * pool.page, page_tokens=pool.page)

    def resize(self, new, in_place=True):
        granted, copies = self.attn.resize_pages(self.table, self.lens, i32(new), self.refs,
                                                 granted=self.lens if in_place else None)
        self.lens = granted
        return copies

    def check(self, pool, what=""):
        assert self.lens.tolist() == pool.lens, what
        assert self.table.tolist() == pool.table, what
        assert self.refs.tolist() == pool.refs, what


@pytest.mark.parametrize("seqs,width,page,pages", [(1, 1, 16, 1), (3, 4, 16, 9), (40, 30, 16, 500), (130, 260, 32, 9000),
                                                   (1500, 9, 16, 3000), (7, 600, 48, 70001)])
def test_random_lives(seqs, width, page, pages):
    """Rows grow, shrink, empty and fork, also past what the pool has."""
    rng = np.random.default_rng(seqs)
    pool = Pool(seqs, width, page, pages)
    dev = OnDevice(pool)
    for step in range(14):
        if step % 3 == 2:
            parents = np.where(rng.random(seqs) < 0.4, rng.integers(-1, seqs + 1, seqs), -1).tolist()
            dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32(parents))
            pool.fork(parents)
            dev.check(pool, f"fork {step}")
            continue
        kind = rng.integers(0, 4, seqs)
        most = width * page
        new = np.select([kind == 0, kind == 1, kind == 2],
                        [np.array(pool.lens) + rng.integers(0, 70, seqs), rng.integers(-3, most + 2, seqs),
                         np.array(pool.lens)], rng.integers(0, max(2, pages * page // seqs), seqs))
        if step == 10:
            new[:] = 0
        copies = dev.resize(new.tolist(), in_place=bool(step % 2))
        assert copies.tolist() == pool.resize(new.tolist()), step
        dev.check(pool, f"resize {step}")
    # every held page is counted, every other free
    held = np.zeros(pages, int)
    for row, n in zip(pool.table, pool.lens):
        for p in row[:pool.held(n)]:
            held[p] += 1
    assert held.tolist() == pool.refs


def test_pool_runs_out():
    pool = Pool(5, 6, 16, 10)
    dev = OnDevice(pool)
    for new in ([90, 20, 0, 10, 0], [96, 20, 64, 16, 5], [0, 20, 64, 16, 5], [0, 33, 64, 17, 97], [0] * 5):
        copies = dev.resize(new)
        assert copies.tolist() == pool.resize(new)
        dev.check(pool, str(new))
    assert pool.refs == [0] * 10


@pytest.mark.parametrize("seqs,pages", [(6, 24), (20, 100), (64, 300)])
def test_state_in_one_buffer(seqs, pages):
    """Lengths, tables, counts and outputs right behind each other: what is counted shares cache lines
    with what is read before, in either order."""
    rng = np.random.default_rng(seqs)
    width, page = 4, 16
    for order in (["lens", "new", "refs", "table"], ["table", "refs", "new", "lens"], ["refs", "lens", "table", "new"]):
        pool = Pool(seqs, width, page, pages)
        sizes = dict(lens=seqs, new=seqs, refs=pages, table=seqs * width)
        ws = (2 * seqs + pages + 3) // 4 * 4
        state = torch.zeros(ws + sum(sizes.values()), dtype=torch.int32, device="cuda")
        part, at = {}, ws
        for name in order:
            part[name] = state[at:at + sizes[name]]
            at += sizes[name]
        table = part["table"].view(seqs, width)
        table.fill_(-1)
        with DecodeAttention(2, 2, seqs, width * page, page_tokens=page) as attn:
            for step in range(12):
                new = rng.integers(0, width * page + 1, seqs).tolist()
                part["new"].copy_(i32(new))
                granted, copies = attn.resize_pages(table, part["lens"], part["new"], part["refs"], granted=part["lens"],
                                                    workspace=state[:ws].view(torch.uint8))
                want = pool.resize(new)
                assert granted.tolist() == pool.lens and copies.tolist() == want, (order, step)
                assert table.tolist() == pool.table and part["refs"].tolist() == pool.refs, (order, step)


def test_no_pages_and_broken_tables():
    pool = Pool(3, 2, 16, 0)
    dev = OnDevice(pool)
    dev.resize([5, 0, 40])
    pool.resize([5, 0, 40])
    dev.check(pool)
    # entries that name no page hold none
    pool = Pool(3, 4, 16, 6)
    pool.table = [[5, -7, 99, -1], [2, 3, -1, -1], [-1] * 4]
    pool.lens, pool.refs = [40, 20, 0], [0, 0, 1, 1, 0, 1]
    dev = OnDevice(pool)
    dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32([-1, -1, 0]))
    pool.fork([-1, -1, 0])
    dev.check(pool, "fork")
    copies = dev.resize([50, 25, 64])
    assert copies.tolist() == pool.resize([50, 25, 64])
    dev.check(pool, "resize")
    copies = dev.resize([0, 0, 0])
    pool.resize([0, 0, 0])
    dev.check(pool, "free")


def test_forks_of_forks_stay_as_they_are():
    pool = Pool(6, 3, 16, 20)
    dev = OnDevice(pool)
    new = [40, 17, 5, 0, 48, 1]
    dev.resize(new), pool.resize(new)
    for parents in ([-1, 0, 1, 2, 0, 5], [1, 0, -1, 3, 6, -9], [1, 2, 0, 2, 2, 2]):
        dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32(parents))
        pool.fork(parents)
        dev.check(pool, str(parents))


def caches(seed, pages, page, hkv):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((pages, page, hkv, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]


@pytest.mark.parametrize("page,hkv", [(16, 1), (16, 8), (48, 5), (256, 16)])
def test_copies(page, hkv):
    pages = 30
    k, v = caches(1, pages, page, hkv)
    k[3, 0, 0, 5] = float("nan")
    want = [x.view(torch.int16).clone() for x in (k, v)]
    copies = [[3, 7], [-1, -1], [3, 0], [5, 5], [29, 12], [30, 1], [2, 30], [-1, 4], [6, -1], [8, 28]]
    for x in want:
        old = x.clone()
        for s, d in copies:
            if 0 <= s < pages and 0 <= d < pages:
                x[d] = old[s]
    with DecodeAttention(hkv, hkv, 4, 64, page_tokens=page) as attn:
        attn.copy_pages(k, v, i32(copies))
        attn.copy_pages(k, v, torch.empty((0, 2), dtype=torch.int32).cuda())
    assert torch.equal(k.view(torch.int16), want[0]) and torch.equal(v.view(torch.int16), want[1])


class Kept:
    """A batch of sequences with shuffled pages and what of their last tokens is kept."""

    def __init__(self, seed, lens, new, kept, page, hkv, gap=2):
        rng = np.random.default_rng(seed)
        self.page, self.hkv, self.lens, self.new, self.kept = page, hkv, lens, new, kept
        pages = [-(-max(n, 0) // page) for n in lens]
        order = rng.permutation(sum(pages) + 3)
        self.table = np.full((len(lens), max(pages + [0]) + 1), -1, np.int32)
        at = 0
        for b, m in enumerate(pages):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.starts, row = np.zeros(len(lens), np.int32), gap
        for b in rng.permutation(len(lens)):
            self.starts[b] = row
            row += new[b] + gap
        self.rows = row
        self.keep = np.full(row, -5, np.int32)
        for b, x in enumerate(kept):
            self.keep[self.starts[b]:self.starts[b] + len(x)] = x
        self.k, self.v = caches(seed, len(order), page, hkv)

    def row(self, b, t):
        return int(self.table[b, t // self.page]) * self.page + t % self.page

    def want(self):
        out = []
        for x in (self.k, self.v):
            flat = x.view(torch.int16).clone().view(-1, self.hkv * D)
            old = flat.clone()
            for b, (n, m, kept) in enumerate(zip(self.lens, self.new, self.kept)):
                src = [self.row(b, n - m + t) for t in kept]
                dst = [self.row(b, n - m + i) for i in range(len(kept))]
                flat[dst] = old[src]
            # places past a sequence's kept tokens stay as they were
            out.append(flat.view(x.shape))
        return out

    def run(self, **kw):
        with DecodeAttention(self.hkv, self.hkv, len(self.lens), 4096, page_tokens=self.page) as attn:
            return attn.compact_paged(self.k, self.v, i32(self.table), i32(self.lens), i32(self.starts), i32(self.new),
                                      i32(self.keep), i32([len(x) for x in self.kept]), **kw)


def some(rng, n, share):
    return np.nonzero(rng.random(n) < share)[0].tolist()


@pytest.mark.parametrize("seed,page,hkv,lens,new", [
    (1, 16, 1, [1], [1]),
    (2, 16, 2, [40, 3, 17, 0], [9, 3, 0, 0]),
    (3, 16, 8, [100, 1000, 333], [100, 64, 128]),
    (4, 48, 4, [1000, 2000], [1000, 1999]),
    (5, 64, 5, [4000, 129, 128, 127], [4000, 129, 128, 127]),
    (6, 16, 8, list(range(20, 84)), [n // 2 for n in range(20, 84)]),
])
@pytest.mark.parametrize("share", [0.0, 0.1, 0.5, 0.95, 1.0])
def test_compaction(seed, page, hkv, lens, new, share):
    rng = np.random.default_rng(seed)
    c = Kept(seed, lens, new, [some(rng, m, share) for m in new], page, hkv)
    want = c.want()
    got = c.run()
    assert got.tolist() == [n - m + len(x) for n, m, x in zip(c.lens, c.new, c.kept)]
    assert torch.equal(c.k.view(torch.int16), want[0]) and torch.equal(c.v.view(torch.int16), want[1])


def test_compaction_leaves_out_what_is_not_there():
    """Kept tokens outside the sequence's, rows outside the list and entries that name no page."""
    c = Kept(9, [70, 70, 70], [30, 30, 30], [[1, 4, 29], [2, 99, -4, 7], [5, 6]], 16, 2)
    c.table[2, 2:] = 1000  # tokens 32 ..
    old = [x.clone() for x in (c.k, c.v)]
    new = torch.full((3,), -1, dtype=torch.int32).cuda()
    with DecodeAttention(2, 2, 3, 4096, page_tokens=16) as attn:
        starts = i32([c.starts[0], c.starts[1], c.starts[2]])
        attn.compact_paged(c.k, c.v, i32(c.table), i32(c.lens), starts, i32(c.new), i32(c.keep), i32([3, 4, 2]),
                           new_lens=new)
        assert new.tolist() == [43, 44, 42]
        for x, was in ((c.k, old[0]), (c.v, old[1])):
            x, was = x.view(-1, 2, D), was.view(-1, 2, D)
            assert torch.equal(x[c.row(0, 42)], was[c.row(0, 69)]) and torch.equal(x[c.row(1, 40)], was[c.row(1, 42)])
            assert torch.equal(x[c.row(1, 43)], was[c.row(1, 47)])
            assert torch.equal(x[c.row(1, 41)], was[c.row(1, 41)])  # its token is none
            touched = {c.row(0, 40), c.row(0, 41), c.row(0, 42), c.row(1, 40), c.row(1, 43)}
            rest = [r for r in range(x.shape[0]) if r not in touched]
            assert torch.equal(x[rest], was[rest])
        # rows past the list
        now = [x.clone() for x in (c.k, c.v)]
        far = i32([c.rows - 1, -2, 2 ** 31 - 1])
        attn.compact_paged(c.k, c.v, i32(c.table[:, :1]), i32(c.lens), far, i32(c.new), i32(c.keep), i32([3, 4, 2]))
        assert torch.equal(c.k, now[0]) and torch.equal(c.v, now[1])


def test_forked_row_gets_its_own_page():
    """What a fork appends is not seen by its parent."""
    hkv, page = 2, 16
    pool = Pool(3, 4, page, 9)
    k, v = caches(3, 9, page, hkv)
    with DecodeAttention(hkv, hkv, 3, 64, page_tokens=page) as attn:
        table, lens, refs = i32(pool.table), i32(pool.lens), i32(pool.refs)
        lens, _ = attn.resize_pages(table, lens, i32([20, 0, 0]), refs)
        attn.fork_pages(table, lens, refs, i32([-1, 0, 0]))
        before = k.view(-1, hkv, D)[[int(table[0, t // page]) * page + t % page for t in range(20)]].clone()
        lens, copies = attn.resize_pages(table, lens, lens + i32([0, 1, 2]), refs)
        attn.copy_pages(k, v, copies)
        new = torch.randn(3, hkv, D, device="cuda").to(torch.bfloat16)
        attn.append_paged(new, new, k, v, table, lens, q_starts=i32([0, 0, 1]), q_lens=i32([0, 1, 2]))
        rows = lambda b, n: k.view(-1, hkv, D)[[int(table[b, t // page]) * page + t % page for t in range(n)]]  # noqa: E731
        for b, n in ((0, 20), (1, 21), (2, 22)):
            assert torch.equal(rows(b, 20), before), b
        assert torch.equal(rows(1, 21)[20:], new[:1]) and torch.equal(rows(2, 22)[20:], new[1:])
        assert sorted(refs.tolist()) == [0, 0, 0, 0, 0, 1, 1, 1, 3]


def test_graph_of_a_cycle():
    """Fork, growth, copies and trim captured once and replayed."""
    hkv, page, seqs = 2, 16, 12
    pool = Pool(seqs, 20, page, 400)
    dev = OnDevice(pool, hkv)
    k, v = caches(4, 400, page, hkv)
    first = [37, 100, 16, 250] + [0] * 8
    dev.resize(first), pool.resize(first)
    parents = [-1] * 4 + [b % 4 for b in range(8)]
    pd, extra = i32(parents), i32([11] * seqs)

    def cycle():
        dev.attn.fork_pages(dev.table, dev.lens, dev.refs, pd)
        want = dev.lens + extra
        granted, copies = dev.attn.resize_pages(dev.table, dev.lens, want, dev.refs)
        dev.attn.copy_pages(k, v, copies)
        dev.attn.resize_pages(dev.table, granted, dev.lens, dev.refs)
        return granted, copies

    cycle()
    pool.fork(parents)
    now = list(pool.lens)
    pool.resize([n + 11 for n in now])
    pool.resize(now)
    dev.check(pool, "eager")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        granted, copies = cycle()
    for r in range(4):
        graph.replay()
        pool.fork(parents)
        want = pool.resize([n + 11 for n in now])
        assert granted.tolist() == pool.lens and copies.tolist() == want, r
        pool.resize(now)
        dev.check(pool, f"replay {r}")


def test_refusals():
    pool = Pool(3, 4, 16, 6)
    dev = OnDevice(pool)
    k, v = caches(1, 6, 16, 2)
    with pytest.raises(ValueError, match="parents"):
        dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32([-1, -1]))
    with pytest.raises(TypeError):
        dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32([-1, -1, 0]).long())
    with pytest.raises(ValueError):
        dev.attn.resize_pages(dev.table, dev.lens, i32([1, 2, 3, 4]), dev.refs)
    with pytest.raises(ValueError):
        dev.attn.resize_pages(dev.table[:2].contiguous(), dev.lens, i32([1, 2, 3]), dev.refs)
    with pytest.raises(CtxError, match="workspace"):
        dev.attn.resize_pages(dev.table, dev.lens, dev.lens, dev.refs, workspace=torch.empty(8, dtype=torch.uint8).cuda())
    with pytest.raises(ValueError):
        dev.attn.copy_pages(k, v[:4], i32([[0, 1]]))
    with pytest.raises(ValueError):
        dev.attn.copy_pages(k, v, i32([0, 1]))
    with pytest.raises(CtxError, match="new_lens"):
        dev.attn.compact_paged(k, v, dev.table, dev.lens, dev.lens, dev.lens, dev.lens, dev.lens, new_lens=dev.lens)
    with DecodeAttention(2, 2, 3, 64) as plain, pytest.raises(CtxError, match="page_tokens"):
        plain.fork_pages(dev.table, dev.lens, dev.refs, i32([-1, -1, 0]))
    dev.attn.close()
    with pytest.raises(RuntimeError):
        dev.attn.fork_pages(dev.table, dev.lens, dev.refs, i32([-1, -1, 0]))
