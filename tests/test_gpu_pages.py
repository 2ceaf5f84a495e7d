"""GPU tests of the page bookkeeping against a plain model in Python, and of the bytes that move: everything is exact."""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
PAGE = 16


class Model:
    """The definition: reference counts and rows of pages as Python lists."""

    def __init__(self, nb, rows, cols):
        self.refs, self.rows, self.lens, self.cols = [0] * nb, [[] for _ in range(rows)], [0] * rows, cols

    def free(self, rows):
        for r in rows:
            for p in self.rows[r]:
                self.refs[p] -= 1
            self.rows[r], self.lens[r] = [], 0

    def fork(self, requests, extra):
        """Returns the copy pairs; refuses by the rules of the call."""
        old_rows, old_lens = [list(r) for r in self.rows], list(self.lens)
        writer, pairs, out_of_pages, refused = {}, [], False, 0
        for i, (_, d) in enumerate(requests):
            writer.setdefault(d, i)
        free = [p for p, c in enumerate(self.refs) if c == 0]
        for i, (s, d) in enumerate(requests):
            pair = (-1, -1)
            length = old_lens[s] if s >= 0 else 0
            whole, need = length // PAGE, -(-(length + extra) // PAGE)
            good = writer[d] == i and need <= self.cols
            if s != d:
                good = good and not old_rows[d] and old_lens[d] == 0
                if s >= 0 and s in writer and requests[writer[s]][0] != s:
                    good = False
            if not good:
                refused += 1
                pairs.append(pair)
                continue
            fresh = max(0, need - (len(old_rows[d]) if s == d else whole))
            if fresh > 0 and (out_of_pages or fresh > len(free)):
                out_of_pages = True
                pairs.append(pair)
                continue
            pages, free = free[:fresh], free[fresh:]
            for p in pages:
                self.refs[p] = 1
            if s == d:
                self.rows[d] = old_rows[d] + pages
            else:
                shared = old_rows[s][:whole] if s >= 0 else []
                for p in shared:
                    self.refs[p] += 1
                self.rows[d], self.lens[d] = shared + pages, length
                if length % PAGE:
                    pair = (old_rows[s][whole], pages[0])
            pairs.append(pair)
        return pairs, refused, out_of_pages

    def compact(self):
        n = sum(c > 0 for c in self.refs)
        high = [p for p, c in enumerate(self.refs) if c > 0 and p >= n]
        low = [p for p in range(n) if self.refs[p] == 0]
        move = dict(zip(high, low))
        for a, b in move.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[move.get(p, p) for p in r] for r in self.rows]
        return list(zip(high, low)), n

    def table(self):
        t = np.full((len(self.rows), self.cols), -1, np.int32)
        for i, r in enumerate(self.rows):
            t[i, :len(r)] = r
        return t


class Pool:
    def __init__(self, dev, nb, rows, cols, hkv=2, d=64, layers=0, pad=0):
        self.dev, self.model = dev, Model(nb, rows, cols)
        wide = torch.full((rows, cols + pad), -1, dtype=torch.int32, device=dev)
        wide[:, cols:] = 77
        self.wide, self.table = wide, wide[:, :cols]
        self.lens = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.refs = torch.zeros(nb, dtype=torch.int32, device=dev)
        shape = ((layers,) if layers else ()) + (nb, hkv, PAGE, d)
        self.k, self.v = (torch.randn(shape, device=dev).bfloat16() for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def ints(self, x):
        return torch.tensor(list(x), dtype=torch.int32, device=self.dev)

    def fork(self, requests, extra, copy=True, expect=0):
        pairs = rpx.pages_fork(self.table, self.lens, self.refs, self.ints(s for s, _ in requests),
                               self.ints(d for _, d in requests), extra, device_status=self.status)
        want, refused, short = self.model.fork(requests, extra)
        assert list(zip(*(p.tolist() for p in pairs))) == want
        self.expect(expect)
        if copy:
            rpx.cache_copy_pages(self.k, self.v, *pairs, device_status=self.status)
        return refused, short

    def free(self, rows):
        rpx.pages_free(self.table, self.lens, self.refs, self.ints(rows), device_status=self.status)
        self.model.free(dict.fromkeys(rows))

    def set_len(self, row, n):
        self.lens[row] = n
        self.model.lens[row] = n

    def expect(self, status):
        assert int(self.status.item()) == status
        self.status.zero_()

    def check(self):
        assert np.array_equal(self.table.cpu().numpy(), self.model.table())
        assert self.refs.tolist() == self.model.refs and self.lens.tolist() == self.model.lens
        assert bool((self.wide[:, self.table.shape[1]:] == 77).all())

    def tokens(self, row):
        """K of a row's cached tokens (all layers)."""
        n = self.model.lens[row]
        pages = torch.tensor(self.model.rows[row], device=self.dev)[:-(-n // PAGE)].long()
        x = self.k[..., pages, :, :, :].movedim(-2, -4 + 1)
        return x.reshape(*x.shape[:-4], -1, *x.shape[-2:])[..., :n, :, :]


def test_new_rows_grow_and_free(cuda_device):
    p = Pool(cuda_device, 40, 6, 12, pad=3)
    p.fork([(-1, 0), (-1, 3)], 50)        # 4 pages each
    p.check()
    p.fork([(-1, 1)], 0)                  # a sequence of nothing
    p.check()
    p.set_len(0, 50)
    p.fork([(0, 0), (3, 3)], 20)          # 70 tokens: one more; 20 from none: nothing new
    p.check()
    assert len(p.model.rows[0]) == 5 and len(p.model.rows[3]) == 4
    p.free([3, 1, 3])                     # a row twice
    p.check()
    p.fork([(-1, 5)], 33)                 # the lowest free pages are those of row 3
    p.check()
    assert p.model.rows[5] == [4, 5, 6]
    p.expect(0)


@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 32, 47])
@pytest.mark.parametrize("extra", [0, 1, 16, 40])
def test_branches_share_whole_pages(cuda_device, length, extra):
    p = Pool(cuda_device, 64, 5, 8, layers=2)
    p.fork([(-1, 0)], 60)
    p.set_len(0, length)
    want = p.tokens(0)
    p.fork([(0, 2), (0, 4)], extra)
    p.check()
    for r in (2, 4):
        assert torch.equal(p.tokens(r), want)
        assert p.model.rows[r][:length // PAGE] == p.model.rows[0][:length // PAGE]
    own = [q for r in (2, 4) for q in p.model.rows[r][length // PAGE:]]
    assert len(set(own)) == len(own)
    p.free([0])
    p.check()
    for r in (2, 4):
        assert torch.equal(p.tokens(r), want)  # the branches live on


def test_refusals_change_nothing(cuda_device):
    p = Pool(cuda_device, 30, 8, 6)
    p.fork([(-1, 0), (-1, 1)], 30)
    p.set_len(0, 20)
    p.set_len(1, 30)
    # the same destination twice; a destination that holds pages; a row forked into and from; too many pages for the table
    refused, _ = p.fork([(0, 2), (1, 2), (0, 1), (2, 3), (0, 4)], 10, expect=-8)
    assert refused == 3
    p.check()
    assert len(p.model.rows[2]) == 2 and len(p.model.rows[4]) == 2
    refused, _ = p.fork([(1, 5)], 6 * PAGE, expect=-8)
    assert refused == 1
    p.check()
    # rows outside the table
    for src, dst in ((0, 8), (0, -1), (8, 6), (-2, 6)):
        pairs = rpx.pages_fork(p.table, p.lens, p.refs, p.ints([src]), p.ints([dst]), 5, device_status=p.status)
        assert [x.tolist() for x in pairs] == [[-1], [-1]]
        p.expect(-8)
        p.check()
    # a length beyond the held pages
    p.lens[4] = 40
    rpx.pages_fork(p.table, p.lens, p.refs, p.ints([4]), p.ints([6]), 5, device_status=p.status)
    p.expect(-8)
    p.lens[4] = 20
    p.check()
    rpx.pages_free(p.table, p.lens, p.refs, p.ints([8, -1]), device_status=p.status)
    p.expect(-8)
    p.check()


def test_too_few_pages(cuda_device):
    p = Pool(cuda_device, 10, 8, 12)
    p.fork([(-1, 0)], 16 * 6)
    p.set_len(0, 16 * 5)
    # 2 pages, then 3 that are not there, then 1 that a later request does not get, then one that needs none
    p.model.lens[1] = 0
    _, short = p.fork([(0, 1), (0, 2), (0, 3)], 32, expect=-10)
    assert short
    p.check()
    assert p.model.rows[1] and p.model.rows[2] and not p.model.rows[3]
    p.fork([(0, 4)], 0)
    p.check()


def test_double_counted_entries_are_reported(cuda_device):
    p = Pool(cuda_device, 12, 2, 4)
    p.table[0, 0] = 5   # nobody counted for it
    p.table[0, 1] = 99  # not a page
    rpx.pages_free(p.table, p.lens, p.refs, p.ints([0]), device_status=p.status)
    p.expect(-8)
    assert p.refs.tolist() == [0] * 12 and bool((p.table[0] == -1).all())


@pytest.mark.parametrize("nb,seed", [(1, 0), (7, 1), (1000, 2), (1024, 3), (4096, 6), (4097, 7), (5000, 4), (40000, 5)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compaction(cuda_device, nb, seed, in_place):
    rng = np.random.default_rng(seed)
    rows, cols = 9, max(1, min(nb // 4, 900 if nb == 4096 else nb))
    p = Pool(cuda_device, nb, rows, cols, pad=2, hkv=1)
    for r in range(rows - 1):
        take = rng.permutation(nb)[:rng.integers(0, max(1, nb // 10) + 1)][:cols]
        take = [int(q) for q in take if p.model.refs[q] == 0 or rng.random() < 0.1]
        p.model.rows[r] = take
        for q in take:
            p.model.refs[q] += 1
    p.table.copy_(torch.from_numpy(p.model.table()))
    p.refs.copy_(torch.tensor(p.model.refs, dtype=torch.int32))
    table, refs = p.table.clone(), p.refs.clone()
    before = [p.k[torch.tensor(r, dtype=torch.long, device=cuda_device)].clone() for r in p.model.rows]
    kw = {} if in_place else dict(table_out=p.table, ref_counts_out=torch.full_like(p.refs, 9))
    src_table = p.table if in_place else table
    src, dst, n_live = rpx.pages_compact(src_table, p.refs, device_status=p.status, **kw)
    moves, n = p.model.compact()
    assert int(n_live.item()) == n
    assert list(zip(src.tolist(), dst.tolist())) == moves + [(-1, -1)] * (nb // 2 - len(moves))
    rpx.cache_copy_pages(p.k, p.v, src, dst, device_status=p.status)
    if not in_place:
        assert torch.equal(p.refs, refs)  # the input stays
        p.refs.copy_(kw["ref_counts_out"])
    p.expect(0)
    p.check()
    for r, x in zip(p.model.rows, before):
        assert torch.equal(p.k[torch.tensor(r, dtype=torch.long, device=cuda_device)], x)


def test_compaction_of_a_full_and_an_empty_pool(cuda_device):
    for refs in ([1] * 50, [0] * 50, [0] * 49 + [3]):
        p = Pool(cuda_device, 50, 2, 50)
        p.model.refs = list(refs)
        p.model.rows[0] = [i for i, c in enumerate(refs) if c]
        p.table.copy_(torch.from_numpy(p.model.table()))
        p.refs.copy_(torch.tensor(refs, dtype=torch.int32))
        src, dst, n_live = rpx.pages_compact(p.table, p.refs, device_status=p.status)
        moves, n = p.model.compact()
        assert int(n_live.item()) == n and src.tolist()[:len(moves)] == [a for a, _ in moves]
        p.expect(0)
        p.check()


def test_compaction_reports_stale_entries(cuda_device):
    p = Pool(cuda_device, 20, 2, 4)
    p.refs[15] = 1
    p.table[0, 0], p.table[0, 1], p.table[1, 0], p.table[1, 1] = 15, 3, 18, 25
    rpx.pages_compact(p.table, p.refs, device_status=p.status)
    p.expect(-8)
    assert p.table.tolist() == [[0, -1, -1, -1], [-1, -1, -1, -1]]


@pytest.mark.parametrize("hkv,d,layers", [(1, 64, 0), (4, 128, 3), (8, 128, 1), (3, 64, 2)])
def test_copying_pages(cuda_device, hkv, d, layers):
    p = Pool(cuda_device, 700, 1, 1, hkv=hkv, d=d, layers=layers)
    perm = np.random.default_rng(0).permutation(700)
    src, dst = perm[:300].copy(), perm[300:600].copy()
    src[1], src[5] = src[0], src[0]  # one page to several places
    src[::7], dst[::7] = -1, -1
    k, v = p.k.clone(), p.v.clone()
    keep = src >= 0
    a, b = (torch.from_numpy(x[keep]).long().to(cuda_device) for x in (src, dst))
    for t in (k, v):
        if layers:
            t[:, b] = t[:, a]
        else:
            t[b] = t[a]
    rpx.cache_copy_pages(p.k, p.v, p.ints(src), p.ints(dst), device_status=p.status)
    p.expect(0)
    assert torch.equal(p.k, k) and torch.equal(p.v, v)
    rpx.cache_copy_pages(p.k, p.v, p.ints([3, 700, 4]), p.ints([699, 2, -1]), device_status=p.status)
    p.expect(-8)
    if layers:
        k[:, 699], v[:, 699] = k[:, 3], v[:, 3]
    else:
        k[699], v[699] = k[3], v[3]
    assert torch.equal(p.k, k) and torch.equal(p.v, v)  # the bad pairs are skipped
    rpx.cache_copy_pages(p.k, p.v, p.ints([]), p.ints([]))


def test_copying_far_pages(cuda_device):
    """Pools of 5 GB each: byte offsets beyond 2^32."""
    nb = 150000
    k = torch.zeros((nb, 8, PAGE, 128), dtype=torch.bfloat16, device=cuda_device)
    v = torch.zeros_like(k)
    k[nb - 1], v[nb - 1] = 1.5, -2.5
    rpx.cache_copy_pages(k, v, torch.tensor([nb - 1], dtype=torch.int32, device=cuda_device),
                         torch.tensor([nb - 3], dtype=torch.int32, device=cuda_device))
    assert bool((k[nb - 3] == 1.5).all()) and bool((v[nb - 3] == -2.5).all()) and not bool(k[nb - 2].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hkv,d", [(2, 64), (5, 128), (8, 128)])
@pytest.mark.parametrize("listed", [False, True])
def test_append(cuda_device, dtype, hkv, d, listed):
    gen = torch.Generator().manual_seed(1)
    counts, lens = [3, 0, 1, 20, 7], [0, 5, 31, 14, 48]
    p = Pool(cuda_device, 60, 5, 5, hkv=hkv, d=d)
    p.fork([(-1, r) for r in range(5)], 70)
    total = sum(counts) + 6
    kv = torch.randn(total, 2 * hkv * d + 16, generator=gen).to(dtype).to(cuda_device)  # strided views of one tensor
    k, v = kv[:, :hkv * d].unflatten(1, (hkv, d)), kv[:, hkv * d:2 * hkv * d].unflatten(1, (hkv, d))
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    ids = torch.randint(0, total, (sum(counts),), generator=gen, dtype=torch.int32) if listed else torch.arange(sum(counts))
    want_k, want_v = p.k.clone(), p.v.clone()
    for s, (n, at) in enumerate(zip(counts, lens)):
        for i in range(n):
            page, slot = p.model.rows[s][(at + i) // PAGE], (at + i) % PAGE
            token = int(ids[cu[s] + i])
            want_k[page, :, slot], want_v[page, :, slot] = k[token].bfloat16(), v[token].bfloat16()
    rpx.cache_append(k, v, p.ints(cu), p.ints(lens), 20, (p.k, p.v, p.table),
                     token_ids=ids.to(cuda_device) if listed else None, device_status=p.status)
    p.expect(0)
    assert torch.equal(p.k, want_k) and torch.equal(p.v, want_v)


def test_append_reports_what_does_not_fit(cuda_device):
    p = Pool(cuda_device, 30, 3, 4)
    p.fork([(-1, 0), (-1, 1)], 64)
    k = torch.randn(10, 2, 64, device=cuda_device).bfloat16()
    before = p.k.clone()
    cases = [
        (dict(lens=[60, 0, 0], cu=[0, 5, 5, 5]), {}),          # beyond the table
        (dict(lens=[0, 0, 0], cu=[0, 0, 0, 4]), {}),           # a row without pages
        (dict(lens=[-1, 0, 0], cu=[0, 1, 1, 1]), {}),
        (dict(lens=[0, 0, 0], cu=[0, 4, 2, 2]), {}),           # runs backwards (the first sequence is fine)
        (dict(lens=[0, 0, 0], cu=[0, 11, 11, 11]), {}),        # beyond the tokens
        (dict(lens=[0, 0, 0], cu=[0, 9, 9, 9], most=8), {}),   # beyond the caller's bound
        (dict(lens=[0, 0, 0], cu=[0, 1, 1, 1]), dict(token_ids=p.ints([10]))),
    ]
    for c, kw in cases:
        rpx.cache_append(k, k, p.ints(c["cu"]), p.ints(c["lens"]), c.get("most", 10), (p.k, p.v, p.table),
                         device_status=p.status, **kw)
        p.expect(-8)
    p.k[p.model.rows[0][0], :, :4] = before[p.model.rows[0][0], :, :4]
    assert torch.equal(p.k, before)


def test_random_life_of_a_pool(cuda_device):
    """Two hundred steps of branching, growing, appending, dropping and compacting, in step with the model; every row's
    tokens stay what was appended to it."""
    rng = np.random.default_rng(7)
    rows, cols, nb = 24, 9, 110
    p = Pool(cuda_device, nb, rows, cols, hkv=2, d=64)
    held = {}  # row -> its K as a tensor
    for step in range(200):
        empty = [r for r in range(rows) if not p.model.rows[r]]
        full = [r for r in range(rows) if p.model.rows[r]]
        what = rng.choice(["new", "fork", "append", "free", "compact"], p=[0.15, 0.3, 0.3, 0.15, 0.1])
        if what == "new" and empty:
            r = int(rng.choice(empty))
            p.model.lens[r] = 0
            _, short = p.fork([(-1, r)], 1 + int(rng.integers(0, 40)), expect=0 if sum(c == 0 for c in p.model.refs) >= 3 else -10)
            if p.model.rows[r]:
                held[r] = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=cuda_device)
        elif what == "fork" and full and empty:
            n = int(rng.integers(1, min(4, len(empty)) + 1))
            src = [int(x) for x in rng.choice(full, n)]
            dst = [int(x) for x in rng.permutation(empty)[:n]]
            need = [-(-(p.model.lens[s] + 5) // PAGE) - p.model.lens[s] // PAGE for s in src]
            if sum(need) > sum(c == 0 for c in p.model.refs) or any(p.model.lens[s] + 5 > cols * PAGE for s in src):
                continue
            p.fork(list(zip(src, dst)), 5)
            for s, d in zip(src, dst):
                if p.model.rows[d]:
                    held[d] = held[s].clone()
        elif what == "append" and full:
            r = int(rng.choice(full))
            n = int(rng.integers(1, 24))
            need = -(-(p.model.lens[r] + n) // PAGE) - len(p.model.rows[r])
            if need > sum(c == 0 for c in p.model.refs) or p.model.lens[r] + n > cols * PAGE:
                continue
            p.fork([(r, r)], n)
            x = torch.randn(n, 2, 64, device=cuda_device).bfloat16()
            cu = [0] * (r + 1) + [n] * (rows - r)
            rpx.cache_append(x, x, p.ints(cu), p.lens, n, (p.k, p.v, p.table), device_status=p.status)
            p.set_len(r, p.model.lens[r] + n)
            held[r] = torch.cat([held[r], x])
        elif what == "free" and full:
            r = int(rng.choice(full))
            p.free([r])
            held.pop(r)
        elif what == "compact":
            src, dst, _ = rpx.pages_compact(p.table, p.refs, device_status=p.status)
            rpx.cache_copy_pages(p.k, p.v, src, dst, device_status=p.status)
            p.model.compact()
        p.expect(0)
        p.check()
        for r, x in held.items():
            assert torch.equal(p.tokens(r), x), (step, what, r)


def test_large_fork(cuda_device):
    """More requests than the planning block has threads, free pages scattered over a large pool."""
    rng = np.random.default_rng(1)
    n, nb = 2500, 90001
    p = Pool(cuda_device, nb, n + 3, 5, hkv=1)
    busy = rng.random(nb) < 0.9
    p.model.refs = [int(b) for b in busy]
    p.model.rows[0] = [int(x) for x in np.flatnonzero(busy)[:3]]
    p.table.copy_(torch.from_numpy(p.model.table()))
    p.refs.copy_(torch.tensor(p.model.refs, dtype=torch.int32))
    p.set_len(0, 40)
    p.fork([(0, i + 1) for i in range(n)], 30)
    p.check()


def test_graph_replay(cuda_device):
    p = Pool(cuda_device, 64, 4, 8)
    p.fork([(-1, 0)], 40)
    p.set_len(0, 40)
    src, dst, rows = p.ints([0, 0]), p.ints([1, 2]), p.ints([1, 2])
    ws = torch.empty(4096, dtype=torch.uint8, device=cuda_device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rpx.pages_free(p.table, p.lens, p.refs, rows, device_status=p.status)
        pairs = rpx.pages_fork(p.table, p.lens, p.refs, src, dst, 10, workspace=ws, device_status=p.status)
        rpx.cache_copy_pages(p.k, p.v, *pairs, device_status=p.status)
    for length in (40, 33, 20):
        p.set_len(0, length)
        graph.replay()
        p.model.free([1, 2])
        want, _, _ = p.model.fork([(0, 1), (0, 2)], 10)
        assert list(zip(*(x.tolist() for x in pairs))) == want
        p.expect(0)
        p.check()
        assert torch.equal(p.tokens(1), p.tokens(0)) and torch.equal(p.tokens(2), p.tokens(0))


def test_a_rollout_with_drafted_trees(cuda_device):
    """The operators together, as a rollout uses them: norm + rotation and the prefix pass fill the cache; two branches are
    forked; each step verifies a drafted tree over each branch, appends the accepted path; one branch is dropped, the pool
    compacted; at the end one-pass attention over each branch's whole sequence gives what the last tree pass gave."""
    dev, hq, hkv, d, prompt = cuda_device, 8, 2, 128, 45
    gen = torch.Generator().manual_seed(0)
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).bfloat16().to(dev) for _ in range(2)]
    inv = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().to(dev)
    axis = rpx.mrope_pair_axis([16, 24, 24])
    p = Pool(dev, 40, 4, 12, hkv=hkv, d=d)
    cache = (p.k, p.v, p.table)

    def project(positions):
        n = positions.shape[0]
        x = torch.randn(n, hq + 2 * hkv, d, generator=gen).bfloat16().to(dev)
        pos = torch.stack([positions, positions // 3, positions % 5]).to(torch.int32).to(dev)
        q, k = rpx.qk_norm_rope(x[:, :hq], x[:, hq:hq + hkv], pos, inv, w[0], w[1], axis)
        return q, k, x[:, hq + hkv:].contiguous()

    p.fork([(-1, 0)], prompt)
    q, k, v = project(torch.arange(prompt))
    rpx.prefix_attn(q, k, v, p.ints([0, prompt]), prompt, cache=(p.k, p.v, p.table[:1]), device_status=p.status)
    p.set_len(0, prompt)
    p.fork([(0, 1), (0, 3)], 40)
    seqs = {r: [(k, v)] for r in (1, 3)}
    parents = [-1, 0, 0, 1, -2, 3]  # 0 - 1 - 3 - 5 and 2 behind 0; node 4 is padding
    path = [0, 1, 3]
    last = {}
    for step in range(5):
        rows = [1, 3] if step < 3 else [3]
        counts = [6 if r in rows else 0 for r in range(4)]
        cu = np.concatenate([[0], np.cumsum(counts)])
        depth = torch.tensor([0, 1, 1, 2, 0, 3])
        q, k, v = project(torch.cat([p.model.lens[r] + depth for r in rows]))
        out, lse = rpx.tree_attn(q, k, v, p.ints(cu), p.ints(parents * len(rows)), p.lens, 6, 12 * PAGE, cache, return_lse=True,
                                 device_status=p.status)
        ids = [int(cu[r]) + j for r in rows for j in path]
        cu_acc = np.concatenate([[0], np.cumsum([3 if r in rows else 0 for r in range(4)])])
        rpx.cache_append(k, v, p.ints(cu_acc), p.lens, 3, cache, token_ids=p.ints(ids), device_status=p.status)
        for r in rows:
            a = int(cu[r])
            idx = torch.tensor([a + j for j in path], device=dev)
            seqs[r].append((k[idx], v[idx]))
            last[r] = (q[idx], out[idx], lse[idx])
            p.set_len(r, p.model.lens[r] + 3)
        if step == 2:
            p.free([0, 1])
            src, dst, _ = rpx.pages_compact(p.table, p.refs, device_status=p.status)
            rpx.cache_copy_pages(p.k, p.v, src, dst, device_status=p.status)
            p.model.compact()
    p.expect(0)
    p.check()
    for r in (1, 3):
        kk, vv = torch.cat([x for x, _ in seqs[r]]).double(), torch.cat([x for _, x in seqs[r]]).double()
        n = kk.shape[0]
        if r == 3:
            assert torch.equal(p.tokens(3).double(), kk)
        qq, out, lse = last[r]
        seen = torch.arange(n, device=dev) <= torch.arange(n - 3, n, device=dev)[:, None]
        z = torch.einsum("ihd,jhd->hij", qq.double(), kk.repeat_interleave(hq // hkv, 1)) * d ** -0.5
        z = z.masked_fill(~seen, -np.inf)
        ref = torch.einsum("hij,jhd->ihd", torch.softmax(z, -1), vv.repeat_interleave(hq // hkv, 1))
        # bf16 output half step 2^-8 |out| and the weights' error on values below 5
        assert float((out.double() - ref).abs().max()) <= 2.0 ** -8 * float(ref.abs().max()) + 5 * 2.0 ** -11
        assert float((lse.double() - torch.logsumexp(z, -1).t()).abs().max()) <= 5e-4


def test_append_of_an_empty_list_stores_nothing(cuda_device):
    """An empty list of accepted tokens is a list: nothing is stored, and offsets that reach into it are reported."""
    p = Pool(cuda_device, 30, 2, 4)
    p.fork([(-1, 0), (-1, 1)], 40)
    k = torch.randn(10, 2, 64, device=cuda_device).bfloat16()
    before = p.k.clone(), p.v.clone()
    rpx.cache_append(k, k, p.ints([0, 0, 0]), p.ints([3, 5]), 4, (p.k, p.v, p.table), token_ids=p.ints([]), device_status=p.status)
    p.expect(0)
    rpx.cache_append(k, k, p.ints([0, 2, 2]), p.ints([3, 5]), 4, (p.k, p.v, p.table), token_ids=p.ints([]), device_status=p.status)
    p.expect(-8)
    assert torch.equal(p.k, before[0]) and torch.equal(p.v, before[1])


def test_pair_lists_in_longer_buffers(cuda_device):
    """Buffers made for the most a program ever asks for: what comes back holds this call's pairs and none of an earlier one."""
    p = Pool(cuda_device, 41, 6, 8)
    room = [torch.full((50,), 3, dtype=torch.int32, device=cuda_device) for _ in range(2)]
    p.fork([(-1, 0)], 60)
    p.set_len(0, 37)
    pairs = rpx.pages_fork(p.table, p.lens, p.refs, p.ints([0, 0]), p.ints([2, 3]), 5, copy_src=room[0], copy_dst=room[1],
                           device_status=p.status)
    want, _, _ = p.model.fork([(0, 2), (0, 3)], 5)
    assert list(zip(*(x.tolist() for x in pairs))) == want
    assert [x.data_ptr() for x in pairs] == [x.data_ptr() for x in room]
    p.free([0])
    before = p.k.clone()
    src, dst, n_live = rpx.pages_compact(p.table, p.refs, copy_src=room[0], copy_dst=room[1], n_live=p.ints([9, 9]),
                                         device_status=p.status)
    moves, n = p.model.compact()
    assert n_live.tolist() == [n] and list(zip(src.tolist(), dst.tolist())) == moves + [(-1, -1)] * (20 - len(moves))
    rpx.cache_copy_pages(p.k, p.v, src, dst, device_status=p.status)
    p.expect(0)
    p.check()
    for a, b in moves:
        before[b] = before[a]
    assert torch.equal(p.k, before)
