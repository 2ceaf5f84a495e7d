"""GPU parity of tree attention over the paged cache against the definition in 64 bits.

Tolerances (half steps: bf16 2^-8, float32 2^-24, relative).  bf16: the output's own rounding 2^-8 |out|; the probabilities'
rounding in front of the P V product, 2^-8 sum(p |v|) - 2^-15 where the pass keeps them in two bf16 terms (up to 256 keys
and 128 nodes); and 2^-11 sum(p |v|) for the weights themselves: the polynomial exp2 is off by 1e-4, a score by 128 products'
fp32 accumulation, 128 * 2^-24 * sum|q k| * scale < 1e-4 for N(0, 1) values.  float32 calls: L fp32 additions in a row,
L * 2^-23 sum(p |v|), and the same score error.  lse: 5e-4 on the same grounds."""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
PAGE = 16
NAN = float("nan")


def draw_parents(rng, n, kind, unused):
    out = []
    for i in range(n):
        if unused and rng.random() < unused:
            out.append(-2)
            continue
        if kind == "chain":
            p = i - 1
            while p >= 0 and out[p] == -2:
                p -= 1
        elif kind == "star":
            p = -1
        else:
            p = int(rng.integers(max(-1, i - 9), i)) if i else -1
            if p >= 0 and out[p] == -2:
                p = -1
        out.append(p)
    return out


class Case:
    def __init__(self, dev, lens, nodes, hq, hkv, d, dtype=torch.bfloat16, kind="random", unused=0.0, seed=0, pad=0, extra=0,
                 scale=1.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.nodes, self.hq, self.hkv, self.d, self.dtype = lens, nodes, hq, hkv, d, dtype
        pages = [-(-p // PAGE) for p in lens]
        nb = sum(pages) + 4
        perm = rng.permutation(nb)
        table = np.full((len(lens), max(1, max(pages)) + extra), -1, np.int32)
        k = torch.full((nb, hkv, PAGE, d), NAN)
        v = torch.full((nb, hkv, PAGE, d), NAN)  # what no sequence owns must not be read into a result
        at = 0
        for s, n in enumerate(pages):
            table[s, :n] = perm[at:at + n]
            for i in range(n):
                held = min(PAGE, lens[s] - i * PAGE)
                k[perm[at + i], :, :held] = torch.randn(hkv, held, d, generator=gen)
                v[perm[at + i], :, :held] = torch.randn(hkv, held, d, generator=gen)
            at += n
        total = sum(nodes) + pad
        rows = hq + 2 * hkv
        qkv = torch.randn(total, rows * d + 8 * extra, generator=gen)
        self.parents = sum((draw_parents(rng, n, kind, unused) for n in nodes), []) + [-2] * pad
        off = torch.tensor(self.parents) < -1
        qkv[off] = NAN  # padding nodes hold anything
        qkv[:, :hq * d] *= scale
        qkv = qkv.to(dtype).to(dev)
        self.q = qkv[:, :hq * d].unflatten(1, (hq, d))
        self.k = qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        self.v = qkv[:, (hq + hkv) * d:rows * d].unflatten(1, (hkv, d))
        self.cache = (k.bfloat16().to(dev), v.bfloat16().to(dev), torch.from_numpy(table).to(dev))
        cu = np.zeros(len(nodes) + 1, np.int32)
        np.cumsum(nodes, out=cu[1:])
        self.cu = torch.from_numpy(cu).to(dev)
        self.parents_dev = torch.tensor(self.parents, dtype=torch.int32, device=dev)
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def run(self, **kw):
        args = dict(max_tree_len=max(self.nodes), max_cached_len=max(self.lens), cache=self.cache, return_lse=True,
                    device_status=self.status)
        args.update(kw)
        return rpx.tree_attn(self.q, self.k, self.v, self.cu, self.parents_dev, self.lens_dev, **args)

    def reference(self, s, scale=None):
        """out, lse, sum(p |v|) of one sequence's nodes in 64 bits on the CPU."""
        dev = self.q.device
        a, b = sum(self.nodes[:s]), sum(self.nodes[:s + 1])
        n, p, g = b - a, self.lens[s], self.hq // self.hkv
        pages = self.cache[2][s, :-(-p // PAGE)].long()

        def keys(cache, own):
            old = cache[pages].permute(0, 2, 1, 3).reshape(-1, self.hkv, self.d)[:p].double()
            return torch.cat([old, own[a:b].double()]).repeat_interleave(g, 1)

        kk, vv = keys(self.cache[0], self.k), keys(self.cache[1], self.v)
        seen = torch.zeros(n, p + n, dtype=torch.bool)
        for i in range(n):
            up = self.parents[a + i]
            if up < -1:
                continue
            seen[i, p:] = seen[up, p:] if up >= 0 else False
            seen[i, :p] = True
            seen[i, p + i] = True
        seen = seen.to(dev)
        z = torch.einsum("ihd,jhd->hij", self.q[a:b].double(), kk) * (scale or self.d ** -0.5)
        z = z.masked_fill(~seen, -np.inf)
        lse = torch.logsumexp(z, -1)
        w = torch.where(seen, torch.exp(z - lse[..., None]), 0.0)
        vv = torch.nan_to_num(vv)
        vv = torch.where(seen.any(0)[:, None, None], vv, 0.0)
        return torch.einsum("hij,jhd->ihd", w, vv), lse.t(), torch.einsum("hij,jhd->ihd", w, vv.abs())

    def check(self, out, lse, scale=None):
        for s, n in enumerate(self.nodes):
            if n == 0:
                continue
            a = sum(self.nodes[:s])
            ref, ref_lse, size = self.reference(s, scale)
            if self.dtype == torch.float32:
                tol = 2.0 ** -24 * ref.abs() + ((self.lens[s] + n) * 2.0 ** -23 + 2.0 ** -11) * size
            else:
                few = self.lens[s] + n <= 128 and max(self.nodes) <= 128
                tol = 2.0 ** -8 * ref.abs() + ((2.0 ** -15 if few else 2.0 ** -8) + 2.0 ** -11) * size
            err = (out[a:a + n].double() - ref).abs()
            assert bool((err <= tol).all()), f"sequence {s}: {float((err - tol).max()):.3e} over, {int((~(err <= tol)).sum())} values"
            used = torch.isfinite(ref_lse)
            assert torch.equal(torch.isneginf(lse[a:a + n]), ~used)
            if bool(used.any()):
                assert float((lse[a:a + n].double() - ref_lse)[used].abs().max()) <= 5e-4
        assert int(self.status.item()) == 0


CASES = [
    # lens, nodes, hq, hkv, d
    ([5], [1], 4, 2, 128),
    ([0], [1], 4, 2, 64),
    ([0, 1, 15, 16, 17], [1, 1, 1, 1, 1], 28, 4, 128),
    ([63, 64, 65, 128, 129], [3, 1, 5, 2, 4], 7, 1, 64),
    ([1000], [1], 40, 8, 128),
    ([4096, 0, 333], [8, 0, 8], 28, 4, 128),
    ([20000], [4], 28, 4, 128),
    ([700, 31, 5000, 64], [16, 1, 33, 9], 40, 8, 128),
    ([513, 2000], [64, 17], 16, 1, 64),
    ([100, 1500], [65, 128], 4, 4, 128),
    ([300, 40], [128, 100], 8, 8, 64),
    ([2500, 0, 77], [129, 200, 3], 28, 4, 128),
    ([640], [300], 4, 4, 64),
    ([1024, 100], [256, 31], 16, 1, 128),
    ([50], [1024], 6, 2, 64),
    ([900, 4000], [150, 140], 5, 5, 128),
    ([300, 60], [3, 2], 160, 1, 64),
    ([128, 256, 384, 5000], [18, 18, 17, 9], 28, 4, 128),
    ([9000], [30], 40, 8, 128),
    ([140, 0, 12000, 260], [25, 26, 60, 51], 40, 8, 128),
    ([2000] * 20, [40] * 20, 8, 2, 64),
]


@pytest.mark.parametrize("kind", ["random", "chain", "star"])
@pytest.mark.parametrize("lens,nodes,hq,hkv,d", CASES)
def test_trees(cuda_device, lens, nodes, hq, hkv, d, kind):
    c = Case(cuda_device, lens, nodes, hq, hkv, d, kind=kind, unused=0.1, seed=len(lens) + nodes[0], extra=3)
    c.check(*c.run())


@pytest.mark.parametrize("lens,nodes,hq,hkv,d", [CASES[i] for i in (2, 3, 7, 9, 11)])
def test_float32(cuda_device, lens, nodes, hq, hkv, d):
    c = Case(cuda_device, lens, nodes, hq, hkv, d, dtype=torch.float32, unused=0.2, seed=5)
    c.check(*c.run())


def test_many_sequences(cuda_device):
    """More sequences than a CTA has threads: the cut of the line of tiles runs over several rounds."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 90, 400).tolist()
    nodes = rng.integers(0, 4, 400).tolist()
    c = Case(cuda_device, lens, nodes, 4, 2, 64, unused=0.1)
    c.check(*c.run())


def test_all_unused_and_one_used(cuda_device):
    for nodes in ([6], [140]):
        c = Case(cuda_device, [700], nodes, 28, 4, 128, kind="star")
        c.parents = [-2] * (nodes[0] - 1) + [-1]
        c.parents_dev.copy_(torch.tensor(c.parents, dtype=torch.int32))
        c.q[:-1], c.k[:-1], c.v[:-1] = NAN, NAN, NAN
        c.check(*c.run())
        c.parents[-1] = -7
        c.parents_dev.copy_(torch.tensor(c.parents, dtype=torch.int32))
        out, lse = c.run()
        assert torch.equal(out, torch.zeros_like(out)) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("nodes", [[7, 0, 5], [150, 0, 20]])
def test_rows_behind_the_last_sequence_stay(cuda_device, nodes):
    c = Case(cuda_device, [300, 10, 20], nodes, 28, 4, 128, pad=9)
    out = torch.full(tuple(c.q.shape), 7.0, dtype=torch.bfloat16, device=cuda_device)
    lse = torch.full(tuple(c.q.shape[:2]), 7.0, device=cuda_device)
    c.run(out=out, lse=lse)
    c.check(out, lse)
    assert bool((out[-9:] == 7.0).all()) and bool((lse[-9:] == 7.0).all())


@pytest.mark.parametrize("nodes", [[9, 5], [140, 30], [33, 129]])
def test_a_sequence_does_not_meet_its_neighbours_values(cuda_device, nodes):
    """Non-finite values in one sequence's nodes and cache leave every other sequence as it was."""
    c = Case(cuda_device, [200, 77], nodes, 28, 4, 128)
    want, want_lse = c.run()
    a = nodes[0]
    for own, other in ((slice(a, None), slice(0, a)), (slice(0, a), slice(a, None))):
        k, v = c.k.clone(), c.v.clone()
        c.k[own], c.v[own] = NAN, float("inf")
        out, lse = c.run()
        assert torch.equal(out[other], want[other]) and torch.equal(lse[other], want_lse[other])
        assert not bool(torch.isfinite(out[own]).any())
        c.k.copy_(k), c.v.copy_(v)


@pytest.mark.parametrize("nodes", [[20], [160]])
def test_peaked_scores_and_scale(cuda_device, nodes):
    """Scores up to hundreds: the running maximum moves by more than its threshold many times."""
    c = Case(cuda_device, [1500], nodes, 8, 2, 64, scale=2.0)
    c.cache[0].mul_(torch.linspace(0.1, 2.0, c.cache[0].shape[0], device=cuda_device).view(-1, 1, 1, 1).bfloat16())
    c.check(*c.run(softmax_scale=0.5), scale=0.5)


@pytest.mark.parametrize("nodes", [[12, 12], [130, 12]])
def test_bad_data_is_reported_and_contained(cuda_device, nodes):
    c = Case(cuda_device, [400, 90], nodes, 28, 4, 128, kind="chain")
    want, want_lse = c.run()
    a = nodes[0]
    # a parent that is not an earlier node: it and what hangs on it count as not in use, the rest is as before
    c.parents_dev[5] = 6
    out, lse = c.run()
    assert int(c.status.item()) == -8
    assert torch.equal(out[:5], want[:5]) and torch.equal(out[a:], want[a:])
    assert bool((out[5:a] == 0).all()) and bool(torch.isneginf(lse[5:a]).all())
    c.parents_dev[5] = 4
    # hanging on a padding node
    c.status.zero_()
    c.parents_dev[3] = -2
    out, _ = c.run()
    assert int(c.status.item()) == -8
    assert torch.equal(out[:3], want[:3]) and bool((out[3:a] == 0).all())
    c.parents_dev[3] = 2
    # a block id outside the pool
    c.status.zero_()
    c.cache[2][1, 0] = 10 ** 6
    out, _ = c.run()
    assert int(c.status.item()) == -8 and torch.equal(out[:a], want[:a])
    c.cache[2][1, 0] = 0


@pytest.mark.parametrize("nodes", [[12, 12], [130, 12]])
def test_offsets_that_do_not_fit_skip_the_sequence(cuda_device, nodes):
    c = Case(cuda_device, [400, 90], nodes, 28, 4, 128)
    want, _ = c.run()
    a = nodes[0]
    for change in ("pages", "negative", "bound"):
        c.status.zero_()
        lens, kw = c.lens_dev.clone(), {}
        if change == "pages":
            c.lens_dev[1] = 10 ** 6
        elif change == "negative":
            c.lens_dev[1] = -5
        out = torch.full_like(want, 3.0)
        if change == "bound":
            kw["max_tree_len"] = nodes[0] - 1
            c.run(out=out, **kw)
            assert bool((out[:a] == 3.0).all())
        else:
            c.run(out=out)
            assert torch.equal(out[:a], want[:a]) and bool((out[a:] == 3.0).all())
        assert int(c.status.item()) == -8
        c.lens_dev.copy_(lens)


@pytest.mark.parametrize("nodes", [[3, 9], [140, 9]])
def test_repeats_streams_graph_and_workspace(cuda_device, nodes):
    c = Case(cuda_device, [6000, 410], nodes, 28, 4, 128)
    want, want_lse = c.run()
    again = c.run()
    assert torch.equal(again[0], want) and torch.equal(again[1], want_lse)
    need = rpx.tree_attn_workspace_bytes(28, 4, 128, 0, sum(nodes), 2, max(nodes))
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=cuda_device)  # whatever it held before
    got = c.run(workspace=ws[:need])
    assert torch.equal(got[0], want) and torch.equal(got[1], want_lse)
    assert bool((ws[need:] == 255).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = c.run(workspace=ws[:need])
    out.zero_()
    c.lens_dev[0] = 5000  # a captured call reads the lengths when it is replayed
    graph.replay()
    c.lens[0] = 5000
    c.check(out, lse)


def test_single_nodes_equal_the_suffix_pass(cuda_device):
    """A tree of one node per sequence is a one-token suffix; both round the same inputs once."""
    c = Case(cuda_device, [777, 1, 2048], [1, 1, 1], 28, 4, 128)
    out, lse = c.run()
    ref, ref_lse = rpx.suffix_attn(c.q, c.k, c.v, c.cu, c.lens_dev, 1, 2048, c.cache, return_lse=True)
    assert float((out.float() - ref.float()).abs().max()) <= 1e-2
    assert float((lse - ref_lse).abs().max()) <= 1e-3


def test_far_pages_pass_32_bits(cuda_device):
    """Pages whose byte and element offsets pass 2^32 (a pool of 5 GB per tensor, read at its far end)."""
    hkv, d, nb = 8, 128, 150000
    c = Case(cuda_device, [100], [3], 16, hkv, d)
    k = torch.empty((nb, hkv, PAGE, d), dtype=torch.bfloat16, device=cuda_device)
    v = torch.empty_like(k)
    table = c.cache[2].clone()
    for i in range(7):
        old = int(table[0, i])
        k[nb - 1 - i], v[nb - 1 - i] = c.cache[0][old], c.cache[1][old]
        table[0, i] = nb - 1 - i
    want = c.run()
    c.cache = (k, v, table)
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# streaming, one query tile, two query tiles; float32 - each with sequences that are not cut and with cut ones
@pytest.mark.parametrize("lens", [[300, 40], [2900, 700]])
@pytest.mark.parametrize("nodes,dtype", [([3, 2], torch.bfloat16), ([40, 9], torch.bfloat16), ([150, 20], torch.bfloat16),
                                         ([5, 2], torch.float32)])
def test_a_score_that_is_no_number_reaches_its_rows(cuda_device, lens, nodes, dtype):
    """NaN, and +inf (inf - inf in the softmax), make a row NaN as the definition does; -inf only takes its key out."""
    c = Case(cuda_device, lens, nodes, 4, 2, 64, dtype=dtype, seed=3)
    clean, clean_lse = c.run()
    k_cache, table = c.cache[0], c.cache[2]

    def place(s, key):
        return int(table[s, key // PAGE]), key % PAGE

    spots = [[(0, j)] for j in (*range(9), 130, lens[0] - 1)] + [[(1, 3)]] + [[(0, j) for j in range(n)] for n in (lens[0], lens[0] * 2 // 3)]
    for spot in spots:
        saved = k_cache.clone()
        for s, key in spot:
            page, at = place(s, key)
            k_cache[page, 0, at] = NAN
        out, lse = c.run()
        k_cache.copy_(saved)
        seq = torch.zeros(len(c.parents), dtype=torch.bool, device=cuda_device)
        lo = sum(nodes[:spot[0][0]])
        seq[lo:lo + nodes[spot[0][0]]] = True
        assert out[seq][:, :2].isnan().all() and lse[seq][:, :2].isnan().all(), spot
        assert torch.equal(out[:, 2:], clean[:, 2:]) and torch.equal(lse[:, 2:], clean_lse[:, 2:])
        assert torch.equal(out[~seq], clean[~seq]) and torch.equal(lse[~seq], clean_lse[~seq])
    for key in range(8):
        saved = k_cache.clone()
        page, at = place(0, key)
        k_cache[page, 0, at, 0] = float("inf")
        out, lse = c.run()
        k_cache.copy_(saved)
        up = c.q[:nodes[0], :2, 0] > 0
        assert torch.equal(out[:nodes[0], :2].isnan().all(-1), up) and torch.equal(out[:nodes[0], :2].isnan().any(-1), up), key
        assert torch.equal(lse[:nodes[0], :2].isnan(), up)
    assert c.status.item() == 0


def test_tensors_that_do_not_fit_are_refused(cuda_device):
    c = Case(cuda_device, [20, 40], [3, 2], 4, 2, 64)
    k_cache, v_cache, table = c.cache
    for cache in ((k_cache[:, :1].contiguous(), v_cache[:, :1].contiguous(), table), (k_cache, v_cache[:-1], table),
                  (k_cache, v_cache, table[:1])):
        with pytest.raises(ValueError):
            c.run(cache=cache)
    with pytest.raises(ValueError):
        c.run(out=torch.empty(5, 4, 64, device=cuda_device))
    with pytest.raises(ValueError):
        c.run(out=torch.empty(5, 8, 64, dtype=torch.bfloat16, device=cuda_device)[:, ::2])
    with pytest.raises(ValueError):
        c.run(lse=torch.empty(4, 5, device=cuda_device).t())
    for k, v in ((c.k, c.v[:, :1]), (c.k.float(), c.v), (c.k[:-1], c.v[:-1])):
        with pytest.raises(ValueError):
            rpx.tree_attn(c.q, k, v, c.cu, c.parents_dev, c.lens_dev, 3, 40, c.cache)


# streaming, one query tile, two query tiles; float32
FORMS = [([3, 2], torch.bfloat16), ([40, 9], torch.bfloat16), ([150, 20], torch.bfloat16), ([5, 2], torch.float32)]


@pytest.mark.parametrize("lens", [[300, 40], [2900, 700]])
@pytest.mark.parametrize("nodes,dtype", FORMS)
def test_masked_values_weigh_nothing(cuda_device, lens, nodes, dtype):
    """A node's V, however large, leaves every row alone that it is no ancestor of: the same bits as with V of 0."""
    c = Case(cuda_device, lens, nodes, 4, 2, 64, dtype=dtype, kind="star", seed=4)
    for j in range(min(18, nodes[0])):  # wherever the key lies within 16
        saved, got = c.v[j].clone(), []
        for value in (1e38, 0.0):
            c.v[j] = value
            got.append(c.run())
        c.v[j] = saved
        others = torch.arange(len(c.parents), device=cuda_device) != j
        assert torch.equal(got[0][0][others], got[1][0][others]) and torch.equal(got[0][1][others], got[1][1][others]), j
    assert c.status.item() == 0


@pytest.mark.parametrize("nodes,dtype", FORMS)
def test_far_smaller_scores_weigh_nothing(cuda_device, nodes, dtype):
    """Keys whose weight is 2^-300 and less add nothing, not even to values of 1e38 (2^126)."""
    c = Case(cuda_device, [300, 40], nodes, 4, 2, 64, dtype=dtype, seed=6)
    k, v, table = c.cache
    c.q.fill_(4.0), c.k.fill_(4.0)
    # scores of 64 * 4 * 8 / 8 = 256 against 0 at a third of the keys: e^-256 < 2^-300
    low = [key for key in range(300) if key % 3 == 0]
    for key in range(300):
        k[int(table[0, key // PAGE]), :, key % PAGE] = 0.0 if key % 3 == 0 else 8.0
    got = []
    for value in (1e38, 0.0):
        for key in low:
            v[int(table[0, key // PAGE]), :, key % PAGE] = value
        got.append(c.run())
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert c.status.item() == 0
