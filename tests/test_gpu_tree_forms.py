"""Tree attention: what must hold in every form of the pass, with the form of each size asserted.

The forms: streaming in blocks of 16, 32 and 64 rows, tensor cores with one and with two query tiles, float32.  A size that
another rule of choice would hand to another form fails here instead of leaving its form untested.

Tolerance, on the grounds of the parity tests of this pass: the output's rounding 2^-8 |out|, 2^-11 sum(p |v|) for the weights
themselves, and for the probabilities' rounding 2^-15 sum(p |v|) where they are two bf16 terms - streaming blocks of up to 32
rows at every length - and 2^-8 sum(p |v|) elsewhere; float32: L 2^-23 sum(p |v|) for L additions in a row.  lse 5e-4."""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx
from test_gpu_tree_attn import NAN, PAGE, Case

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# form: (nodes of the two sequences, query heads, KV heads, head_dim, element type)
SIZES = {
    "stream16": ([6, 5], 4, 2, 128, BF16),
    "stream32": ([12, 9], 4, 2, 128, BF16),
    "stream64": ([7, 3], 160, 1, 64, BF16),
    "tile1": ([40, 9], 4, 2, 128, BF16),
    "tile2": ([150, 20], 4, 2, 64, BF16),
    "float32": ([9, 5], 4, 2, 64, F32),
}
LENS = {"whole": [150, 90], "cut": [5000, 700]}


def form_of(nodes, hq, hkv, d, dtype):
    if dtype == F32:
        return "float32"
    most, group = max(nodes), hq // hkv

    def size(tokens):
        return rpx.tree_attn_workspace_bytes(hq, hkv, d, 0, tokens, 1, most)

    if size(2000) == size(1000):  # only the streaming form keeps nothing per token
        return f"stream{16 if most * group <= 16 else 32 if most * group <= 32 else 64}"
    return "tile1" if size(1) < 1.5 * 148 * 256 * (8 + 4 * d) else "tile2"  # rows of a piece: 128 or 256


@pytest.fixture(params=list(SIZES))
def size(request):
    nodes, hq, hkv, d, dtype = SIZES[request.param]
    assert form_of(nodes, hq, hkv, d, dtype) == request.param
    return nodes, hq, hkv, d, dtype


@pytest.fixture(params=list(LENS))
def lens(request):
    return LENS[request.param]


def make(dev, lens, size, **kw):
    nodes, hq, hkv, d, dtype = size
    return Case(dev, lens, nodes, hq, hkv, d, dtype=dtype, **kw)


def check(c, out, lse, scale=None, only=None):
    two_terms = form_of(c.nodes, c.hq, c.hkv, c.d, c.dtype) in ("stream16", "stream32")
    for s, n in enumerate(c.nodes):
        if n == 0 or (only is not None and s != only):
            continue
        a = sum(c.nodes[:s])
        ref, ref_lse, size = c.reference(s, scale)
        if c.dtype == F32:
            tol = 2.0 ** -24 * ref.abs() + ((c.lens[s] + n) * 2.0 ** -23 + 2.0 ** -11) * size
        else:
            tol = 2.0 ** -8 * ref.abs() + ((2.0 ** -15 if two_terms else 2.0 ** -8) + 2.0 ** -11) * size
        err = (out[a:a + n].double() - ref).abs()
        assert bool((err <= tol).all()), f"sequence {s}: {float((err - tol).max()):.3e} over, {int((~(err <= tol)).sum())} values"
        used = torch.isfinite(ref_lse)
        assert torch.equal(torch.isneginf(lse[a:a + n]), ~used)
        if bool(used.any()):
            assert float((lse[a:a + n].double() - ref_lse)[used].abs().max()) <= 5e-4
    assert only is not None or int(c.status.item()) == 0


@pytest.mark.parametrize("kind", ["random", "chain", "star"])
def test_against_the_definition(cuda_device, size, lens, kind):
    c = make(cuda_device, lens, size, kind=kind, unused=0.15, extra=2, seed=1)
    check(c, *c.run())


def test_all_unused_and_one_used(cuda_device, size, lens):
    c = make(cuda_device, lens, size, kind="star")
    total = len(c.parents)
    c.parents = [-2] * (total - 1) + [-1]
    c.parents_dev.copy_(torch.tensor(c.parents, dtype=torch.int32))
    c.q[:-1], c.k[:-1], c.v[:-1] = NAN, NAN, NAN
    check(c, *c.run())
    c.parents_dev[-1] = -9
    out, lse = c.run()
    assert torch.equal(out, torch.zeros_like(out)) and bool(torch.isneginf(lse).all())


def test_rows_behind_the_last_sequence_stay(cuda_device, size, lens):
    c = make(cuda_device, lens, size, pad=9)
    out = torch.full(tuple(c.q.shape), 7.0, dtype=c.dtype, device=cuda_device)
    lse = torch.full(tuple(c.q.shape[:2]), 7.0, device=cuda_device)
    c.run(out=out, lse=lse)
    check(c, out, lse)
    assert bool((out[-9:] == 7.0).all()) and bool((lse[-9:] == 7.0).all())


def test_a_sequence_does_not_meet_its_neighbours_values(cuda_device, size, lens):
    c = make(cuda_device, lens, size)
    want, want_lse = c.run()
    a = c.nodes[0]
    for own, other in ((slice(a, None), slice(0, a)), (slice(0, a), slice(a, None))):
        k, v = c.k.clone(), c.v.clone()
        c.k[own], c.v[own] = NAN, float("inf")
        out, lse = c.run()
        assert torch.equal(out[other], want[other]) and torch.equal(lse[other], want_lse[other])
        assert not bool(torch.isfinite(out[own]).any())
        c.k.copy_(k), c.v.copy_(v)


def test_peaked_scores_and_scale(cuda_device, size, lens):
    """Scores up to hundreds: the running maximum moves by more than its threshold many times."""
    c = make(cuda_device, lens, size, scale=2.0)
    c.cache[0].mul_(torch.linspace(0.1, 2.0, c.cache[0].shape[0], device=cuda_device).view(-1, 1, 1, 1).bfloat16())
    out, lse = c.run(softmax_scale=0.5)
    # scores have twice the usual size and more: their error, relative to them, grows with them; the smallest exponent that
    # covers it is taken from the largest score.  |error of a score| <= 128 * 2^-24 * sum|q k| * scale
    for s, n in enumerate(c.nodes):
        a = sum(c.nodes[:s])
        ref, ref_lse, size_ = c.reference(s, 0.5)
        pages = c.cache[2][s, :-(-c.lens[s] // PAGE)].long()
        keys = c.cache[0][pages].permute(0, 2, 1, 3).reshape(-1, c.hkv, c.d)[:c.lens[s]].double()
        keys = torch.cat([keys, c.k[a:a + n].double()]).abs().repeat_interleave(c.hq // c.hkv, 1)
        most = torch.einsum("ihd,jhd->hij", c.q[a:a + n].double().abs(), keys).amax() * 0.5
        z_err = float(128 * 2.0 ** -24 * most)
        two_terms = form_of(c.nodes, c.hq, c.hkv, c.d, c.dtype) in ("stream16", "stream32")
        p_err = (c.lens[s] + n) * 2.0 ** -23 if c.dtype == F32 else 2.0 ** -15 if two_terms else 2.0 ** -8
        tol = (2.0 ** -24 if c.dtype == F32 else 2.0 ** -8) * ref.abs() + (p_err + 2.0 ** -11 + 2 * z_err) * size_
        assert bool(((out[a:a + n].double() - ref).abs() <= tol).all())
        assert float((lse[a:a + n].double() - ref_lse).abs().max()) <= 5e-4 + z_err
    assert int(c.status.item()) == 0


def test_bad_data_is_reported_and_contained(cuda_device, size, lens):
    c = make(cuda_device, lens, size, kind="chain")
    want, want_lse = c.run()
    a = c.nodes[0]

    def reported():
        got = int(c.status.item())
        c.status.zero_()
        return got == -8

    c.parents_dev[4] = 5  # not an earlier node: it and what hangs on it count as not in use, the rest is as before
    out, lse = c.run()
    assert reported() and torch.equal(out[:4], want[:4]) and torch.equal(out[a:], want[a:])
    assert bool((out[4:a] == 0).all()) and bool(torch.isneginf(lse[4:a]).all())
    c.parents_dev[4] = 4  # itself
    out, lse = c.run()
    assert reported() and torch.equal(out[:4], want[:4]) and bool((out[4:a] == 0).all())
    c.parents_dev[4] = 3
    c.parents_dev[2] = -2  # node 3 hangs on padding
    out, lse = c.run()
    assert reported() and torch.equal(out[:2], want[:2]) and bool((out[2:a] == 0).all()) and torch.equal(out[a:], want[a:])
    c.parents_dev[2] = 1
    for page, block in ((0, 10 ** 6), (c.lens[1] // PAGE - 1, -1)):  # no block of the pool, in the first tile and in the last
        saved = int(c.cache[2][1, page])
        c.cache[2][1, page] = block
        out, lse = c.run()
        c.cache[2][1, page] = saved
        assert reported() and torch.equal(out[:a], want[:a]) and torch.equal(lse[:a], want_lse[:a])
    out, lse = c.run()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and int(c.status.item()) == 0


def test_offsets_that_do_not_fit_skip_the_sequence(cuda_device, size, lens):
    """The other sequence is held to the definition and not to the bits of the run before: without the skipped one, the line
    of key tiles is shorter and cut in other places, which is another order of the sums."""
    c = make(cuda_device, lens, size)
    a = c.nodes[0]
    cu = c.cu.clone()
    for lens_1, ends in ((10 ** 6, None), (-5, None), (None, [0, a, a + 10 ** 6]), (None, [0, a, a - 2])):
        c.status.zero_()
        if lens_1 is not None:
            c.lens_dev[1] = lens_1
        else:  # beyond the tokens; backwards
            c.cu.copy_(torch.tensor(ends, dtype=torch.int32))
        out = torch.full(tuple(c.q.shape), 3.0, dtype=c.dtype, device=cuda_device)
        lse = torch.full(tuple(c.q.shape[:2]), 3.0, device=cuda_device)
        c.run(out=out, lse=lse)
        check(c, out, lse, only=0)
        assert bool((out[a:] == 3.0).all()) and bool((lse[a:] == 3.0).all()) and int(c.status.item()) == -8
        c.lens_dev[1] = c.lens[1]
        c.cu.copy_(cu)


def test_a_tree_beyond_the_callers_bound_is_skipped(cuda_device, size, lens):
    c = make(cuda_device, lens, size)
    a, bound = c.nodes[0], c.nodes[0] - 1
    out = torch.full(tuple(c.q.shape), 3.0, dtype=c.dtype, device=cuda_device)
    c.run(out=out, max_tree_len=bound)
    assert int(c.status.item()) == -8 and bool((out[:a] == 3.0).all()) and bool(torch.isfinite(out[a:].float()).all())
    assert not bool((out[a:] == 3.0).all(-1).any())


def test_repeats_streams_graph_and_workspace(cuda_device, size, lens):
    c = make(cuda_device, lens, size)
    want, want_lse = c.run()
    for _ in range(3):
        again = c.run()
        assert torch.equal(again[0], want) and torch.equal(again[1], want_lse)
    need = rpx.tree_attn_workspace_bytes(c.hq, c.hkv, c.d, 1 if c.dtype == F32 else 0, sum(c.nodes), 2, max(c.nodes))
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=cuda_device)  # whatever it held before
    got = c.run(workspace=ws[:need])
    assert torch.equal(got[0], want) and torch.equal(got[1], want_lse) and bool((ws[need:] == 255).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, here = c.run(stream=side), c.run()  # two calls at once, each with a workspace of its own
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want) and torch.equal(here[0], want) and torch.equal(got[1], want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first, first_lse = c.run(workspace=ws[:need])
        second, second_lse = c.run(workspace=ws[:need])  # one after the other in the same workspace
    for t in (first, second):
        t.zero_()
    c.lens[0] = c.lens[0] * 4 // 5
    c.lens_dev[0] = c.lens[0]  # a captured call reads the lengths when it is replayed
    for _ in range(2):
        graph.replay()
    check(c, first, first_lse)
    assert torch.equal(first, second) and torch.equal(first_lse, second_lse)


# ------------------------------------------------------------------ many sequences, long contexts, large groups
@pytest.mark.parametrize("form,nodes,hq,hkv,d", [("stream16", 2, 4, 2, 64), ("stream16", 1, 4, 2, 128), ("stream32", 12, 4, 2, 64),
                                                 ("tile1", 40, 4, 2, 64), ("tile2", 150, 28, 4, 128)])
@pytest.mark.parametrize("batch", [33, 64, 97])
def test_many_sequences_are_cut(cuda_device, form, nodes, hq, hkv, d, batch):
    """More sequences than a warp looks at in a step, and too long not to be cut: the line of tiles, the walk along it and
    the join go over several rounds of 32, with long, short and empty sequences on both sides of each."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 60, batch).tolist()
    counts = rng.integers(0, nodes + 1, batch).tolist()
    for s in (0, 30, 31, 32, 33, 63, 64, 65, 95, 96):
        if s < batch:
            lens[s], counts[s] = int(rng.integers(1100, 3000)), nodes
    for s in (5, 34, 62, 70):
        if s < batch:
            lens[s], counts[s] = int(rng.integers(600, 1500)), max(1, nodes // 2)
    for s in (29, 36, 66):
        if s < batch:
            lens[s], counts[s] = 0, 0
    assert form_of(counts, hq, hkv, d, BF16) == form
    c = Case(cuda_device, lens, counts, hq, hkv, d, unused=0.1, seed=batch)
    check(c, *c.run())


def test_a_batch_of_decoding_steps(cuda_device):
    lens = np.random.default_rng(0).integers(0, 3000, 64).tolist()
    c = Case(cuda_device, lens, [1] * 64, 16, 4, 64)
    check(c, *c.run())


@pytest.mark.parametrize("form,nodes,hq,hkv", [("stream16", 8, 16, 8), ("stream32", 16, 16, 8), ("tile1", 48, 16, 8), ("tile2", 100, 16, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_every_tile_of_a_long_context(cuda_device, form, nodes, hq, hkv, d):
    """Each node looks for one key that matches it: its output is that key's value, so a tile that is missing, stale, taken
    twice or read from another page shows.  4 sequences of 8000 tokens are 13 key tiles a piece and more, several times the
    rings' stages; over the runs every tile of 64 keys is looked for by some node, the last key of a sequence too.

    A matching key is 30 sqrt(d) q / |q|^2: its score is 30, other nodes' matches have N(0, 30^2 / d) and the 8000 other keys
    N(0, 1) or so, whose weights add up to some e^10; up to 100 of the former reach 17.  The match has all but e^-12 of the
    weight, and the output is its value to the roundings of the probability and of the output, 2^-8 each."""
    lens, batch = [8000, 7993, 7936, 8001], 4
    assert form_of([nodes], hq, hkv, d, BF16) == form
    c = Case(cuda_device, lens, [nodes] * batch, hq, hkv, d, kind="star", seed=2)
    gen = torch.Generator().manual_seed(3)
    k_cache, v_cache, table = c.cache
    pages = table.cpu().numpy()
    tiles = -(-max(lens) // 64)
    for run in range(-(-tiles // nodes)):
        want = torch.randn(batch * nodes, d, generator=gen).bfloat16().to(cuda_device)
        c.q.copy_(want[:, None].expand(-1, hq, -1))
        block, slot, row = [], [], []
        for s in range(batch):
            for i in range(nodes):
                tile = (run * nodes + i) % tiles
                at = lens[s] - 1 if tile == tiles - 1 else min(lens[s] - 1, tile * 64 + int(torch.randint(0, 64, (1,), generator=gen)))
                if (int(pages[s, at // PAGE]), at % PAGE) in zip(block, slot):
                    continue  # (the runs' last nodes start over)
                block.append(int(pages[s, at // PAGE])), slot.append(at % PAGE), row.append(s * nodes + i)
        b, t, r = (torch.tensor(x, device=cuda_device) for x in (block, slot, row))
        saved = k_cache[b, :, t].clone()
        match = want[r].float()
        match = match * (30 * d ** 0.5 / match.square().sum(-1, keepdim=True))
        k_cache[b, :, t] = match.bfloat16()[:, None].expand(-1, hkv, -1)
        out, lse = c.run()
        check(c, out, lse)
        # and directly: the output is the value of the key that matches
        match = v_cache[b, :, t].float().repeat_interleave(hq // hkv, 1)
        assert float((out[r].float() - match).abs().max()) <= (2.0 ** -7 + 1e-4) * float(match.abs().max())
        k_cache[b, :, t] = saved


@pytest.mark.parametrize("lens,nodes,hq,hkv", [([300, 60], [100, 128], 160, 1), ([2500, 0], [128, 37], 160, 1), ([700, 5], [9, 100], 258, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_groups_above_128_heads(cuda_device, lens, nodes, hq, hkv, d):
    assert form_of(nodes, hq, hkv, d, BF16) == "stream64"
    c = Case(cuda_device, lens, nodes, hq, hkv, d, unused=0.1, seed=8)
    check(c, *c.run())
