"""GPU parity of group attention over shared pages against the definition in 64 bits.

Tolerances, per value, with u = 2^-8 (bf16's half step), e = 2^-24 and S the largest scale * sum |q_i k_i| of a row: a score is a
float32 sum of d products (off by (d + 4) e S), so every weight is off by that, 2^-21 of the exponential and, where it enters the
product with V as one bf16 term, u; two terms leave 2^-16.  Sums of len terms in float32 in pieces of 128: 2^-14 at most.
  out  u |out| + (2 w + 2^-13) sum p |v|,  w = (d + 4) e S + 2^-21 + (2^-16 or u)        lse  (d + 4) e S + 2^-13 ln 2 + 2^-20 |lse|
The float32 form has no u and none of the rounding of P.
"""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
PAGE = 16


def make(groups, hq, hkv, d, dev, seed=0, dtype=torch.bfloat16, scale=1.0, spare=4, fill=None):
    """groups: [(shared tokens, [(own tokens, query tokens), ..]), ..]; own tokens count from the shared ones on."""
    gen = torch.Generator().manual_seed(seed)
    seqs = [(sh, own, n, g) for g, (sh, members) in enumerate(groups) for own, n in members]
    kv = [sh + own for sh, own, _, _ in seqs]
    news = [n for _, _, n, _ in seqs]
    pages = [-(-x // PAGE) for x in kv]
    nb = sum(sh // PAGE for sh, _ in groups) + sum(pg - s[0] // PAGE for pg, s in zip(pages, seqs)) + spare
    perm = torch.randperm(nb, generator=gen).int()
    table = torch.full((len(seqs), max(pages + [1]) + 1), -1, dtype=torch.int32)
    at, prompt, of = 0, None, -1
    for i, (pg, (sh, _, _, g)) in enumerate(zip(pages, seqs)):
        whole = sh // PAGE
        if g != of:
            prompt, of = perm[at:at + whole], g
            at += whole
        table[i, :whole] = prompt
        table[i, whole:pg] = perm[at:at + pg - whole]
        at += pg - whole
    kc, vc = (torch.randn(nb, hkv, PAGE, d, generator=gen).bfloat16() for _ in range(2))
    if fill is not None:  # what lies in slots that no token maps to
        used = torch.zeros(nb, PAGE, dtype=torch.bool)
        for i, x in enumerate(kv):
            pos = torch.arange(x)
            used[table[i, pos // PAGE].long(), pos % PAGE] = True
        kc[~used[:, None].expand(nb, hkv, PAGE)] = fill
        vc[~used[:, None].expand(nb, hkv, PAGE)] = fill
    members = [len(m) for _, m in groups]
    cum = lambda x: torch.tensor(np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32).to(dev)
    return dict(q=(torch.randn(sum(news), hq, d, generator=gen) * scale).to(dtype).to(dev), kc=kc.to(dev), vc=vc.to(dev),
                table=table.to(dev), cu=cum(news), kv=torch.tensor(kv, dtype=torch.int32).to(dev), cg=cum(members),
                shared=torch.tensor([sh for sh, _ in groups], dtype=torch.int32).to(dev), max_q=max(news + [0]),
                max_group=max([sum(n for _, n in m) for _, m in groups] + [0]), max_kv=max(kv + [0]),
                status=torch.zeros(1, dtype=torch.int32, device=dev), host=(kv, news))


def call(s, **kw):
    a = dict(q=s["q"], cu_seqlens_q=s["cu"], kv_lens=s["kv"], cu_groups=s["cg"], shared_lens=s["shared"], max_q_len=s["max_q"],
             max_group_tokens=s["max_group"], max_kv_len=s["max_kv"], cache=(s["kc"], s["vc"], s["table"]), return_lse=True,
             device_status=s["status"])
    a.update(kw)
    return rpx.group_attn(**a)


def exact(s, softmax_scale=None):
    """out, lse, sum p |v| and S of every row, in 64 bits on the GPU."""
    kv, news = s["host"]
    t, hq, d = s["q"].shape
    hkv = s["kc"].shape[1]
    step, sc = hq // hkv, d ** -0.5 if softmax_scale is None else softmax_scale
    out, pv = (torch.zeros(t, hq, d, dtype=torch.float64, device=s["q"].device) for _ in range(2))
    lse, big = (torch.zeros(t, hq, dtype=torch.float64, device=s["q"].device) for _ in range(2))
    at = 0
    for i, (x, n) in enumerate(zip(kv, news)):
        if n == 0:
            continue
        pages = s["table"][i, :-(-x // PAGE)].long()
        k, v = (c[pages].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :x].double() for c in (s["kc"], s["vc"]))
        q = s["q"][at:at + n].double().view(n, hkv, step, d).permute(1, 2, 0, 3).reshape(hkv, step * n, d)
        z = q @ k.transpose(1, 2) * sc
        seen = torch.ones(n, x, dtype=torch.bool, device=z.device).tril(x - n).repeat(step, 1)
        z = torch.where(seen, z, -np.inf)
        l = torch.logsumexp(z, -1)
        p = torch.where(seen, torch.exp(z - l[..., None]), 0.0)
        back = lambda y: y.view(hkv, step, n, -1).permute(2, 0, 1, 3).reshape(n, hq, -1)
        out[at:at + n], pv[at:at + n] = back(p @ v), back(p @ v.abs())
        lse[at:at + n] = back(l[..., None])[..., 0]
        big[at:at + n] = back((q.abs() @ k.abs().transpose(1, 2) * sc).amax(-1, keepdim=True))[..., 0]
        at += n
    return out, lse, pv, big


def check(s, got, softmax_scale=None):
    """P is one bf16 term only where a block may have more than 64 rows."""
    out, lse, pv, big = exact(s, softmax_scale)
    d = s["q"].shape[2]
    one_term = max(s["max_q"], s["max_group"]) * s["q"].shape[1] // s["kc"].shape[1] > 64
    bf16 = s["q"].dtype == torch.bfloat16
    score = (d + 4) * 2.0 ** -24 * big
    w = score + 2.0 ** -21 + ((2.0 ** -8 if one_term else 2.0 ** -16) if bf16 else 0.0)
    tol = (2.0 ** -8 if bf16 else 2.0 ** -23) * out.abs() + (2 * w + 2.0 ** -13)[..., None] * pv
    err = (got[0].double() - out).abs()
    assert bool((err <= tol).all()), (float(err.max()), float((err / tol).max()))
    gone = (got[1].double() - lse).abs()
    assert bool((gone <= score + 2.0 ** -13 + 2.0 ** -20 * lse.abs()).all()), float(gone.max())


def one(n, own=37):
    return [(own + 5 * i, n) for i in range(3)]


GROUPS = {
    "one_token": [(0, [(1, 1)])],
    "alone_long": [(0, [(5000, 1)])],
    "group_of_8": [(1000, [(1 + 7 * i, 1) for i in range(8)])],
    "shared_in_whole_pages": [(512, [(1, 1)] * 3), (128, [(16, 1)] * 2), (16, [(17, 1)] * 5)],
    "shared_less_than_a_page": [(15, [(1, 1), (2, 1)]), (1, [(130, 1)])],
    "mixed": [(0, [(3, 1)]), (2000, [(300, 1)] * 4), (0, []), (77, [(5, 1), (500, 1), (0 + 1, 1)]), (640, [(129, 1)] * 2)],
    "many_members": [(700, [(1 + i % 40, 1) for i in range(70)])],
    "many_groups": [(i * 13 % 300, [(1 + (i + j) % 50, 1) for j in range(3)]) for i in range(60)],
    "several_tokens": [(900, [(40, 5), (60, 3), (5, 5), (200, 1)]), (33, [(9, 9), (10, 2)])],
    "some_without_queries": [(300, [(40, 1), (60, 0), (5, 2), (0 + 7, 0)]), (64, [(9, 0)])],
    "long_chunks": [(500, [(150, 150), (260, 200)]), (0, [(129, 129)])],
    "long_prompt": [(20000, [(100, 1)] * 2)],
}
HEADS = [(28, 4, 128), (40, 8, 128), (4, 2, 64), (8, 8, 64), (16, 1, 128), (1, 1, 64), (128, 1, 64)]


@pytest.mark.parametrize("name", list(GROUPS))
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_against_the_definition(cuda_device, name, hq, hkv, d):
    s = make(GROUPS[name], hq, hkv, d, cuda_device, fill=float("nan"))
    got = call(s)
    assert int(s["status"]) == 0
    check(s, got)
    again = call(s)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("groups", [[(0, [(1000, 1)])] * 256, [(4090, [(509 + i, 1) for i in range(8)])] * 32,
                                    [(0, [(1 + 17 * i % 999, 1)]) for i in range(300)], [(3000, [(40 + 13 * i, 3) for i in range(5)])] * 20],
                         ids=["alone", "groups", "many_lengths", "three_tokens"])
@pytest.mark.parametrize("hq,hkv,d", [(40, 8, 128), (28, 4, 128), (40, 8, 64)])
def test_many_sequences_that_end_inside_a_page(cuda_device, groups, hq, hkv, d):
    """Every SM goes through dozens of segments whose last page is partly empty (and holds anything)."""
    s = make(groups, hq, hkv, d, cuda_device, fill=float("inf"))
    for bounds in (dict(), dict(max_group_tokens=s["max_group"] + 8), dict(max_group_tokens=s["max_group"] + 40)):
        for _ in range(2):
            check(s, call(s, **bounds))
    assert int(s["status"]) == 0


@pytest.mark.parametrize("name", ["one_token", "group_of_8", "mixed", "several_tokens", "long_chunks"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (6, 2, 128)])
def test_float32(cuda_device, name, hq, hkv, d):
    s = make(GROUPS[name], hq, hkv, d, cuda_device, dtype=torch.float32, fill=float("nan"))
    got = call(s)
    assert int(s["status"]) == 0
    check(s, got)


@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (4, 2, 64)])
def test_sharing_is_the_same_as_not_sharing(cuda_device, hq, hkv, d):
    s = make([(900, [(40, 2), (60, 1), (5, 1)]), (330, [(100, 1)] * 6)], hq, hkv, d, cuda_device)
    for shared in ([900, 330], [0, 0], [17, 331], [1, 15], [896, 0]):
        s["shared"] = torch.tensor(shared, dtype=torch.int32, device=cuda_device)
        check(s, call(s))
    none = torch.zeros(0, dtype=torch.int32, device=cuda_device)
    check(s, call(s, cu_groups=torch.zeros(1, dtype=torch.int32, device=cuda_device), shared_lens=none))
    assert int(s["status"]) == 0


@pytest.mark.parametrize("factor", [0.01, 30.0, 300.0])
def test_scores_far_apart(cuda_device, factor):
    """Sharp rows (one key holds all weight, maxima that rise along the keys) and flat ones."""
    for groups in (GROUPS["mixed"], GROUPS["several_tokens"], GROUPS["many_members"]):
        s = make(groups, 10, 2, 128, cuda_device)
        s["kc"] *= torch.linspace(0.1, 1.0, s["kc"].shape[0], device=cuda_device).to(torch.bfloat16)[:, None, None, None]
        check(s, call(s, softmax_scale=factor / 128), softmax_scale=factor / 128)


def test_rising_maximum_along_a_sequence(cuda_device):
    """Keys grow along the positions, so every tile raises the running maximum by far more than it may lag."""
    for d in (64, 128):
        s = make([(1500, [(700, 1), (20, 1), (400, 3)])], 14, 2, d, cuda_device)
        kv, _ = s["host"]
        q = s["q"].abs()
        s["q"].copy_(q)
        for i, x in enumerate(kv):
            pos = torch.arange(x, device=cuda_device)
            size = (pos.float() / 40 + 0.01)[:, None, None].bfloat16()
            k = s["kc"][s["table"][i, pos // PAGE].long(), :, pos % PAGE]
            s["kc"][s["table"][i, pos // PAGE].long(), :, pos % PAGE] = size * torch.ones_like(k)
        check(s, call(s))


def test_values_that_are_not_finite_stay_with_their_rows(cuda_device):
    inf = float("inf")
    s = make([(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 1), (200, 2)])], 8, 2, 128, cuda_device)
    want = call(s)
    q = s["q"].clone()
    s["q"][1, 3] = float("nan")
    got = call(s)
    assert bool(got[0][1, 3].isnan().all()) and bool(got[1][1, 3].isnan())
    got[0][1, 3], got[1][1, 3] = want[0][1, 3], want[1][1, 3]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s["q"].copy_(q)
    # a key of -inf in sequence 0's own part: rows whose product with it is -inf do without it, the others are NaN
    page, place = int(s["table"][0, 510 // PAGE]), 510 % PAGE
    s["kc"][page, 0, place] = 0
    s["kc"][page, 0, place, 0] = -inf
    s["q"][0, :4, 0] = torch.tensor([1.0, 2.0, -1.0, -3.0], device=cuda_device)
    got = call(s)
    assert bool(got[0][0, 2:4].isnan().all()) and bool(got[0][0, :2].isfinite().all())
    assert torch.equal(got[0][1:], call(s)[0][1:]) and bool(got[0][1:].isfinite().all())


def _groups(dev, cu):
    return torch.tensor(cu, dtype=torch.int32, device=dev)


@pytest.mark.parametrize("change", [
    dict(cg=[0, 3, 2]), dict(cg=[0, 3, 6]), dict(cg=[-1, 3, 5]), dict(cg=[0, 2 ** 31 - 1, 5]), dict(cg=[1, 0, 5]), dict(cg=[0, 5, 3]),
    dict(shared=[-1, 64]), dict(shared=[506, 64]), dict(shared=[500, 2 ** 31 - 1]), dict(max_group=2), dict(shared=[500, 72])])
def test_groups_that_do_not_fit_share_nothing(cuda_device, change):
    s = make([(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 2), (200, 2)])], 8, 2, 128, cuda_device)
    for k, v in change.items():
        s[k] = v if k == "max_group" else torch.tensor(v, dtype=torch.int32, device=cuda_device)
    got = call(s)
    assert int(s["status"]) == -8
    check(s, got)


@pytest.mark.parametrize("change,out_rows", [
    (dict(kv=[540, 560, 505, 1, 264]), [3, 4]), (dict(kv=[540, -1, 505, 73, 264]), [1]), (dict(kv=[540, 10 ** 9, 505, 73, 264]), [1]),
    (dict(max_q=1), [3, 4, 5, 6]), (dict(cu=[0, 1, 2, 3, 5, 8]), [5, 6]), (dict(cu=[-1, 1, 2, 3, 5, 7]), [0]),
    (dict(cu=[0, 1, 2, 3, 5, 2 ** 31 - 1]), [5, 6])])
def test_sequences_that_do_not_fit_are_left_out(cuda_device, change, out_rows):
    s = make([(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 2), (200, 2)])], 8, 2, 128, cuda_device)
    want = exact(s)
    for k, v in change.items():
        s[k] = v if k == "max_q" else torch.tensor(v, dtype=torch.int32, device=cuda_device)
    out = torch.full_like(s["q"], 9.0)
    lse = torch.full(s["q"].shape[:2], 9.0, device=cuda_device)
    got = call(s, out=out, lse=lse)
    assert int(s["status"]) == -8
    for t in range(7):
        if t in out_rows:
            assert bool((got[0][t] == 9).all()) and bool((got[1][t] == 9).all())
        else:
            assert float((got[0][t].double() - want[0][t]).abs().max()) < 0.03


@pytest.mark.parametrize("number", [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_page_numbers_out_of_the_pool(cuda_device, number, dtype):
    """Reported; the other sequences' rows are as they were."""
    s = make([(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 2), (200, 2)])], 8, 2, 128, cuda_device, dtype=dtype)
    want = call(s)
    s["table"][1, 33] = number  # of the second sequence's own pages
    got = call(s)
    assert int(s["status"]) == -8
    rows = [0, 2, 3, 4, 5, 6]
    assert torch.equal(got[0][rows], want[0][rows])


def test_rows_of_no_sequence_strides_and_alignment(cuda_device):
    s = make([(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 2), (200, 2)])], 8, 2, 128, cuda_device)
    want = call(s)
    # queries inside a wider projection; two tokens in front of the first sequence, one behind the last
    wide = torch.randn(10, 16, 128, device=cuda_device).bfloat16()
    wide[2:9, 3:11] = s["q"]
    s["q"], s["cu"] = wide[:, 3:11], s["cu"] + 2
    out = torch.full((10, 8, 128), 9.0, device=cuda_device, dtype=torch.bfloat16)
    got = call(s, out=out)
    assert torch.equal(got[0][2:9], want[0]) and torch.equal(got[1][2:9], want[1])
    assert bool((out[[0, 1, 9]] == 9).all())
    # an output that starts on 16 bytes and no more, and a table with a wider stride
    room = torch.zeros(10 * 8 * 128 + 8, device=cuda_device, dtype=torch.bfloat16)
    table = torch.full((5, 100), -5, dtype=torch.int32, device=cuda_device)
    table[:, 30:30 + s["table"].shape[1]] = s["table"]
    got = call(s, out=room[8:].view(10, 8, 128), cache=(s["kc"], s["vc"], table[:, 30:30 + s["table"].shape[1]]))
    assert torch.equal(got[0][2:9], want[0])


def test_bounds_larger_than_needed(cuda_device):
    s = make(GROUPS["mixed"], 28, 4, 128, cuda_device)
    for bounds in (dict(max_kv_len=100000), dict(max_kv_len=1), dict(max_q_len=7), dict(max_q_len=60), dict(max_group_tokens=5000)):
        check(s, call(s, **bounds))
    assert int(s["status"]) == 0


def test_stream_graph_and_shared_workspace(cuda_device):
    s = make(GROUPS["mixed"], 28, 4, 128, cuda_device)
    s2 = make(GROUPS["several_tokens"], 28, 4, 128, cuda_device)
    want, want2 = call(s), call(s2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(s, stream=side)
    got2 = call(s2)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got2[0], want2[0])
    ws = torch.empty(1 << 28, dtype=torch.uint8, device=cuda_device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(s, workspace=ws)
        got2 = call(s2, workspace=ws)
    for _ in range(3):
        ws.fill_(255)
        for x in (*got, *got2):
            x.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((*got, *got2), (*want, *want2)))
    # the next step: one token more for every sequence of the first batch, through the same graph
    s["q"] *= 0.5
    graph.replay()
    check(s, got)


def test_nothing_to_do(cuda_device):
    s = make([(0, [])], 8, 2, 128, cuda_device)
    assert call(s)[0].shape[0] == 0
    s = make([(100, [(5, 0)])], 8, 2, 128, cuda_device)
    assert call(s)[0].shape[0] == 0
    s = make([(100, [(5, 1)])], 8, 2, 128, cuda_device)
    out = torch.full_like(s["q"], 9.0)
    call(s, max_q_len=0, out=out)
    assert bool((out == 9).all())


def test_random_batches(cuda_device):
    rng = np.random.default_rng(5)
    for seed in range(25):
        hkv = int(rng.choice([1, 2, 4, 8]))
        hq, d = hkv * int(rng.choice([1, 3, 5, 7, 8])), int(rng.choice([64, 128]))
        groups = []
        for _ in range(int(rng.integers(1, 9))):
            members = []
            for _ in range(int(rng.integers(1, 20))):
                n = int(rng.choice([1, 1, 1, 0, 2, 6]))
                members.append((n + int(rng.integers(0, 400)) if rng.random() < 0.8 else max(n, 1), n))
            groups.append((int(rng.choice([0, 5, int(rng.integers(0, 3000))])), members))
        s = make(groups, hq, hkv, d, cuda_device, seed=seed, fill=float("nan"))
        if s["q"].shape[0] == 0:
            continue
        got = call(s)
        assert int(s["status"]) == 0
        check(s, got)
