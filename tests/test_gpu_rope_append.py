"""GPU parity of norm + rotation with K and V stored into the cache on the way: against the formula in 64 bits, and bit for bit
against the two calls that it stands for (qk_norm_rope, then cache_append).

Tolerances as for qk_norm_rope: half a step of the type that is stored (bf16 2^-8, float32 2^-24, relative to the value) and
2^-18 (|y_a| + |y_b|) for the arithmetic of a turned pair.
"""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
PAGE = 16


def make(new, lens, hq, hkv, d, rot, axes, dtype, norm, dev, seed=0, spare=5):
    gen = torch.Generator().manual_seed(seed)
    t, rows = sum(new), hq + 2 * hkv
    scale = torch.exp(0.7 * torch.randn(t, rows, 1, generator=gen))
    qkv = (torch.randn(t, rows, d, generator=gen) * scale).to(DT[dtype]).to(dev)
    pages = [-(-(n + c) // PAGE) for n, c in zip(new, lens)]
    nb = sum(pages) + spare
    perm = torch.randperm(nb, generator=gen).int()
    table = torch.full((len(new), max(pages + [1]) + 2), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n
    n = rot // 2
    s = dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], table=table.to(dev),
             kc=torch.randn(nb, hkv, PAGE, d, generator=gen).bfloat16().to(dev),
             vc=torch.randn(nb, hkv, PAGE, d, generator=gen).bfloat16().to(dev),
             cu=torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).to(dev),
             lens=torch.tensor(lens, dtype=torch.int32).to(dev), max_new=max(new + [0]),
             pos=torch.randint(-5, 200000, (axes, t), generator=gen, dtype=torch.int32).to(dev),
             inv=(10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().to(dev),
             axis=torch.randint(0, axes, (n,), generator=gen).tolist(),
             w=[(1 + 0.3 * torch.randn(d, generator=gen)).to(DT[dtype]).to(dev) if norm else None for _ in range(2)],
             status=torch.zeros(1, dtype=torch.int32, device=dev))
    return s


def call(s, **kw):
    a = dict(q=s["q"], k=s["k"], v=s["v"], positions=s["pos"], inv_freq=s["inv"], cu_append=s["cu"], cached_lens=s["lens"],
             max_append=s["max_new"], cache=(s["kc"], s["vc"], s["table"]), q_weight=s["w"][0], k_weight=s["w"][1],
             pair_axis=s["axis"], eps=1e-6, device_status=s["status"])
    a.update(kw)
    return rpx.qk_norm_rope_append(**a)


def formula(x, w, pos, inv, axis):
    x = x.double().cpu()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double().cpu()
    n = len(axis)
    a = (pos.double().cpu()[axis].t() * inv.double().cpu())[:, None]
    c, s = torch.cos(a), torch.sin(a)
    both = x[..., :n].abs() + x[..., n:2 * n].abs()
    y = torch.cat([x[..., :n] * c - x[..., n:2 * n] * s, x[..., n:2 * n] * c + x[..., :n] * s, x[..., 2 * n:]], -1)
    return y, torch.cat([both, both, x[..., 2 * n:].abs()], -1)


def slots(new, lens, table):
    """(page, place) of every token, in order."""
    out = [(int(table[i, (c + j) // PAGE]), (c + j) % PAGE) for i, (n, c) in enumerate(zip(new, lens)) for j in range(n)]
    return torch.tensor([p for p, _ in out], dtype=torch.long), torch.tensor([x for _, x in out], dtype=torch.long)


CASES = [  # new, cached, hq, hkv, d, rot, axes, dtype, norm
    ([1], [0], 4, 2, 128, 128, 3, "bf16", True),
    ([1] * 37, list(range(0, 37 * 3, 3)), 28, 4, 128, 128, 3, "bf16", True),
    ([17, 0, 1, 130, 16, 0], [15, 7, 16, 31, 0, 0], 40, 8, 128, 64, 2, "bf16", True),
    ([5, 33], [1000, 0], 4, 2, 64, 32, 1, "f32", False),
    ([300], [5], 3, 3, 64, 64, 1, "f32", True),
    ([9, 2, 4], [0, 500, 3], 16, 1, 128, 16, 4, "bf16", False),
    ([1] * 700, [i % 50 for i in range(700)], 4, 1, 64, 48, 1, "bf16", True),
]


@pytest.mark.parametrize("case", CASES)
def test_against_the_formula_and_the_two_calls(cuda_device, case):
    new, lens = case[:2]
    s = make(*case, cuda_device)
    kc0, vc0 = s["kc"].clone(), s["vc"].clone()
    q0 = s["q"].clone()
    q_two, k_two = rpx.qk_norm_rope(s["q"], s["k"], s["pos"], s["inv"], q_weight=s["w"][0], k_weight=s["w"][1], pair_axis=s["axis"], eps=1e-6)
    kc2, vc2 = kc0.clone(), vc0.clone()
    rpx.cache_append(k_two, s["v"].contiguous(), s["cu"], s["lens"], s["max_new"], (kc2, vc2, s["table"]))
    q = call(s)
    assert int(s["status"]) == 0
    assert torch.equal(q, q_two) and torch.equal(s["kc"], kc2) and torch.equal(s["vc"], vc2)
    assert torch.equal(s["q"], q0)
    for got, x, w, in ((q, s["q"], s["w"][0]), (s["kc"][slots(new, lens, s["table"].cpu())[0].to(cuda_device), :, slots(new, lens, s["table"].cpu())[1].to(cuda_device)], s["k"], s["w"][1])):
        ref, size = formula(x, w, s["pos"], s["inv"], s["axis"])
        err = (got.double().cpu() - ref).abs()
        assert bool((err <= HALF_STEP[got.dtype] * ref.abs() + 2.0 ** -18 * size).all()), float(err.max())
    page, place = slots(new, lens, s["table"].cpu())
    kc0[page.to(cuda_device), :, place.to(cuda_device)] = s["kc"][page.to(cuda_device), :, place.to(cuda_device)]
    assert torch.equal(kc0, s["kc"])  # no other slot has changed
    again = s["kc"].clone()
    assert torch.equal(call(s), q) and torch.equal(s["kc"], again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_positions_a_token_takes_its_place(cuda_device, dtype):
    new, lens = [3, 0, 40, 1], [100, 4, 0, 2047]
    s = make(new, lens, 8, 2, 128, 128, 1, dtype, True, cuda_device)
    place = torch.tensor([c + j for n, c in zip(new, lens) for j in range(n)], dtype=torch.int32, device=cuda_device)
    q = call(s, positions=place, pair_axis=None)
    kc = s["kc"].clone()
    assert torch.equal(call(s, positions=None, pair_axis=None), q) and torch.equal(s["kc"], kc)
    with pytest.raises(ValueError):
        call(s, positions=None)


def test_tokens_of_no_sequence_and_in_place(cuda_device):
    new, lens = [6, 5, 7], [3, 30, 0]
    s = make(new, lens, 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    want = call(s)
    kc = s["kc"].clone()
    s["cu"] = torch.tensor([2, 6, 11, 14], dtype=torch.int32, device=cuda_device)  # two tokens in front, four behind
    q_out = torch.full_like(want, 7.0)
    call(s, q_out=q_out)
    assert torch.equal(q_out[2:14], want[2:14]) and bool((q_out[:2] == 7).all()) and bool((q_out[14:] == 7).all())
    assert int(s["status"]) == 0
    s2 = make(new, lens, 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    call(s2, q_out=s2["q"])
    assert torch.equal(s2["q"], want) and torch.equal(s2["kc"], kc)


def _bad(s, dev):
    """Each: what is changed, and the tokens that must not be stored (the others must)."""
    big = 10 ** 9
    return [
        (dict(cached_lens=torch.tensor([3, -1, 0], dtype=torch.int32, device=dev)), range(6, 11)),
        (dict(cached_lens=torch.tensor([3, big, 0], dtype=torch.int32, device=dev)), range(6, 11)),
        (dict(max_append=6), range(11, 18)),
        (dict(cu_append=torch.tensor([0, 6, 11, 19], dtype=torch.int32, device=dev)), range(11, 18)),
        (dict(cu_append=torch.tensor([-1, 6, 11, 18], dtype=torch.int32, device=dev)), range(0, 6)),
        (dict(cu_append=torch.tensor([0, 6, 11, 2 ** 31 - 1], dtype=torch.int32, device=dev)), range(11, 18)),
    ]


@pytest.mark.parametrize("which", range(6))
def test_sequences_that_do_not_fit(cuda_device, which):
    new, lens = [6, 5, 7], [3, 30, 0]
    s = make(new, lens, 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    kc0 = s["kc"].clone()
    want = call(s)
    kc = s["kc"].clone()
    change, left_out = _bad(s, cuda_device)[which]
    s["kc"].copy_(kc0)
    q_out = torch.full_like(want, 7.0)
    call(s, q_out=q_out, **change)
    assert int(s["status"]) == -8
    page, place = slots(new, lens, s["table"].cpu())
    for t in range(18):
        p, x = int(page[t]), int(place[t])
        if t in left_out:
            assert bool((q_out[t] == 7).all()) and torch.equal(s["kc"][p, :, x], kc0[p, :, x])
        else:
            assert torch.equal(q_out[t], want[t]) and torch.equal(s["kc"][p, :, x], kc[p, :, x])


@pytest.mark.parametrize("number", [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1])
def test_page_numbers_out_of_the_pool(cuda_device, number):
    new, lens = [6, 20], [3, 30]
    s = make(new, lens, 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    kc0 = s["kc"].clone()
    want = call(s)
    kc = s["kc"].clone()
    s["kc"].copy_(kc0)
    broken = int(s["table"][1, 2])
    s["table"][1, 2] = number
    assert torch.equal(call(s), want) and int(s["status"]) == -8
    kc[broken] = kc0[broken]
    assert torch.equal(s["kc"], kc)


def test_stream_and_graph(cuda_device):
    new, lens = [1] * 20, [50 + i for i in range(20)]
    s = make(new, lens, 28, 4, 128, 128, 3, "bf16", True, cuda_device)
    want, kc = call(s), s["kc"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(s, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    q_out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, q_out=q_out)
    for _ in range(2):
        s["kc"].zero_()
        q_out.zero_()
        graph.replay()
        page, place = (x.to(cuda_device) for x in slots(new, lens, s["table"].cpu()))
        assert torch.equal(q_out, want) and torch.equal(s["kc"][page, :, place], kc[page, :, place])
    # the lengths have moved on: the same graph stores one place further
    s["lens"] -= 1
    before = s["kc"].clone()
    graph.replay()
    page, place = (x.to(cuda_device) for x in slots(new, [c - 1 for c in lens], s["table"].cpu()))
    before[page, :, place] = s["kc"][page, :, place]
    assert torch.equal(before, s["kc"]) and bool((s["kc"][page, :, place] != 0).any())


def test_empty_calls(cuda_device):
    s = make([4], [0], 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    kc0 = s["kc"].clone()
    none = make([], [], 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    assert call(none).shape[0] == 0
    call(s, max_append=0)
    call(s, cu_append=torch.zeros(1, dtype=torch.int32, device=cuda_device), cached_lens=torch.zeros(0, dtype=torch.int32, device=cuda_device))
    assert torch.equal(s["kc"], kc0) and int(s["status"]) == 0


@pytest.mark.parametrize("batch", [31, 32, 33, 63, 64, 65, 1023, 1024, 1025, 4000])
@pytest.mark.parametrize("norm", [True, False])
def test_any_number_of_sequences(cuda_device, batch, norm):
    """Which sequence a token is in, some of them empty: as cache_append finds it."""
    gen = np.random.default_rng(batch)
    new = gen.integers(0, 4, batch).tolist()
    new[0], new[-1] = (0, 2) if batch % 2 else (1, 0)
    s = make(new, gen.integers(0, 40, batch).tolist(), 4, 2, 64, 64, 2, "bf16", norm, cuda_device)
    q_two, k_two = rpx.qk_norm_rope(s["q"], s["k"], s["pos"], s["inv"], q_weight=s["w"][0], k_weight=s["w"][1], pair_axis=s["axis"], eps=1e-6)
    kc, vc = s["kc"].clone(), s["vc"].clone()
    rpx.cache_append(k_two, s["v"].contiguous(), s["cu"], s["lens"], s["max_new"], (kc, vc, s["table"]))
    q = call(s)
    assert int(s["status"]) == 0
    assert torch.equal(q, q_two) and torch.equal(s["kc"], kc) and torch.equal(s["vc"], vc)
