"""GPU parity of the clipped policy loss and its gradient against the formula in 64 bits (and its gradient against differences).

Tolerances, with e = 2^-24.  A ratio: d rounded once (|d| e), expm1 (2 e), the sum and the reciprocal (2 e); its product with
the advantage and with the weight, itself rounded, and with upstream: (|d| + 8) e relative.  A KL term: f - l rounded once moves
e^x by |x| e^x e, expm1 2 e of itself, series or difference 4 e of |x| e^|x|; coefficient and products 4 e.  The sums of
ratios and of policy terms are by fours in float32 (3 e, of the 8), and all of them in 64 bits beyond, rounded once (e).
"""
import math

import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def make(lens, dev, seed=0, spread=0.3, mask=None, per_token=False, lead=0, tail=0):
    gen = torch.Generator().manual_seed(seed)
    t = sum(lens) + lead + tail
    lp = -torch.rand(t, generator=gen) * 4
    s = dict(lp=lp, old=lp + spread * torch.randn(t, generator=gen), ref=lp + spread * torch.randn(t, generator=gen),
             adv=torch.randn(t if per_token else len(lens), generator=gen),
             cu=torch.tensor(np.concatenate([[lead], lead + np.cumsum(lens)]), dtype=torch.int32),
             mask=None if mask is None else torch.rand(t, generator=gen) < mask)
    return {k: v if v is None else v.to(dev) for k, v in s.items()}


def formula(s, ratio="token", mean="sequences", kl=3, low=0.2, high=0.2, dual=0.0, coef=0.0, count=0.0, up=1.0):
    """Loss terms, gradient and the size of the terms that its roundings go by, in 64 bits."""
    lp = s["lp"].double().cpu()
    old = lp if s["old"] is None else s["old"].double().cpu()
    ref = None if s["ref"] is None or kl == 0 else s["ref"].double().cpu()
    adv, cu = s["adv"].double().cpu(), s["cu"].tolist()
    t = lp.shape[0]
    keep = torch.ones(t, dtype=torch.bool) if s["mask"] is None else s["mask"].cpu() != 0
    n = [int(keep[a:b].sum()) for a, b in zip(cu, cu[1:])]
    total, seqs = sum(n), sum(1 for x in n if x)
    grad, tol = torch.zeros(t, dtype=torch.float64), torch.zeros(t, dtype=torch.float64)
    sums, sizes = np.zeros(4), np.zeros(4)
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        if not n[i]:
            continue
        at = torch.nonzero(keep[a:b])[:, 0] + a
        d = lp[at] - old[at]
        if ratio == "sequence":
            d = d.mean().expand(n[i])
        A = adv[at] if adv.shape[0] == t and adv.shape[0] != len(n) else adv[i].expand(n[i])
        r = torch.exp(d)
        pol = torch.maximum(-A * r, -A * r.clamp(1 - low, 1 + high))
        if dual:
            pol = torch.where(A < 0, torch.minimum(pol, -A * dual), pol)
        cut = pol != -A * r
        w = 1.0 / ((count or total) if mean == "tokens" else n[i] * (count or seqs))
        g, size = torch.where(cut, 0.0, -A * r), torch.where(cut, 0.0, (A * r).abs() * (d.abs() + 8))
        klt, ksize = torch.zeros_like(r), torch.zeros_like(r)
        if ref is not None:
            x = ref[at] - lp[at]
            klt = {1: -x, 2: x * x / 2, 3: torch.exp(x) - 1 - x}[kl]
            dk = {1: torch.ones_like(x), 2: -x, 3: 1 - torch.exp(x)}[kl]
            g = g + coef * dk
            ksize = {1: x.abs(), 2: 4 * klt, 3: 8 * x.abs() * torch.exp(x.abs())}[kl]
            size = size + coef * (dk.abs() * 8 + {1: 0.0, 2: x.abs(), 3: x.abs() * torch.exp(x)}[kl])
        grad[at], tol[at] = up * w * g, abs(up) * w * size * E + 3 * E * (up * w * g).abs()
        for j, (term, part) in enumerate(((pol, (A * r).abs() * (d.abs() + 8)), (klt, ksize), (cut.double(), r * 0), (r, r * (d.abs() + 8)))):
            sums[j] += w * float(term.sum())
            sizes[j] += w * float(part.sum())
    stats = np.array([sums[0] + coef * sums[1], *sums, total])
    stol = E * np.array([sizes[0] + coef * sizes[1], *sizes, 0.0]) + 2 * E * np.abs(stats)
    return stats, stol, grad, tol, keep


def call(s, ratio="token", mean="sequences", kl=3, low=0.2, high=0.2, dual=0.0, coef=0.0, count=0.0, up=None, **kw):
    return rpx.policy_loss(s["lp"], s["old"], s["adv"], s["cu"], mask=s["mask"], ref_logprobs=s["ref"], clip_low=low, clip_high=high,
                           clip_dual=dual, kl_coef=coef, kl=kl, ratio=ratio, mean=mean, count=count,
                           upstream=None if up is None else torch.tensor([up], device=s["lp"].device), **kw)


def check(s, got, **kw):
    stats, stol, grad, tol, _ = formula(s, **{k: v for k, v in kw.items() if not (k == "up" and v is None)})
    inside = torch.zeros(s["lp"].shape[0], dtype=torch.bool)
    inside[int(s["cu"][0]):int(s["cu"][-1])] = True
    err = np.abs(got[0].double().cpu().numpy() - stats)
    assert (err <= stol).all(), (err, stol, stats)
    diff = (got[1].double().cpu() - grad).abs()[inside]
    assert bool((diff <= tol[inside]).all()), (float(diff.max()), float(tol.max()))


LENS = [[1], [250] * 8, [3, 0, 1, 700, 2, 0, 64], [1] * 900, [8191], [4096, 4097], [1, 9000, 5], [2000] * 30, [0, 0, 20000, 0, 1], [1] * 9000]


@pytest.mark.parametrize("lens", LENS, ids=[f"{len(x)}x{max(x)}" for x in LENS])
@pytest.mark.parametrize("ratio,mean,kl,dual,per_token", [("token", "sequences", 3, 0.0, False), ("token", "tokens", 3, 1.5, True),
                                                          ("sequence", "sequences", 2, 1.2, False), ("sequence", "tokens", 1, 0.0, False),
                                                          ("token", "sequences", 0, 2.0, True)])
@pytest.mark.parametrize("mask", [None, 0.6])
def test_against_the_formula(cuda_device, lens, ratio, mean, kl, dual, per_token, mask):
    if per_token and sum(lens) == len(lens):
        pytest.skip("one advantage for each token is one for each sequence")
    s = make(lens, cuda_device, mask=mask, per_token=per_token)
    kw = dict(ratio=ratio, mean=mean, kl=kl, dual=dual, coef=0.05, low=0.1, high=0.3)
    got = call(s, **kw)
    check(s, got, **kw)
    again = call(s, **kw)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_gradient_against_differences(cuda_device):
    """Central differences of the loss: steps of 2^-8 in log-probs on a grid of 2^-10, spread wide enough that few tokens come
    within a step of a border (those are left out)."""
    lens = [40, 3, 90]
    for ratio in ("token", "sequence"):
        s = make(lens, cuda_device, seed=3, mask=0.8)
        for k in ("lp", "old", "ref"):
            s[k] = torch.round(s[k] * 1024) / 1024
        kw = dict(ratio=ratio, mean="tokens", kl=3, dual=1.4, coef=0.3)
        grad = call(s, **kw)[1].cpu()
        h = 2.0 ** -8
        keep = s["mask"].cpu()
        lp0 = s["lp"].clone()
        for i in range(0, sum(lens), 7):
            loss = []
            clipped = []
            for sign in (1, -1):
                s["lp"] = lp0.clone()
                s["lp"][i] += sign * h
                stats = formula(s, **kw)[0]  # (the loss in 64 bits; the kernel's own is compared with it above)
                loss.append(stats[0])
                clipped.append(stats[3])
            s["lp"] = lp0
            if clipped[0] != clipped[1]:
                continue
            want = (loss[0] - loss[1]) / (2 * h)
            # the third derivative of e^x times h^2 / 6, in units of the gradient's own terms
            assert abs(float(grad[i]) - want) <= 1e-4 * max(abs(want), 1.0 / sum(lens)), (i, float(grad[i]), want)
            if not bool(keep[i]):
                assert float(grad[i]) == 0.0


def test_borders_are_decided_in_64_bits(cuda_device):
    """d just inside and just outside of log(1.2) and log(0.8): neighbours in float32 around the border, whose r round alike."""
    for border, a in ((math.log1p(0.2), 1.0), (math.log1p(-0.2), -1.0)):
        d = np.float32(border)
        near = [np.nextafter(d, np.float32(-10)), d, np.nextafter(d, np.float32(10))]
        dev = cuda_device
        lp = torch.tensor(near, dtype=torch.float32, device=dev)
        s = dict(lp=lp, old=torch.zeros(3, device=dev), ref=None, mask=None, adv=torch.tensor([a], device=dev),
                 cu=torch.tensor([0, 3], dtype=torch.int32, device=dev))
        grad = call(s)[1].cpu()
        for i, x in enumerate(near):
            cut = float(x) > border if a > 0 else float(x) < border
            assert (float(grad[i]) == 0.0) == cut, (border, i)


def test_what_lies_at_masked_tokens_is_not_used(cuda_device):
    lens = [100, 5000, 7, 4000]
    for lens in (lens[:1] + lens[2:3], lens):
        s = make(lens, cuda_device, mask=0.5, per_token=True)
        for ratio in ("token", "sequence"):
            if ratio == "sequence":
                s["adv"] = torch.randn(len(lens), device=cuda_device)
            want = call(s, ratio=ratio, coef=0.1)
            dirty = dict(s)
            off = ~s["mask"]
            for k, bad in (("lp", math.nan), ("old", math.inf), ("ref", -math.inf)):
                dirty[k] = torch.where(off, bad, s[k])
            got = call(dirty, ratio=ratio, coef=0.1)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert bool((got[1][off] == 0).all())


def test_nothing_counted(cuda_device):
    for lens in ([5, 0, 3], [6000, 4000]):
        s = make(lens, cuda_device)
        s["mask"] = torch.zeros(sum(lens), dtype=torch.uint8, device=cuda_device)
        for ratio in ("token", "sequence"):
            for mean in ("tokens", "sequences"):
                stats, grad = call(s, ratio=ratio, mean=mean, coef=0.1)
                assert bool((stats == 0).all()) and bool((grad == 0).all())
    s = make([], cuda_device)
    stats, grad = call(s)
    assert bool((stats == 0).all()) and grad.numel() == 0


def test_tokens_of_no_sequence_keep_their_gradient(cuda_device):
    for lens in ([30, 41], [3000, 0, 7001]):
        s = make(lens, cuda_device, lead=5, tail=9, mask=0.7)
        out = torch.full_like(s["lp"], 3.0)
        got = call(s, coef=0.1, dlogprobs=out)
        check(s, got, coef=0.1)
        assert bool((out[:5] == 3).all()) and bool((out[-9:] == 3).all())


def test_count_upstream_and_on_policy(cuda_device):
    for lens in ([30, 41, 200], [3000, 7001]):
        s = make(lens, cuda_device, mask=0.7)
        for mean, count in (("tokens", 12345.0), ("sequences", 64.0)):
            kw = dict(mean=mean, count=count, coef=0.1, up=-2.5)
            check(s, call(s, **kw), **kw)
        s["old"] = None
        got = call(s, coef=0.1)
        check(s, got, coef=0.1)
        assert float(got[0][3]) == 0.0
        stats, none = call(s, coef=0.1, want_grad=False)
        assert none is None and torch.equal(stats, got[0])
        # a batch in two parts: with the whole batch's count the parts add up
        whole = call(s, mean="tokens", coef=0.1)
        cut = int(s["cu"][1])
        parts = []
        for a, b, cu, adv in ((0, cut, [0, cut], s["adv"][:1]), (cut, sum(lens), [0] + [int(x) - cut for x in s["cu"][2:]], s["adv"][1:])):
            part = dict(lp=s["lp"][a:b], old=None, ref=s["ref"][a:b], mask=s["mask"][a:b], adv=adv.contiguous(),
                        cu=torch.tensor(cu, dtype=torch.int32, device=cuda_device))
            parts.append(call(part, mean="tokens", coef=0.1, count=float(whole[0][5])))
        assert torch.equal(torch.cat([parts[0][1], parts[1][1]]), whole[1])
        # each loss is rounded once, their sum once more
        a, b = (float(p[0][0]) for p in parts)
        assert abs(a + b - float(whole[0][0])) <= E * (abs(a) + abs(b) + abs(float(whole[0][0])))


def test_any_alignment(cuda_device):
    for lens in ([33, 100], [3000, 7001]):
        s = make(lens, cuda_device, mask=0.7)
        want = call(s, coef=0.1)
        t = sum(lens)
        for shift in (1, 2, 3):
            off = dict(s)
            for k in ("lp", "old", "ref", "mask"):
                room = torch.zeros(t + 8, dtype=s[k].dtype, device=cuda_device)
                room[shift:shift + t] = s[k]
                off[k] = room[shift:shift + t]
            out = torch.zeros(t + 8, device=cuda_device)
            got = call(off, coef=0.1, dlogprobs=out[shift:shift + t])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert bool((out[:shift] == 0).all()) and bool((out[shift + t:] == 0).all())


@pytest.mark.parametrize("cu", [[0, 50, 40, 100], [-3, 50, 60, 100], [0, 50, 60, 101], [0, 2 ** 31 - 1, 60, 100], [0, -2 ** 31, 60, 100]])
def test_offsets_that_do_not_fit_are_reported(cuda_device, cu):
    for scale in (1, 150):
        s = make([50 * scale, 10 * scale, 40 * scale], cuda_device, mask=0.8)
        s["cu"] = torch.tensor([x * scale if abs(x) < 2 ** 20 else x for x in cu], dtype=torch.int32, device=cuda_device)
        status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
        call(s, coef=0.1, device_status=status)
        assert int(status) == -8


def test_infinities_go_by_the_formula(cuda_device):
    dev = cuda_device
    inf = math.inf
    lp = torch.tensor([-inf, 0.0, 0.0, math.nan], device=dev)
    s = dict(lp=lp, old=torch.tensor([-1.0, -inf, -200.0, 0.0], device=dev), ref=None, mask=None,
             adv=torch.tensor([1.0, 1.0, -1.0, 1.0], device=dev), cu=torch.arange(5, dtype=torch.int32, device=dev))
    stats, grad = call(s, mean="tokens")
    grad = grad.cpu()
    assert float(grad[0]) == 0.0      # r = 0
    assert float(grad[1]) == 0.0      # r = inf, held
    assert float(grad[2]) == inf      # r = e^200, not held on this side
    assert math.isnan(float(grad[3])) and math.isnan(float(stats[0]))


def test_stream_graph_and_two_workspaces(cuda_device):
    for lens in ([250] * 8, [2000] * 30):
        s = make(lens, cuda_device, mask=0.9)
        want = call(s, coef=0.1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(s, coef=0.1, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            stats, grad = call(s, coef=0.1)
            stats2, grad2 = call(s, coef=0.1, ratio="sequence")
        want2 = call(s, coef=0.1, ratio="sequence")
        for _ in range(3):
            grad.zero_()
            stats.zero_()
            graph.replay()
            assert torch.equal(stats, want[0]) and torch.equal(grad, want[1])
            assert torch.equal(stats2, want2[0]) and torch.equal(grad2, want2[1])
        s["lp"] += 0.01
        want = call(s, coef=0.1)
        graph.replay()
        assert torch.equal(stats, want[0]) and torch.equal(grad, want[1])


def test_exponentials_over_their_range(cuda_device):
    """The ratio and the KL term alone, one token a call's sequence, at differences that float32 holds: 8 e relative for the
    ratio's gradient (four roundings of its own, three products); e^x - 1 and e^x - 1 - x to 8 e of themselves below 1/4, of their
    parts above.  Out of range: 0 and infinity."""
    x = torch.cat([torch.linspace(-80, 88, 4001), torch.linspace(-0.4, 0.4, 2001), 2.0 ** torch.arange(-40, 0), -2.0 ** torch.arange(-40, 0)]).float()
    n, zero = x.numel(), torch.zeros(x.numel(), device=cuda_device)
    d = x.to(cuda_device)
    cu = torch.arange(n + 1, dtype=torch.int32, device=cuda_device)
    kw = dict(clip_low=1 - 2.0 ** -50, clip_high=0.0, count=1.0)
    _, dl = rpx.policy_loss(d, zero, -torch.ones(n, device=cuda_device), cu, **kw)
    e = torch.exp(x.double())
    held = x < math.log(2.0 ** -50)
    err, r = (dl.double().cpu() - e).abs(), torch.where(held, 0.0, e)
    assert bool((dl.cpu()[held] == 0).all()) and bool((err[~held] <= 8 * E * r[~held]).all()), float((err / e)[~held].max() / E)
    _, dl = rpx.policy_loss(-d, None, zero, cu, ref_logprobs=zero, kl_coef=1.0, kl=3, **kw)
    want, small = -torch.expm1(x.double()), x.abs() < 0.25
    err = (dl.double().cpu() - want).abs()
    assert bool((err <= 8 * E * torch.where(small, want.abs(), e + 1)).all()), float((err / (e + 1)).max() / E)
    for i in [*range(4001, n, 97), *range(0, 4001, 400)]:
        stats, _ = rpx.policy_loss(-d[i:i + 1], None, zero[:1], cu[:2], ref_logprobs=zero[:1], kl_coef=0.0, kl=3, want_grad=False, **kw)
        t = float(x[i])
        want = t * t / 2 * (1 + t / 3 + t * t / 12 + t ** 3 / 60 + t ** 4 / 360) if abs(t) < 0.01 else math.expm1(t) - t
        size = abs(want) if abs(t) < 0.25 else math.exp(t) + 1 + abs(t)
        assert abs(float(stats[2]) - want) <= 8 * E * size + 2.0 ** -126, (t, float(stats[2]), want)
    far = torch.tensor([89.0, 1e30, math.inf, -200.0, -math.inf, math.nan], device=cuda_device)
    z = torch.zeros(6, device=cuda_device)
    _, dl = rpx.policy_loss(-far, None, z, torch.arange(7, dtype=torch.int32, device=cuda_device), ref_logprobs=z, kl_coef=1.0, kl=3, **kw)
    assert dl.tolist()[:5] == [-math.inf, -math.inf, -math.inf, 1.0, 1.0] and math.isnan(float(dl[5]))


@pytest.mark.parametrize("batch", [31, 33, 1024, 1025, 5000])
@pytest.mark.parametrize("ratio,per_token", [("token", True), ("sequence", False)])
def test_sequences_that_end_inside_a_lanes_tokens(cuda_device, batch, ratio, per_token):
    """Lengths of 0 to 9 and a few long ones: weights change inside a lane's four tokens and inside a warp's."""
    gen = np.random.default_rng(batch)
    lens = gen.integers(0, 10, batch)
    lens[:: 29] = 400
    s = make(lens.tolist(), cuda_device, seed=batch, mask=0.7, per_token=per_token)
    kw = dict(ratio=ratio, mean="sequences", kl=3, coef=0.05, dual=3.0)
    check(s, call(s, **kw), **kw)
