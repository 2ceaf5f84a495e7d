"""Further GPU tests of the clipped policy loss: what its first ones do not reach.  Tolerances are those of test_gpu_policy_loss.py."""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx
from test_gpu_policy_loss import E, call, check, formula, make

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ batches as long as the call takes
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("lens", [[700, 320], [3, 1, 90], [5000, 0, 130]], ids=str)
def test_sequences_next_to_31_bits(cuda_device, lens, shift):
    """Sequences that end with the last of 2^31 - 2 tokens, aligned arrays (read by fours) and others."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 28 GB")
    n = 2 ** 31 - 2 - shift
    for ratio in ("token", "sequence"):
        s = make(lens, cuda_device, mask=0.7)
        kw = dict(ratio=ratio, mean="sequences", kl=0, dual=1.5)
        at = n - sum(lens)
        big = dict(s, ref=None, cu=s["cu"] + at)
        for k in ("lp", "old", "mask"):
            room = torch.empty(n + shift, dtype=s[k].dtype, device=cuda_device)[shift:]
            room[at:] = s[k]
            big[k] = room
        out = torch.empty(n + shift, device=cuda_device)[shift:]
        out[at - 1] = 3.0
        status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
        got = call(big, dlogprobs=out, device_status=status, **kw)
        assert int(status) == 0
        check(s, (got[0], got[1][at:]), **kw)
        assert float(out[at - 1]) == 3.0
        del big, room, out, got
        torch.cuda.empty_cache()


# ------------------------------------------------------------------ tokens of no sequence
def _dirty(n, dev):
    """Leaves NaN in the blocks that the allocator hands out next."""
    for _ in range(4):
        rooms = [torch.full((n,), float("nan"), device=dev) for _ in range(3)]
        del rooms


@pytest.mark.parametrize("lens", [[], [30, 41], [0, 0], [3000, 0, 7001], [1] * 900, [8192]], ids=lambda x: f"{len(x)}x{max(x + [0])}")
@pytest.mark.parametrize("lead,tail", [(5, 9), (0, 1), (3, 20000), (129, 0)])
def test_padding_has_a_gradient_of_zero(cuda_device, lens, lead, tail):
    """A gradient that the call allocates itself goes to token_logprobs_backward as it is."""
    s = make(lens, cuda_device, lead=lead, tail=tail, mask=0.7)
    for ratio in ("token", "sequence"):
        n = s["lp"].shape[0]
        _dirty(n, cuda_device)
        got = call(s, coef=0.1, ratio=ratio)
        check(s, got, coef=0.1, ratio=ratio)
        end = n - tail
        assert bool((got[1][:lead] == 0).all()) and bool((got[1][end:] == 0).all())
        out = torch.full_like(s["lp"], 3.0)
        kept = call(s, coef=0.1, ratio=ratio, dlogprobs=out)
        assert torch.equal(out[lead:end], got[1][lead:end]) and torch.equal(kept[0], got[0])
        assert bool((out[:lead] == 3).all()) and bool((out[end:] == 3).all())


def test_padded_training_step(cuda_device):
    """hidden -> log-probs -> loss -> dW with padding behind the sequences: what lies there reaches no weight."""
    gen = torch.Generator().manual_seed(1)
    lens, t, hdim, vocab = [50, 0, 1, 93, 40], 250, 256, 1000
    hidden = torch.randn(t, hdim, generator=gen).bfloat16().to(cuda_device)
    w = (torch.randn(vocab, hdim, generator=gen) / 16).bfloat16().to(cuda_device)
    ids, adv = torch.randint(vocab, (t,), generator=gen).int().to(cuda_device), torch.randn(len(lens), generator=gen).to(cuda_device)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).to(cuda_device)
    lp, lse = rpx.token_logprobs(hidden, w, ids, return_lse=True)
    old = lp - 0.05
    _dirty(t, cuda_device)
    _, dl = rpx.policy_loss(lp, old, adv, cu)
    dh, dw = rpx.token_logprobs_backward(hidden, w, ids, lse, dl, want_dw=True)
    _, dl = rpx.policy_loss(lp, old, adv, cu, dlogprobs=torch.zeros(t, device=cuda_device))
    dh0, dw0 = rpx.token_logprobs_backward(hidden, w, ids, lse, dl, want_dw=True)
    assert torch.equal(dh, dh0) and torch.equal(dw, dw0) and bool((dh[sum(lens):] == 0).all())


# ------------------------------------------------------------------ ratios whose sum passes float32
@pytest.mark.parametrize("lens", [[4], [4, 1, 7], [3000, 0, 7001]], ids=str)
@pytest.mark.parametrize("mean", ["tokens", "sequences"])
def test_large_ratios_have_a_finite_mean(cuda_device, lens, mean):
    """Ratios up to 3.3e38: four of them add up to more than float32 holds, their weighted sum does not.  Differences lie on a grid
    of 2^-10, so that they are exact; the advantage holds nothing (below 0, no dual clip) or makes the term small."""
    s = make(lens, cuda_device, seed=2)
    gen = torch.Generator().manual_seed(3)
    d = torch.round((88.0 + 0.7 * torch.rand(sum(lens), generator=gen)) * 1024) / 1024
    s["lp"], s["old"], s["ref"] = -torch.ones(sum(lens), device=cuda_device), -1 - d.to(cuda_device), None
    for size in (1.0, 2.0 ** -20):
        s["adv"] = -size * torch.ones(len(lens), device=cuda_device)
        got = call(s, mean=mean)
        assert bool(got[0].isfinite().all()) and float(got[0][4]) > 1.6e38
        check(s, got, mean=mean)


# ------------------------------------------------------------------ many short sequences
@pytest.mark.parametrize("lens", [[1] * 8192, [2] * 4096, [0, 3] * 2000, [100] + [0] * 20000, [64] * 32, [64] * 33, [2048], [2049], [0] * 31 + [2048], [0] * 32 + [2048]],
                         ids=lambda x: f"{len(x)}x{x[-1]}")
@pytest.mark.parametrize("ratio,mean", [("token", "sequences"), ("sequence", "tokens"), ("sequence", "sequences")])
@pytest.mark.parametrize("mask", [None, 0.6])
def test_few_tokens_in_many_sequences(cuda_device, lens, ratio, mean, mask):
    """Few tokens in many sequences, and both sides of what one launch of one CTA takes."""
    s = make(lens, cuda_device, mask=mask, lead=1, tail=2)
    kw = dict(ratio=ratio, mean=mean, kl=3, coef=0.05, dual=2.0)
    got = call(s, **kw)
    check(s, got, **kw)
    again = call(s, **kw)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_time_of_few_tokens_in_many_sequences(cuda_device):
    """One-token sequences are spread over the GPU: three times as long as the same tokens in eight sequences, and by no
    means eight times (one CTA that goes through them all takes seventeen times as long)."""
    n = 8192
    lp = -torch.rand(n, device=cuda_device)
    mask = torch.ones(n, dtype=torch.bool, device=cuda_device)
    times = []
    for batch in (8, n):
        cu = (torch.arange(batch + 1, device=cuda_device) * (n // batch)).int()
        adv = torch.ones(batch, device=cuda_device)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            rpx.policy_loss(lp, lp, adv, cu, mask=mask)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for _ in range(20):
                    rpx.policy_loss(lp, lp, adv, cu, mask=mask)
        best = float("inf")
        for _ in range(10):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            graph.replay()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
    assert times[1] <= 8 * times[0], times


# ------------------------------------------------------------------ exponentials down to where they end
def test_ratios_down_to_the_smallest(cuda_device):
    """The ratio alone (advantage 1, one token a sequence, weight 1), in units of e = 2^-24: x = n ln 2 + g leaves g off by e / 2,
    q = e^g - 1 is a sum of g and less than 0.07, rounded once (e / 2), 1 + q once more (e), scaling by 2^n is exact, all against
    1 + q >= 0.7: 3 e, and e each for the products with the advantage and the weight.  0 below 2^-125.5; 2^-126 holds 2 roundings
    of the border."""
    x = torch.cat([torch.linspace(-87.5, -86.5, 4001), torch.linspace(-87.0, -40.0, 4001), torch.tensor([-88.0, -100.0, -1e30, -float("inf")])]).float()
    n = x.numel()
    cu = torch.arange(n + 1, dtype=torch.int32, device=cuda_device)
    stats, dl = rpx.policy_loss(x.to(cuda_device), torch.zeros(n, device=cuda_device), torch.ones(n, device=cuda_device), cu, count=1.0)
    r = -dl.double().cpu()
    want = torch.exp(x.double())
    border = -125.5 * np.log(2.0)
    over, under = x.double() > border + 2.0 ** -16, x.double() < border - 2.0 ** -16
    assert bool(((r - want).abs() <= 5 * E * want)[over].all()), float(((r - want).abs() / want)[over].max() / E)
    assert bool((r[under] == 0).all()) and int(under.sum()) > 2000
