"""The cached step and the policy's step as they are used: prompts stored into the cache, branched, decoded together by groups,
eagerly and from a captured graph; log-probs, their clipped loss, and its gradient down to the LM head.

Tolerances: attention's are those of test_gpu_group_attn.  The LM head's gradients are sums of g W (or g h) with
g = dl (onehot - p): with u = 2^-8, g is rounded to bf16 once (u), the result of bf16 once more (u), and what float32 leaves of
log-probs, loss and sums is far below the third u: 3 u sum |g| |W|.
"""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx
from test_gpu_group_attn import PAGE, call, check, make

pytestmark = pytest.mark.gpu
HQ, HKV, D = 28, 4, 128


class Run:
    """Two prompts in rows 6 and 7, three branches of each in rows 0 .. 5, and beside the cache what every row has stored."""

    def __init__(self, dev, prompts=(45, 130)):
        self.dev, gen = dev, torch.Generator(dev).manual_seed(3)
        self.gen = gen
        self.kc, self.vc = (torch.full((64, HKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device=dev) for _ in range(2))
        self.table = torch.full((8, 12), -1, dtype=torch.int32, device=dev)
        self.lens, self.refs = self.ints([0] * 8), self.ints([0] * 64)
        self.status = self.ints([0])
        self.weight = [torch.rand(D, generator=gen, device=dev).bfloat16() for _ in range(2)]
        self.inv_freq = (10000.0 ** (-torch.arange(D // 2, device=dev, dtype=torch.float64) / (D // 2))).float()
        rpx.pages_fork(self.table, self.lens, self.refs, self.ints([-1, -1]), self.ints([6, 7]), max(prompts), device_status=self.status)
        x, cu = self.tokens(sum(prompts)), self.ints([0, prompts[0], sum(prompts)])
        self.append(x, cu, self.lens[6:], max(prompts), self.table[6:])
        k, v = self.stored(x, torch.cat([torch.arange(n) for n in prompts]))
        self.lens[6:] = self.ints(prompts)
        pairs = rpx.pages_fork(self.table, self.lens, self.refs, self.ints([6, 6, 6, 7, 7, 7]), self.ints(range(6)), 40,
                               device_status=self.status)
        rpx.cache_copy_pages(self.kc, self.vc, *pairs, device_status=self.status)
        rpx.pages_free(self.table, self.lens, self.refs, self.ints([6, 7]), device_status=self.status)
        self.cg, self.shared = self.ints([0, 3, 6]), self.ints(prompts)
        cut = [slice(0, prompts[0])] * 3 + [slice(prompts[0], None)] * 3
        self.k, self.v = [k[c] for c in cut], [v[c] for c in cut]

    def ints(self, x):
        return torch.tensor(list(x), dtype=torch.int32, device=self.dev)

    def tokens(self, n):
        return torch.randn(n, HQ + 2 * HKV, D, generator=self.gen, device=self.dev).bfloat16()

    def append(self, x, cu, lens, most, table, **kw):
        return rpx.qk_norm_rope_append(x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], None, self.inv_freq, cu, lens, most,
                                       (self.kc, self.vc, table), q_weight=self.weight[0], k_weight=self.weight[1],
                                       device_status=self.status, **kw)

    def stored(self, x, places):
        _, k = rpx.qk_norm_rope(x[:, :HQ], x[:, HQ:HQ + HKV], places.int().to(self.dev), self.inv_freq, self.weight[0], self.weight[1])
        return k, x[:, HQ + HKV:].clone()

    def step(self, x, cu, most, group_most, **kw):
        """One step of six rows; the lengths move on."""
        lens = self.lens[:6]
        q = self.append(x, cu, lens, most, self.table[:6], **kw)
        lens += cu[1:] - cu[:-1]
        got = rpx.group_attn(q, cu, lens, self.cg, self.shared, most, group_most, 180, (self.kc, self.vc, self.table[:6]),
                             return_lse=True, device_status=self.status)
        return q, got

    def remember(self, x, news):
        places = torch.cat([torch.arange(n) + len(self.k[i]) for i, n in enumerate(news)])
        k, v = self.stored(x, places)
        at = 0
        for i, n in enumerate(news):
            self.k[i], self.v[i] = torch.cat([self.k[i], k[at:at + n]]), torch.cat([self.v[i], v[at:at + n]])
            at += n

    def expect(self, q, got, news):
        """What the rows have stored, laid into pages of their own, against the definition."""
        kv = [len(k) for k in self.k]
        pages = [-(-n // PAGE) for n in kv]
        kc, vc = (torch.zeros(sum(pages), HKV, PAGE, D, dtype=torch.bfloat16, device=self.dev) for _ in range(2))
        table, at = torch.zeros(6, max(pages), dtype=torch.int32, device=self.dev), 0
        for i, n in enumerate(kv):
            table[i, :pages[i]] = torch.arange(at, at + pages[i])
            for c, x in ((kc, self.k[i]), (vc, self.v[i])):
                flat = torch.zeros(pages[i] * PAGE, HKV, D, dtype=torch.bfloat16, device=self.dev)
                flat[:n] = x
                c[at:at + pages[i]] = flat.view(pages[i], PAGE, HKV, D).transpose(1, 2)
            at += pages[i]
        check(dict(q=q, kc=kc, vc=vc, table=table, host=(kv, list(news)), max_q=max(news), max_group=sum(news[:3]) + sum(news[3:])), got)


@pytest.mark.parametrize("prompts", [(45, 130), (16, 1)])
def test_prompts_branches_and_steps(cuda_device, prompts):
    run = Run(cuda_device, prompts)
    for news in ([1] * 6, [1] * 6, [3, 1, 0, 2, 5, 1], [0, 0, 7, 0, 0, 0], [1] * 6):
        x, cu = run.tokens(sum(news)), run.ints(np.concatenate([[0], np.cumsum(news)]))
        q, got = run.step(x, cu, max(news), max(sum(news[:3]), sum(news[3:])))
        run.remember(x, news)
        run.expect(q, got, news)
    assert int(run.status.item()) == 0


def test_a_captured_step(cuda_device):
    """The step, replayed with other tokens, does what the calls do."""
    run = Run(cuda_device)
    x, cu = run.tokens(6), run.ints(range(7))
    side = torch.cuda.Stream(cuda_device)
    side.wait_stream(torch.cuda.current_stream(cuda_device))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        q, got = run.step(x, cu, 1, 3)
    for i in range(3):
        x.copy_(run.tokens(6))
        before = [t.clone() for t in (run.kc, run.vc, run.lens)]
        graph.replay()
        after = [t.clone() for t in (run.kc, run.vc, run.lens, q, *got)]
        for t, b in zip((run.kc, run.vc, run.lens), before):
            t.copy_(b)
        q2, got2 = run.step(x, cu, 1, 3)
        for a, b in zip(after, (run.kc, run.vc, run.lens, q2, *got2)):
            assert torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8)), i
        run.remember(x, [1] * 6)
        run.expect(q2, got2, [1] * 6)
    assert int(run.status.item()) == 0


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 2, 64), (112, 1, 128), (128, 1, 64)])
@pytest.mark.parametrize("groups", [[(0, [(1 + i % 37, 1)]) for i in range(1500)],
                                    [(i * 29 % 90, [(1 + (3 * i + j) % 21, 1 + (i + j) % 2 if (3 * i + j) % 21 else 1) for j in range(4)])
                                     for i in range(400)],
                                    [(64, [(20 + i % 3, 1) for i in range(1300)])]], ids=["alone", "groups_of_4", "one_group"])
def test_more_than_a_thousand_sequences(cuda_device, groups, hq, hkv, d):
    s = make(groups, hq, hkv, d, cuda_device, fill=float("nan"))
    got = call(s)
    assert int(s["status"].item()) == 0
    check(s, got)


def test_heads_a_kv_head_has_room_for(cuda_device):
    s = make([(20, [(3, 1)])], 113, 1, 128, cuda_device)
    with pytest.raises(rpx.RpxError):
        call(s)


@pytest.mark.parametrize("ratio,mean,kl", [("token", "sequences", 3), ("sequence", "tokens", 2)])
def test_policy_step(cuda_device, ratio, mean, kl):
    """hidden -> log-probs -> loss -> dl -> dhidden, dW; behind the last sequence lie tokens of none."""
    gen = torch.Generator().manual_seed(5)
    lens, t, hdim, vocab, low, high, coef = [50, 0, 1, 93, 40], 190, 256, 1000, 0.2, 0.25, 0.04
    hidden, w = torch.randn(t, hdim, generator=gen).bfloat16(), (torch.randn(vocab, hdim, generator=gen) / 16).bfloat16()
    ids, cu = torch.randint(vocab, (t,), generator=gen).int(), np.concatenate([[0], np.cumsum(lens)])
    mask, adv = torch.rand(t, generator=gen) < 0.8, torch.randn(len(lens), generator=gen)
    h64, w64 = hidden.double().requires_grad_(), w.double().requires_grad_()
    lp64 = torch.log_softmax(h64 @ w64.T, -1).gather(1, ids.long()[:, None])[:, 0]
    steps = torch.tensor([0.0, 0.05, -0.05, 0.1, 0.3, -0.3])  # away from the borders: -0.223 and 0.223
    old = (lp64.detach() - steps[torch.randint(6, (t,), generator=gen)]).float()
    ref = (lp64.detach() + 0.2 * torch.randn(t, generator=gen)).float()
    loss, seqs, total = 0.0, sum(1 for a, b in zip(cu, cu[1:]) if mask[a:b].any()), int(mask[:cu[-1]].sum())
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        at = torch.nonzero(mask[a:b])[:, 0] + a
        if not len(at):
            continue
        d = lp64[at] - old[at].double()
        if ratio == "sequence":
            d = d.mean().expand(len(at))
        r, A = d.exp(), adv[i].double()
        term = torch.maximum(-A * r, -A * r.clamp(1 - low, 1 + high))
        x = ref[at].double() - lp64[at]
        term = term + coef * (x.exp() - 1 - x if kl == 3 else x * x / 2)
        loss = loss + term.sum() / (len(at) * seqs if mean == "sequences" else total)
    loss.backward()
    dev = lambda x: x.to(cuda_device)
    lp, lse = rpx.token_logprobs(dev(hidden), dev(w), dev(ids), return_lse=True)
    stats, dl = rpx.policy_loss(lp, dev(old), dev(adv), dev(torch.tensor(cu, dtype=torch.int32)), mask=dev(mask), ref_logprobs=dev(ref),
                                clip_low=low, clip_high=high, kl_coef=coef, kl=kl, ratio=ratio, mean=mean,
                                dlogprobs=torch.zeros(t, device=cuda_device))
    dh, dw = rpx.token_logprobs_backward(dev(hidden), dev(w), dev(ids), lse, dl, want_dw=True)
    assert abs(float(stats[0]) - float(loss.detach())) <= 2.0 ** -14 * (1 + abs(float(loss.detach()))) and int(stats[5]) == total
    with torch.no_grad():
        g = torch.nn.functional.one_hot(ids.long(), vocab) - torch.softmax(h64 @ w64.T, -1)
        g = (g * dl.double().cpu()[:, None]).abs()
        for got, want, tol in ((dh, h64.grad, g @ w64.abs()), (dw, w64.grad, g.T @ h64.abs())):
            err = (got.double().cpu() - want).abs()
            assert bool((err <= 3 * 2.0 ** -8 * tol + 1e-12).all()), (float(err.max()), float((err / (tol + 1e-12)).max()))
