"""Host-only checks of the calls around a prompt group's step (norm + rotation + append, group attention, policy loss): refusals
before any launch, legal no-ops, the wrappers' own checks."""
import ctypes

import pytest
import torch

from paper_2608_14498_b200 import binding as B

P = 0x1000  # an aligned address that nothing is launched with


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14498_b200 import build

    build.build()
    return B.load_library()


def cache(k=P, v=P, blocks=8, size=16, table=P, stride=4):
    return B.KvCache(k, v, blocks, size, table, stride)


# ------------------------------------------------------------------ norm + rotation + append
def append(lib, desc=None, q=P, k=P, v=P, qs=512, ks=256, vs=256, wq=P, wk=P, pos=P, ps=16, inv=P, n=16, cu=P, lens=P, batch=2,
           max_append=8, c=None, qo=P, qos=512):
    desc = B.RopeDesc(4, 2, 128, 128, 1, None, 1e-6, B.RPX_BF16) if desc is None else desc
    return lib.rpx_qk_norm_rope_append(ctypes.byref(desc) if desc else None, q, k, v, qs, ks, vs, wq, wk, pos, ps, inv, n, cu, lens,
                                       batch, max_append, ctypes.byref(cache() if c is None else c) if c is not False else None, qo,
                                       qos, None, None)


def test_append_refusals(lib):
    assert append(lib, desc=False) == -1
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(inv=None), dict(qo=None), dict(cu=None), dict(lens=None), dict(c=False),
                dict(wq=None), dict(c=cache(k=None)), dict(c=cache(table=None))):
        assert append(lib, **bad) == -1, bad
    for bad in (dict(qs=504), dict(ks=128), dict(vs=128), dict(qos=504), dict(ps=15), dict(n=-1), dict(batch=-1), dict(max_append=-1),
                dict(c=cache(size=32)), dict(c=cache(blocks=0)), dict(c=cache(stride=0)),
                dict(desc=B.RopeDesc(4, 2, 96, 64, 1, None, 1e-6, 0)), dict(desc=B.RopeDesc(4, 2, 128, 136, 1, None, 1e-6, 0))):
        assert append(lib, **bad) == -2, bad
    assert append(lib, desc=B.RopeDesc(4, 2, 128, 128, 1, None, 1e-6, 3)) == -3
    for bad in (dict(qs=516), dict(vs=260), dict(q=P + 8), dict(v=P + 2), dict(qo=P + 4), dict(c=cache(v=P + 8))):
        assert append(lib, **bad) == -4, bad
    for empty in (dict(n=0), dict(batch=0), dict(max_append=0)):
        assert append(lib, **empty) == 0, empty
    assert append(lib, n=0, q=None, k=None, v=None, c=cache(k=None, v=None, table=None)) == 0


# ------------------------------------------------------------------ group attention
def group(lib, desc=None, q=P, qs=512, cu=P, kv=P, batch=2, total=2, max_q=1, max_kv=100, cg=P, shared=P, groups=1, max_group=2, c=None,
          out=P, ws=P, ws_bytes=1 << 40):
    desc = B.AttnDesc(4, 2, 128, 0.0, B.RPX_BF16) if desc is None else desc
    return lib.rpx_group_attn(ctypes.byref(desc) if desc else None, q, qs, cu, kv, batch, total, max_q, max_kv, cg, shared, groups,
                              max_group, ctypes.byref(cache() if c is None else c) if c is not False else None, out, None, ws, ws_bytes,
                              None, None)


def test_group_refusals(lib):
    assert group(lib, desc=False) == -1
    for bad in (dict(q=None), dict(cu=None), dict(kv=None), dict(cg=None), dict(shared=None), dict(c=False), dict(out=None),
                dict(c=cache(v=None))):
        assert group(lib, **bad) == -1, bad
    for bad in (dict(qs=504), dict(batch=-1), dict(total=-1), dict(total=2 ** 31 - 1), dict(max_q=-1), dict(max_kv=-1), dict(groups=-1),
                dict(max_group=-1), dict(c=cache(size=8)), dict(c=cache(blocks=2 ** 32)), dict(desc=B.AttnDesc(4, 3, 128, 0.0, 0)),
                dict(desc=B.AttnDesc(4, 2, 80, 0.0, 0)), dict(desc=B.AttnDesc(258, 2, 64, 0.0, 0)), dict(desc=B.AttnDesc(0, 2, 64, 0.0, 0))):
        assert group(lib, **bad) == -2, bad
    assert group(lib, desc=B.AttnDesc(226, 2, 128, 0.0, 0)) == -2  # 113 heads a KV head of 128 values
    assert group(lib, desc=B.AttnDesc(4, 2, 128, 0.0, 7)) == -3
    for bad in (dict(qs=516), dict(q=P + 8), dict(out=P + 2), dict(c=cache(k=P + 8))):
        assert group(lib, **bad) == -4, bad
    need = B.group_attn_workspace_bytes(4, 2, 128, B.RPX_BF16, 2, 2, 1, 1, 2)
    if need:
        assert group(lib, ws=None) == -5 and group(lib, ws_bytes=need - 1) == -5
        assert group(lib, ws=P + 16, ws_bytes=need) == -4
    for empty in (dict(batch=0), dict(total=0), dict(max_q=0)):
        assert group(lib, **empty) == 0, empty
    assert group(lib, total=0, batch=0, q=None, c=cache(k=None, v=None, table=None)) == 0


def test_group_workspace_of_what_is_refused(lib):
    for a in ((4, 3, 128, 0, 2, 2, 1, 1, 2), (4, 0, 128, 0, 2, 2, 1, 1, 2), (258, 2, 64, 0, 2, 2, 1, 1, 2), (4, 2, 128, 0, -1, 2, 1, 1, 2),
              (4, 2, 128, 0, 2, -2, 1, 1, 2), (4, 2, 128, 0, 2, 2, -1, 1, 2), (4, 2, 128, 0, 2, 2, 1, 0, 2), (4, 2, 128, 0, 2, 2, 1, 1, -2)):
        assert B.group_attn_workspace_bytes(*a) == 0, a


# ------------------------------------------------------------------ policy loss
def policy(lib, ratio=0, mean=1, kl=3, per_token=0, low=0.2, high=0.2, dual=0.0, coef=0.1, count=0.0, lp=P, old=P, ref=P, adv=P, mask=P,
           cu=P, batch=2, n=16, up=None, stats=P, dl=P, ws=P, ws_bytes=1 << 30, desc=True):
    d = B.PolicyDesc(ratio, mean, kl, per_token, low, high, dual, coef, count)
    return lib.rpx_policy_loss(ctypes.byref(d) if desc else None, lp, old, ref, adv, mask, cu, batch, n, up, stats, dl, ws, ws_bytes,
                               None, None)


def test_policy_refusals(lib):
    nan = float("nan")
    assert policy(lib, desc=False) == -1
    for bad in (dict(ratio=2), dict(ratio=-1), dict(mean=2), dict(kl=4), dict(kl=-1), dict(per_token=2), dict(ratio=1, per_token=1),
                dict(low=1.0), dict(low=-0.1), dict(low=nan), dict(high=-0.1), dict(high=nan), dict(dual=1.0), dict(dual=-2.0), dict(dual=nan),
                dict(coef=nan), dict(count=-1.0), dict(count=nan), dict(batch=-1), dict(n=-1), dict(n=2 ** 31 - 1)):
        assert policy(lib, **bad) == -2, bad
    for bad in (dict(lp=None), dict(ref=None), dict(adv=None), dict(cu=None), dict(stats=None)):
        assert policy(lib, **bad) == -1, bad
    assert policy(lib, ws=None) == -5 and policy(lib, ws_bytes=8) == -5
    for bad in (dict(ws=P + 16), dict(lp=P + 2), dict(dl=P + 1), dict(cu=P + 2)):
        assert policy(lib, **bad) == -4, bad


def test_policy_wrapper_checks():
    n, b = 6, 2
    lp, adv, cu = torch.zeros(n), torch.zeros(b), torch.tensor([0, 2, 6], dtype=torch.int32)

    def make(**kw):
        a = dict(logprobs=lp, old_logprobs=lp, advantages=adv, cu_seqlens=cu)
        a.update(kw)
        return B.policy_loss.__wrapped__(**a)

    for bad in (dict(logprobs=lp.double()), dict(old_logprobs=lp[:5]), dict(ref_logprobs=torch.zeros(n, 1)), dict(advantages=torch.zeros(3)),
                dict(advantages=torch.zeros(n, 2)), dict(advantages=adv.half()), dict(mask=torch.ones(n)), dict(mask=torch.ones(5, dtype=torch.bool)),
                dict(ratio="group"), dict(mean="token"), dict(stats=torch.zeros(5)), dict(upstream=torch.zeros(2)),
                dict(logprobs=torch.zeros(2 * n)[::2]), dict(dlogprobs=torch.zeros(n + 1))):
        with pytest.raises(ValueError):
            make(**bad)
    with pytest.raises(TypeError):
        make(cu_seqlens=cu.long())


def test_append_and_group_wrapper_checks():
    bf = torch.bfloat16
    pools = (torch.zeros(3, 2, 16, 64, dtype=bf), torch.zeros(3, 2, 16, 64, dtype=bf), torch.zeros(2, 2, dtype=torch.int32))
    q, k = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)

    def make(**kw):
        a = dict(q=q, k=k, v=k, positions=i32(0, 1, 2), inv_freq=torch.ones(32), cu_append=i32(0, 1, 3), cached_lens=i32(0, 0), max_append=2,
                 cache=pools)
        a.update(kw)
        return B.qk_norm_rope_append.__wrapped__(**a)

    for bad in (dict(v=k[:2]), dict(v=k.float()), dict(k=torch.zeros(3, 1, 64, dtype=bf), v=torch.zeros(3, 1, 64, dtype=bf)), dict(cu_append=i32(0, 1)),
                dict(positions=i32(0, 1)), dict(positions=None, pair_axis=[0] * 32), dict(max_append=-1), dict(max_append=2 ** 31),
                dict(cu_append=i32(0, 1, 2, 3), cached_lens=i32(0, 0, 0)), dict(q_out=q.float()),
                dict(cache=(pools[0], pools[1][:2], pools[2]))):
        with pytest.raises(ValueError):
            make(**bad)
    for bad in (dict(positions=torch.zeros(3)), dict(cached_lens=torch.zeros(2)), dict(cu_append=torch.zeros(3)), dict(k=k.float(), v=k.float())):
        with pytest.raises(TypeError):
            make(**bad)

    def attn(**kw):
        a = dict(q=q, cu_seqlens_q=i32(0, 1, 3), kv_lens=i32(4, 5), cu_groups=i32(0, 2), shared_lens=i32(0), max_q_len=2, max_group_tokens=3,
                 max_kv_len=5, cache=pools)
        a.update(kw)
        return B.group_attn.__wrapped__(**a)

    for bad in (dict(q=q[0]), dict(q=torch.zeros(3, 4, 128, dtype=bf)), dict(cu_seqlens_q=i32(0, 3)), dict(cu_groups=i32(0)),
                dict(out=q[:2]), dict(out=q.float()), dict(lse=torch.zeros(3, 3)), dict(lse=torch.zeros(3, 4).double()), dict(max_q_len=-1),
                dict(max_kv_len=2 ** 31), dict(cu_seqlens_q=i32(0, 1, 2, 3), kv_lens=i32(1, 1, 1)), dict(cache=(pools[0], pools[1][:2], pools[2]))):
        with pytest.raises(ValueError):
            attn(**bad)
    for bad in (dict(kv_lens=torch.zeros(2)), dict(shared_lens=torch.zeros(1)), dict(q=q.half())):
        with pytest.raises(TypeError):
            attn(**bad)
