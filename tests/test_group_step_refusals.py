"""Host-only checks of the calls around a prompt group's step: arguments that ask for what the call would not do."""
import ctypes

import pytest
import torch

from paper_2608_14498_b200 import binding as B


class Reached(Exception):
    """The library's entry point was called."""


@pytest.fixture
def stubbed(monkeypatch):
    class Lib:
        def rpx_policy_loss_workspace_bytes(self, batch, n):
            return 0

        def rpx_policy_loss(self, *args):
            raise Reached

    monkeypatch.setattr(B, "load_library", Lib)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)

    def make(**kw):
        lp = torch.zeros(6)
        a = dict(logprobs=lp, old_logprobs=lp, advantages=torch.zeros(2), cu_seqlens=torch.tensor([0, 2, 6], dtype=torch.int32))
        a.update(kw)
        return B.policy_loss.__wrapped__(**a)
    return make


def test_a_kl_term_without_reference_is_refused(stubbed):
    for bad in (dict(kl_coef=0.1), dict(kl_coef=-1e-3, kl=1), dict(kl_coef=float("nan"), kl=2), dict(kl=4), dict(kl=-1),
                dict(kl=7, ref_logprobs=torch.zeros(6)), dict(kl=5, kl_coef=0.0)):
        with pytest.raises(ValueError):
            stubbed(**bad)
    for good in (dict(), dict(kl=0, kl_coef=0.1), dict(kl=1), dict(kl_coef=0.1, ref_logprobs=torch.zeros(6)), dict(kl=0, ref_logprobs=torch.zeros(6))):
        with pytest.raises(Reached):
            stubbed(**good)


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14498_b200 import build

    build.build()
    return B.load_library()


def test_a_gradient_that_overlaps_another_array_is_refused(lib):
    """Addresses that nothing is launched with: the refusal comes before the device is asked."""
    n, batch = 16, 2
    at = {k: 0x10000 * (i + 1) for i, k in enumerate(("lp", "old", "ref", "adv", "mask", "cu", "up", "stats", "ws", "dl"))}
    size = dict(lp=4 * n, old=4 * n, ref=4 * n, adv=4 * batch, mask=n, cu=4 * (batch + 1), up=4, stats=24, ws=B.load_library().rpx_policy_loss_workspace_bytes(batch, n))

    def policy(kl=3, **kw):
        a = dict(at, **kw)
        d = B.PolicyDesc(0, 1, kl, 0, 0.2, 0.2, 0.0, 0.1, 0.0)
        if torch.cuda.is_available():
            return None  # (these addresses would be launched with)
        return lib.rpx_policy_loss(ctypes.byref(d), a["lp"], a["old"], a["ref"], a["adv"], a["mask"], a["cu"], batch, n, a["up"], a["stats"],
                                   a["dl"], a["ws"], 1 << 20, None, None)

    if torch.cuda.is_available():
        pytest.skip("host-only")
    passed = policy()
    assert passed in (-6, -7)  # no such device
    for k, bytes_ in size.items():
        assert policy(dl=at[k]) == -2, k
        assert policy(dl=at[k] + bytes_ - 4 + bytes_ % 4) == -2, k
        assert policy(dl=at[k] - 4 * n + 4) == -2, k
        assert policy(dl=at[k] + (bytes_ + 3) // 4 * 4) == passed and policy(dl=at[k] - 4 * n) == passed, k
    assert policy(kl=0, dl=at["ref"]) == passed and policy(dl=None) == passed


def test_more_sequences_than_32_bits_can_step_over_are_refused(lib):
    """Loops over sequences go a grid beyond the last one."""
    if torch.cuda.is_available():
        pytest.skip("host-only")
    P, most = 0x1000, 2 ** 31 - 1 - 65536
    cache = B.KvCache(P, P, 8, 16, P, 4)
    for batch in (most + 1, 2 ** 31 - 2, 2 ** 31 - 1):
        d = B.PolicyDesc(0, 1, 0, 0, 0.2, 0.2, 0.0, 0.0, 0.0)
        assert lib.rpx_policy_loss(ctypes.byref(d), P, P, None, P, None, P, batch, 16, None, P, None, P, 1 << 60, None, None) == -2
        d = B.RopeDesc(4, 2, 128, 128, 1, None, 1e-6, B.RPX_BF16)
        assert lib.rpx_qk_norm_rope_append(ctypes.byref(d), P, P, P, 512, 256, 256, P, P, P, 16, P, 16, P, P, batch, 8, ctypes.byref(cache), P, 512,
                                           None, None) == -2
        d = B.AttnDesc(4, 2, 128, 0.0, B.RPX_BF16)
        for b, groups in ((batch, 0), (batch - 5, 5), (2, batch), (batch, batch)):
            assert lib.rpx_group_attn(ctypes.byref(d), P, 512, P, P, b, 2, 1, 100, P, P, groups, 2, ctypes.byref(cache), P, None, P, 1 << 62, None, None) == -2
            assert lib.rpx_group_attn_workspace_bytes(ctypes.byref(d), 2, b, groups, 1, 2) == 0


def test_outputs_across_the_queries_are_refused(lib):
    if torch.cuda.is_available():
        pytest.skip("host-only")
    P, q, t = 0x1000, 0x100000, 3
    cache = B.KvCache(P, P, 8, 16, P, 4)

    def group(out, stride=512, dtype=B.RPX_BF16):
        d = B.AttnDesc(4, 2, 128, 0.0, dtype)
        return lib.rpx_group_attn(ctypes.byref(d), q, stride, P, P, 2, t, 2, 100, P, P, 1, 3, ctypes.byref(cache), out, None, P, 1 << 40, None, None)

    for stride, dtype, size in ((512, B.RPX_BF16, 2), (1536, B.RPX_BF16, 2), (512, B.RPX_F32, 4)):
        end, room = q + (2 * stride + 512) * size, t * 512 * size
        for out in (q + 16, end - 16, q - room + 16) + (() if stride == 512 else (q,)):
            assert group(out, stride, dtype) == -2, (stride, out)
        for out in (end, q - room) + ((q,) if stride == 512 else ()):
            assert group(out, stride, dtype) in (-6, -7), (stride, out)  # no such device
