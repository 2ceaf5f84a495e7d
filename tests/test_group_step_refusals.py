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
