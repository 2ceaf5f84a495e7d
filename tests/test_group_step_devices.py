"""The calls around a prompt group's step look at every tensor's device before anything is launched, take their arguments in any
order, and do so from another current device's point of view as well as the usual one."""
import inspect

import pytest
import torch

import paper_2608_14498_b200 as rpx
from paper_2608_14498_b200 import binding as B


def arguments(dev):
    def i32(*x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device=dev)

    def f32(*shape):
        return torch.zeros(shape, device=dev)

    ws = torch.zeros(64 << 20, dtype=torch.uint8, device=dev)
    cache = (bf16(4, 2, 16, 64), bf16(4, 2, 16, 64), torch.zeros(1, 2, dtype=torch.int32, device=dev))
    status = i32(0)
    return {
        "qk_norm_rope_append": dict(q=bf16(3, 4, 64), k=bf16(3, 2, 64), v=bf16(3, 2, 64), positions=i32(0, 1, 2), inv_freq=f32(32),
                                    cu_append=i32(0, 3), cached_lens=i32(0), max_append=3, cache=cache, q_weight=bf16(64),
                                    k_weight=bf16(64), q_out=bf16(3, 4, 64), device_status=status),
        "group_attn": dict(q=bf16(3, 4, 64), cu_seqlens_q=i32(0, 3), kv_lens=i32(20), cu_groups=i32(0, 1), shared_lens=i32(16),
                           max_q_len=3, max_group_tokens=3, max_kv_len=20, cache=cache, out=bf16(3, 4, 64), lse=f32(3, 4),
                           workspace=ws, device_status=status),
        "policy_loss": dict(logprobs=f32(3), old_logprobs=f32(3), advantages=f32(1), cu_seqlens=i32(0, 3),
                            mask=torch.ones(3, dtype=torch.bool, device=dev), ref_logprobs=f32(3), upstream=f32(1), stats=f32(6),
                            dlogprobs=f32(3), workspace=ws, device_status=status),
    }


CALLS = sorted(arguments("cpu"))


class Seen(Exception):
    pass


@pytest.mark.parametrize("name", CALLS)
def test_every_tensor_is_looked_at(name, monkeypatch):
    args = arguments("cpu")[name]
    seen = []

    def note(*tensors):
        seen.extend(id(t) for t in tensors)
        raise Seen

    monkeypatch.setattr(B, "_one_device", note)
    fn = getattr(rpx, name).__wrapped__
    with pytest.raises(Seen):
        fn(**args)
    given = [x for x in args.values() if torch.is_tensor(x)] + list(args.get("cache", ()))
    assert {id(t) for t in given} <= set(seen)
    plain = {"stream", "softmax_scale", "return_lse", "pair_axis", "eps", "clip_low", "clip_high", "clip_dual", "kl_coef", "kl", "ratio",
             "mean", "count", "want_grad"}
    assert set(inspect.signature(fn).parameters) - set(args) <= plain  # nothing that could be a tensor was left out


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_are_refused_and_keywords_in_any_order(cuda_device, name):
    args = arguments(cuda_device)[name]
    fn = getattr(rpx, name)
    fn(**args)
    fn(**dict(reversed(args.items())))
    assert int(args["device_status"]) == 0
    for n in [n for n, x in args.items() if torch.is_tensor(x)][1:]:
        with pytest.raises(ValueError, match="one device"):
            fn(**{**args, n: args[n].cpu()})
    if "cache" in args:
        for i in range(3):
            with pytest.raises(ValueError, match="one device"):
                fn(**{**args, "cache": tuple(x.cpu() if i == j else x for j, x in enumerate(args["cache"]))})


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_workspaces_that_are_too_small(cuda_device, name):
    args = arguments(cuda_device)[name]
    if "workspace" not in args:
        pytest.skip("keeps none")
    need = (B.group_attn_workspace_bytes(4, 2, 64, B.RPX_BF16, 3, 1, 1, 3, 3) if name == "group_attn"
            else int(B.load_library().rpx_policy_loss_workspace_bytes(1, 3)))
    if need > 0:
        with pytest.raises(ValueError):
            getattr(rpx, name)(**{**args, "workspace": args["workspace"][:need - 1]})
        with pytest.raises(rpx.RpxError):
            getattr(rpx, name)(**{**args, "workspace": args["workspace"][16:]})
    getattr(rpx, name)(**{**args, "workspace": args["workspace"][:max(need, 256)]})
