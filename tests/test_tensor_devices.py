"""Calls around the cache check what only the binding can see before anything is launched: that all tensors are on one device
(kernels take bare pointers, and index tensors are often built on the host), strides of single tokens, bounds beyond 32 bits."""
import inspect

import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx
from paper_2608_14498_b200 import binding as B


def arguments(dev):
    """Every call with all of its tensors, optional ones among them, as {name: (function, keyword arguments)}."""
    def i32(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=dev)

    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device=dev)

    def f32(*shape):
        return torch.zeros(shape, device=dev)

    ws = torch.zeros(16 << 20, dtype=torch.uint8, device=dev)
    pools = [bf16(4, 2, 16, 64), bf16(4, 2, 16, 64)]
    status = i32(1)
    rope = dict(q=bf16(3, 4, 64), k=bf16(3, 2, 64), positions=i32(3), inv_freq=f32(32), q_weight=bf16(64), k_weight=bf16(64))
    pool = dict(block_table=torch.full((3, 4), -1, dtype=torch.int32, device=dev), lens=i32(3), ref_counts=i32(9))
    return {
        "tree_attn": dict(q=bf16(3, 4, 64), k=bf16(3, 2, 64), v=bf16(3, 2, 64), cu_seqlens_tree=i32(2), parents=i32(3) - 1,
                          cached_lens=i32(1), max_tree_len=3, max_cached_len=16, cache=(*pools, i32(1, 2)), out=bf16(3, 4, 64),
                          lse=f32(3, 4), workspace=ws, device_status=status),
        "qk_norm_rope": dict(**rope, q_out=bf16(3, 4, 64), k_out=bf16(3, 2, 64)),
        "qk_norm_rope_backward": dict(q=rope["q"], k=rope["k"], dq=f32(3, 4, 64), dk=f32(3, 2, 64),
                                      **{n: rope[n] for n in ("positions", "inv_freq", "q_weight", "k_weight")},
                                      dq_in=bf16(3, 4, 64), dk_in=bf16(3, 2, 64), dq_weight=f32(64), dk_weight=f32(64), workspace=ws),
        "pages_free": dict(**pool, rows=i32(1), device_status=status),
        "pages_fork": dict(**pool, src_rows=i32(1) - 1, dst_rows=i32(1), copy_src=i32(1), copy_dst=i32(1), workspace=ws,
                           device_status=status),
        "pages_compact": dict(block_table=pool["block_table"], ref_counts=pool["ref_counts"], table_out=i32(3, 4),
                              ref_counts_out=i32(9), copy_src=i32(4), copy_dst=i32(4), n_live=i32(1), workspace=ws,
                              device_status=status),
        "cache_copy_pages": dict(k_cache=pools[0], v_cache=pools[1], src=i32(1) - 1, dst=i32(1) - 1, device_status=status),
        "cache_append": dict(k=bf16(3, 2, 64), v=bf16(3, 2, 64), cu_append=i32(2), cached_lens=i32(1), max_append=2,
                             cache=(*pools, i32(1, 2)), token_ids=i32(3), device_status=status),
    }


CALLS = sorted(arguments("cpu"))


def moved(args, dev):
    """The arguments with one tensor after the other (but the first) on another device, as (name, arguments)."""
    names = [n for n, x in args.items() if torch.is_tensor(x)]
    for name in names[1:]:
        yield name, {**args, name: args[name].to(dev)}
    if "cache" in args:
        for i in range(3):
            yield f"cache[{i}]", {**args, "cache": tuple(x.to(dev) if i == j else x for j, x in enumerate(args["cache"]))}


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
    # nothing that could be a tensor was left out of this test
    plain = {"stream", "softmax_scale", "return_lse", "pair_axis", "eps", "accumulate_dw", "extra_tokens"}
    assert set(inspect.signature(fn).parameters) - set(args) <= plain


def test_the_check():
    class On:
        def __init__(self, n):
            self.device = n

        def get_device(self):
            return self.device

    B._one_device(On(0), None, On(0), None)
    for others in ((On(-1),), (None, On(0), On(1))):
        with pytest.raises(ValueError):
            B._one_device(On(0), *others)


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_are_refused(cuda_device, name):
    args = arguments(cuda_device)[name]
    getattr(rpx, name)(**args)
    torch.cuda.synchronize()
    for what, bad in moved(args, "cpu"):
        with pytest.raises(ValueError, match="one device"):
            getattr(rpx, name)(**bad)
    torch.cuda.synchronize()


def test_token_strides():
    """The heads of one token are looked at as those of many are: a single decoded token may be a view of anything."""
    x = torch.zeros(1, 8, 128)
    for t, stride in ((x, 1024), (x[:, 2:5], 384), (x[:, :1, :64], 64), (x[:, 3:4], 128), (x[:0, ::2], 512),
                      (torch.zeros(5, 8, 64)[2:3], 512), (torch.zeros(5, 8, 64)[1:4, 2:4], 512)):
        assert B._tok_stride(t) == stride, (t.shape, t.stride())
    for t in (x[:, ::2], x[..., :64], x.transpose(1, 2), x[..., ::2], torch.zeros(5, 8, 64)[2:3, ::2], torch.zeros(5, 8, 64)[:, ::2]):
        with pytest.raises(ValueError):
            B._tok_stride(t)


@pytest.mark.gpu
def test_one_token_with_heads_apart_is_refused(cuda_device):
    args = arguments(cuda_device)
    wide = torch.randn(1, 8, 64, device=cuda_device).bfloat16()
    rope = {n: args["qk_norm_rope"][n] for n in ("inv_freq", "q_weight", "k_weight")}
    pos = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    for q, k in ((wide[:, ::2], wide[:, :2]), (wide[:, :4], wide[:, ::4])):
        with pytest.raises(ValueError):
            rpx.qk_norm_rope(q, k, pos, **rope)
        with pytest.raises(ValueError):
            rpx.tree_attn(q, k, k, pos.new_tensor([0, 1]), pos - 1, pos, 1, 16, args["tree_attn"]["cache"])
    with pytest.raises(ValueError):
        rpx.qk_norm_rope(wide[:, :4], wide[:, :2], pos, **rope, q_out=wide.clone()[:, ::2])
    with pytest.raises(ValueError):
        rpx.cache_append(wide[:, ::4], wide[:, ::4], pos.new_tensor([0, 1]), pos, 1, args["tree_attn"]["cache"])


def test_bounds():
    for x in (0, 7, np.int64(7), np.int32(7), torch.tensor(7), 2 ** 31 - 1):
        assert B._bound(x) == int(x) and type(B._bound(x)) is int
    for x in (-1, 2 ** 31, 2 ** 32 + 5):  # 2^32 + 5 arrived as 5
        with pytest.raises(ValueError):
            B._bound(x)


@pytest.mark.gpu
def test_bounds_of_any_kind(cuda_device):
    args = arguments(cuda_device)
    for name, bounds in (("tree_attn", ("max_tree_len", "max_cached_len")), ("pages_fork", ("extra_tokens",)), ("cache_append", ("max_append",))):
        call = {**args[name], **{b: 3 for b in bounds}}
        for kind in (np.int64, np.int32, torch.tensor):
            getattr(rpx, name)(**{**call, **{b: kind(3) for b in bounds}})
        for b in bounds:
            for bad in (2 ** 32 + 3, -1):
                with pytest.raises(ValueError):
                    getattr(rpx, name)(**{**call, b: bad})
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_keywords_in_any_order(cuda_device, name):
    """Numbers, tuples and None may come before the first tensor."""
    args = arguments(cuda_device)[name]
    late = {n: x for n, x in args.items() if torch.is_tensor(x)}
    early = {n: x for n, x in args.items() if n not in late}
    getattr(rpx, name)(stream=None, **early, **late)
    torch.cuda.synchronize()
