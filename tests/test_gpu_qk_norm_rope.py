"""GPU parity of the query/key norm + rotation pass and its backward against the formulas in 64 bits.

Tolerances, per value, with e the output type's half step (bf16 2^-8, float32 2^-24, relative to the value):
  forward   e |out| + 2^-18 (|y_a| + |y_b|): a turned value is a difference of two products of the pair's normed values; each
            carries the norm's factor (sum of 128 squares in a tree of 16 + 3 steps, rsqrt to 2 ulp), the cosine (angle to
            2^-23, sincospi to 2 ulp) and four roundings, together under 40 * 2^-24 < 2^-18
  dx        e |dx| + 2^-17 r (G |w| + |u| mean(G |w| |u|)) with G = |g_a| + |g_b| of the pair that arrives: the same
            relative error on both products, and once more on the row's dot product
  dw        2^-15 sum(G |u|): sums of at most 256 terms in a row, 2^-16, on top of the terms' own 2^-18 each
"""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def make(tokens, hq, hkv, d, rot, axes, dtype, norm, dev, seed=0, far=100000, extra=0):
    gen = torch.Generator().manual_seed(seed)
    rows = hq + 2 * hkv
    scale = torch.exp(0.7 * torch.randn(tokens, rows, 1, generator=gen))
    qkv = torch.zeros(tokens, rows * d + extra)
    qkv[:, :rows * d] = (torch.randn(tokens, rows, d, generator=gen) * scale).reshape(tokens, rows * d)
    qkv = qkv.to(DT[dtype]).to(dev)
    q = qkv[:, :hq * d].unflatten(1, (hq, d))
    k = qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    pos = torch.randint(-far, far, (axes, tokens), generator=gen, dtype=torch.int32).to(dev)
    n = rot // 2
    inv = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().to(dev)
    axis = torch.randint(0, axes, (n,), generator=gen).tolist()
    w = [(1 + 0.3 * torch.randn(d, generator=gen)).to(DT[dtype]).to(dev) if norm else None for _ in range(2)]
    return q, k, pos, inv, axis, w


def angles(pos, inv, axis):
    a = pos.double().cpu()[axis].t() * inv.double().cpu()  # [T, n]
    return torch.cos(a)[:, None], torch.sin(a)[:, None]


def turn(x, c, s):
    n = c.shape[-1]
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * n:]], -1)


def pair_sum(x, rot):
    """|x_a| + |x_b| of the pair each element belongs to (|x| itself beyond rot)."""
    n = rot // 2
    both = x[..., :n].abs() + x[..., n:rot].abs()
    return torch.cat([both, both, x[..., rot:].abs()], -1)


def ref_forward(x, w, pos, inv, axis, eps):
    x = x.double().cpu()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double().cpu()
    return turn(x, *angles(pos, inv, axis)), pair_sum(x, 2 * len(axis))


def ref_backward(x, dy, w, pos, inv, axis, eps):
    x, dy = x.double().cpu(), dy.double().cpu()
    c, s = angles(pos, inv, axis)
    g, big = turn(dy, c, -s), pair_sum(dy, 2 * len(axis))
    if w is None:
        return g, None, big, None
    w = w.double().cpu()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u = x * r
    dx = r * (g * w - u * (g * w * u).mean(-1, keepdim=True))
    size = r * (big * w.abs() + u.abs() * (big * w.abs() * u.abs()).mean(-1, keepdim=True))
    return dx, (g * u).sum((0, 1)), size, (big * u.abs()).sum((0, 1))


def close(got, ref, tol, what):
    err = (got.double().cpu() - ref).abs()
    bad = err > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err - tol).max()):.3e} over"


SHAPES = [
    # tokens, hq, hkv, d, rot, axes, dtype, norm
    (1, 28, 4, 128, 128, 3, "bf16", True),
    (3, 28, 4, 128, 128, 1, "bf16", False),
    (37, 5, 3, 64, 64, 2, "bf16", True),
    (130, 40, 8, 128, 64, 3, "bf16", True),
    (64, 1, 1, 64, 16, 1, "f32", True),
    (289, 4, 2, 64, 32, 1, "f32", True),
    (77, 12, 4, 128, 48, 8, "f32", True),
    (257, 7, 7, 128, 112, 3, "bf16", True),
    (31, 9, 1, 128, 128, 3, "f32", False),
    (5000, 28, 4, 128, 128, 3, "bf16", True),
]


@pytest.mark.parametrize("tokens,hq,hkv,d,rot,axes,dtype,norm", SHAPES)
def test_forward(cuda_device, tokens, hq, hkv, d, rot, axes, dtype, norm):
    q, k, pos, inv, axis, w = make(tokens, hq, hkv, d, rot, axes, dtype, norm, cuda_device)
    out = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis, eps=1e-5)
    for x, y, wt, name in ((q, out[0], w[0], "q"), (k, out[1], w[1], "k")):
        assert y.dtype == x.dtype and y.shape == x.shape and y.is_contiguous()
        ref, size = ref_forward(x, wt, pos, inv, axis, 1e-5)
        close(y, ref, HALF_STEP[dtype] * ref.abs() + 2.0 ** -18 * size, name)


@pytest.mark.parametrize("tokens,hq,hkv,d,rot,axes,dtype,norm", SHAPES)
def test_backward(cuda_device, tokens, hq, hkv, d, rot, axes, dtype, norm):
    q, k, pos, inv, axis, w = make(tokens, hq, hkv, d, rot, axes, dtype, norm, cuda_device, seed=1)
    gen = torch.Generator().manual_seed(2)
    dq = torch.randn(tokens, hq, d, generator=gen).to(cuda_device)
    dk = torch.randn(tokens, hkv, d, generator=gen).to(cuda_device)
    gq, gk, gwq, gwk = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis, eps=1e-5)
    for x, dy, wt, g, gw, name in ((q, dq, w[0], gq, gwq, "q"), (k, dk, w[1], gk, gwk, "k")):
        dx, dw, size, wsize = ref_backward(x, dy, wt, pos, inv, axis, 1e-5)
        close(g, dx, HALF_STEP[dtype] * dx.abs() + 2.0 ** -17 * size, "d" + name)
        assert (gw is None) == (wt is None)
        if wt is not None:
            close(gw, dw, 2.0 ** -15 * wsize, "dw of " + name)


def test_gradient_against_differences(cuda_device):
    """The backward pass against central differences of the FORWARD call, float32 in 64-bit sums.

    f = sum(out * c); with steps of 2^-6 on one value the difference quotient carries rounding 2^-24 * sqrt(values of a row)
    * |out c| / 2^-6 < 2e-4 of the row's size and a third-derivative term of (2^-6)^2 relative to the row's scale."""
    q, k, pos, inv, axis, w = make(3, 2, 1, 64, 64, 2, "f32", True, cuda_device, seed=3)
    q, k = q.contiguous(), k.contiguous()
    gen = torch.Generator().manual_seed(4)
    cq, ck = torch.randn(q.shape, generator=gen).to(cuda_device), torch.randn(k.shape, generator=gen).to(cuda_device)

    def f(q, k, wq, wk):
        a, b = rpx.qk_norm_rope(q, k, pos, inv, wq, wk, axis)
        return float((a.double() * cq.double()).sum() + (b.double() * ck.double()).sum())

    grads = rpx.qk_norm_rope_backward(q, k, cq, ck, pos, inv, w[0], w[1], axis)
    leaves = [q, k, w[0], w[1]]
    for n, (leaf, g) in enumerate(zip(leaves, grads)):
        for i in (0, 17, leaf.numel() - 1):
            step = 2.0 ** -6
            values = []
            for sign in (1, -1):
                moved = [x.clone() for x in leaves]
                moved[n].view(-1)[i] += sign * step
                values.append(f(*moved))
            got = (values[0] - values[1]) / (2 * step)
            want = float(g.reshape(-1)[i])
            assert abs(got - want) <= 5e-3 * max(1.0, float(g.abs().max())), (n, i, got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(cuda_device, dtype):
    q, k, pos, inv, axis, w = make(6, 4, 2, 128, 128, 1, dtype, True, cuda_device)
    pos.copy_(torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1000003, -1, 0]], dtype=torch.int32))
    out, _ = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    ref, size = ref_forward(q, w[0], pos, inv, axis, 1e-6)
    close(out, ref, HALF_STEP[dtype] * ref.abs() + 2.0 ** -18 * size, "far positions")


def test_one_row_of_positions_for_all_axes(cuda_device):
    q, k, pos, inv, axis, w = make(20, 4, 2, 64, 64, 3, "bf16", True, cuda_device)
    want = rpx.qk_norm_rope(q, k, pos[:1].repeat(3, 1), inv, w[0], w[1], axis)
    got = rpx.qk_norm_rope(q, k, pos[0].expand(3, -1), inv, w[0], w[1], axis)
    also = rpx.qk_norm_rope(q, k, pos[0], inv, w[0], w[1])  # text: one axis
    for x in (got, also):
        assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])


def test_unaligned_float32_rows(cuda_device):
    """float32 tensors that start on 16 bytes only take the narrower accesses and give the same bits."""
    q, k, pos, inv, axis, w = make(30, 4, 2, 64, 64, 1, "f32", True, cuda_device)
    dq, dk = torch.randn(30, 4, 64, device=cuda_device), torch.randn(30, 2, 64, device=cuda_device)
    room = torch.zeros(30 * 4 * 64 + 4, device=cuda_device)
    q2 = room[4:].view(30, 4, 64)
    q2.copy_(q)
    assert q2.data_ptr() % 32 == 16
    q = q.contiguous()
    assert all(torch.equal(a, b) for a, b in zip(rpx.qk_norm_rope(q2, k, pos, inv, w[0], w[1], axis),
                                                 rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)))
    assert all(torch.equal(a, b) for a, b in zip(rpx.qk_norm_rope_backward(q2, k, dq, dk, pos, inv, w[0], w[1], axis),
                                                 rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)))


def test_in_place_strided_and_padded(cuda_device):
    q, k, pos, inv, axis, w = make(50, 6, 2, 128, 96, 3, "bf16", True, cuda_device, extra=24)
    base = q._base if q._base is not None else q
    want = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    storage = base.clone()
    got = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis, q_out=q, k_out=k)
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    rest = slice((6 + 2) * 128, None)
    assert torch.equal(base.view(50, -1)[:, rest], storage.view(50, -1)[:, rest])  # v and the padding stay as they were


def test_rows_do_not_touch_each_other(cuda_device):
    q, k, pos, inv, axis, w = make(9, 6, 2, 128, 128, 3, "bf16", True, cuda_device)
    want = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    bad = q.clone()
    bad[4, 2, 7] = float("nan")
    bad[6, 5, 100] = float("inf")
    got, _ = rpx.qk_norm_rope(bad, k, pos, inv, w[0], w[1], axis)
    keep = torch.ones(9, 6, dtype=torch.bool, device=cuda_device)
    keep[4, 2] = keep[6, 5] = False
    assert torch.equal(got[keep], want[0][keep])
    assert got[4, 2].isnan().all()


def test_zero_rows(cuda_device):
    q, k, pos, inv, axis, w = make(4, 5, 1, 64, 64, 1, "f32", True, cuda_device)
    q = torch.zeros_like(q)
    dq, dk = torch.randn(4, 5, 64, device=cuda_device), torch.randn(4, 1, 64, device=cuda_device)
    out, _ = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis, eps=1e-6)
    assert torch.equal(out, torch.zeros_like(out))
    gq, _, gwq, _ = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis, eps=1e-6)
    dx, _, size, _ = ref_backward(q, dq, w[0], pos, inv, axis, 1e-6)
    close(gq, dx, 2.0 ** -24 * dx.abs() + 2.0 ** -17 * size, "dq of zero rows")
    assert torch.equal(gwq, torch.zeros_like(gwq))


def test_no_tokens(cuda_device):
    q, k, pos, inv, axis, w = make(0, 4, 2, 64, 64, 1, "bf16", True, cuda_device)
    out = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    assert out[0].shape == (0, 4, 64)
    g = rpx.qk_norm_rope_backward(q, k, q.float(), k.float(), pos, inv, w[0], w[1], axis)
    assert torch.equal(g[2], torch.zeros(64, device=cuda_device)) and torch.equal(g[3], torch.zeros(64, device=cuda_device))


def test_weight_gradient_accumulates_and_repeats(cuda_device):
    q, k, pos, inv, axis, w = make(700, 8, 2, 128, 128, 3, "bf16", True, cuda_device)
    dq, dk = torch.randn(700, 8, 128, device=cuda_device), torch.randn(700, 2, 128, device=cuda_device)
    a = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)
    b = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)
    assert all(torch.equal(x, y) for x, y in zip(a, b))  # a fixed order of summation
    hold = [torch.full((128,), 3.0, device=cuda_device) for _ in range(2)]
    rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis, dq_weight=hold[0], dk_weight=hold[1],
                              accumulate_dw=True)
    for h, x in zip(hold, a[2:]):
        # one rounding of the sum against one of each term
        assert float((h.double() - (x.double() + 3.0)).abs().max()) <= 2.0 ** -22 * float(x.abs().max() + 3)


def test_streams_and_graph(cuda_device):
    q, k, pos, inv, axis, w = make(200, 8, 2, 128, 128, 3, "bf16", True, cuda_device)
    dq, dk = torch.randn(200, 8, 128, device=cuda_device), torch.randn(200, 2, 128, device=cuda_device)
    want = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    want_b = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
        g = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)
    for t in (*y, *g):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*y, *g), (*want, *want_b)))


def test_attention_backward_feeds_it(cuda_device):
    """raw q, k -> norm + rotation -> attention -> its backward -> this backward: the gradients of the whole chain against
    64-bit autograd, within 2 % of the largest one (the attention backward's own tolerance is 1 %)."""
    tokens, hq, hkv, d = 150, 4, 2, 128
    q, k, pos, inv, axis, w = make(tokens, hq, hkv, d, d, 3, "bf16", True, cuda_device, far=200)
    gen = torch.Generator().manual_seed(9)
    v = torch.randn(tokens, hkv, d, generator=gen).bfloat16().to(cuda_device)
    dout = torch.randn(tokens, hq, d, generator=gen).bfloat16().to(cuda_device)
    cu = torch.tensor([0, 90, tokens], dtype=torch.int32, device=cuda_device)
    qr, kr = rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)
    out, lse = rpx.prefix_attn(qr, kr, v, cu, 90, return_lse=True)
    dq, dk, _ = rpx.attn_backward(qr, kr, v, out, dout, lse, cu, 90)
    got = rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)

    leaves = [x.double().cpu().requires_grad_() for x in (q, k, w[0], w[1])]
    c, s = angles(pos, inv, axis)

    def one(x, wt):
        return turn(x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * wt, c, s)

    a, b = one(leaves[0], leaves[2]), one(leaves[1], leaves[3]).repeat_interleave(hq // hkv, 1)
    z = torch.einsum("ihd,jhd->hij", a, b) * d ** -0.5
    i = torch.arange(tokens)
    seen = (i[:, None] >= i) & ((i[:, None] < 90) == (i < 90))
    p = torch.softmax(z.masked_fill(~seen, -np.inf), -1)
    o = torch.einsum("hij,jhd->ihd", p, v.double().cpu().repeat_interleave(hq // hkv, 1))
    ref = torch.autograd.grad((o * dout.double().cpu()).sum(), leaves)
    for name, x, y in zip(("dq", "dk", "dwq", "dwk"), got, ref):
        rel = float((x.double().cpu() - y).abs().max() / y.abs().max())
        assert rel <= 2e-2, (name, rel)


@pytest.mark.parametrize("as_kind", [np.array, lambda a: np.array(a, dtype=np.int32), tuple, torch.tensor])
def test_pair_axis_of_any_kind(cuda_device, as_kind):
    """The axes as an array, a tuple or a CPU tensor give the bits that a list gives, both ways."""
    q, k, pos, inv, axis, w = make(20, 4, 2, 64, 64, 3, "bf16", True, cuda_device)
    dq, dk = torch.randn(20, 4, 64, device=cuda_device), torch.randn(20, 2, 64, device=cuda_device)
    assert all(torch.equal(a, b) for a, b in zip(rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], as_kind(axis)),
                                                 rpx.qk_norm_rope(q, k, pos, inv, w[0], w[1], axis)))
    assert all(torch.equal(a, b) for a, b in zip(rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], as_kind(axis)),
                                                 rpx.qk_norm_rope_backward(q, k, dq, dk, pos, inv, w[0], w[1], axis)))
