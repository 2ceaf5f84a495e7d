"""Further GPU tests of group attention: what its first ones do not reach.

Tolerances as in test_gpu_group_attn.py (u = 2^-8, e = 2^-24, S the largest scale * sum |q_i k_i| of a row), with the 2^-16 of two
bf16 terms of P for every batch: out  u |out| + (2 w + 2^-13) sum p |v|,  w = (d + 4) e S + 2^-21 + 2^-16.
"""
import numpy as np
import pytest
import torch

import paper_2608_14498_b200 as rpx
from test_gpu_group_attn import GROUPS, call, exact, make

pytestmark = pytest.mark.gpu


def check_two_terms(s, got, softmax_scale=None):
    out, lse, pv, big = exact(s, softmax_scale)
    score = (s["q"].shape[2] + 4) * 2.0 ** -24 * big
    tol = 2.0 ** -8 * out.abs() + (2 * (score + 2.0 ** -21 + 2.0 ** -16) + 2.0 ** -13)[..., None] * pv
    err = (got[0].double() - out).abs()
    assert bool((err <= tol).all()), (float(err.max()), float((err / tol).max()))
    assert bool(((got[1].double() - lse).abs() <= score + 2.0 ** -13 + 2.0 ** -20 * lse.abs()).all())


# ------------------------------------------------------------------ probabilities in two terms, whoever else is in the group
MANY_ROWS = {
    "members": [(1500, [(1 + i % 40, 1) for i in range(70)])],
    "tokens": [(900, [(40, 5), (600, 13), (5, 5), (200, 1)] * 3)],
    "chunks": [(500, [(150, 150), (260, 200)]), (0, [(1029, 129)])],
}


@pytest.mark.parametrize("name", list(MANY_ROWS))
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (16, 2, 64), (64, 1, 128), (5, 5, 128)])
@pytest.mark.parametrize("factor", [1.0, 6.0])
def test_probabilities_are_two_terms_in_large_blocks(cuda_device, name, hq, hkv, d, factor):
    """Groups and chunks of far more rows than a block holds; with the larger scale few keys hold a row's weight, so that a
    probability of one bf16 term is off by many times the tolerance."""
    scale = factor * d ** -0.5
    s = make(MANY_ROWS[name], hq, hkv, d, cuda_device)
    got = call(s, softmax_scale=scale)
    assert int(s["status"]) == 0
    check_two_terms(s, got, scale)


def test_bounds_do_not_change_how_exact_a_row_is(cuda_device):
    s = make([(700, [(20 + i, 1) for i in range(6)]), (0, [(400, 1)])], 28, 4, 128, cuda_device)
    for bounds in (dict(), dict(max_group_tokens=40), dict(max_group_tokens=5000), dict(max_q_len=300)):
        check_two_terms(s, call(s, softmax_scale=0.6, **bounds), 0.6)


@pytest.mark.parametrize("hq,hkv,d", [(65, 1, 128), (112, 1, 128), (222, 2, 128), (224, 2, 128), (128, 1, 64), (381, 3, 64), (200, 2, 64)])
def test_more_heads_to_a_kv_head_than_a_block_has_rows(cuda_device, hq, hkv, d):
    """Parts of a KV head's query heads, equal and unequal ones, with several tokens, shared keys, cut segments and rows of nobody."""
    for groups in (MANY_ROWS["tokens"], [(700, [(1 + i % 40, 1) for i in range(9)]), (0, [(3000, 2), (1, 1)])], [(0, [(129, 129)])], [(0, [(20000, 1)])]):
        s = make(groups, hq, hkv, d, cuda_device, fill=float("nan"))
        out = torch.full((s["q"].shape[0] + 2, hq, d), 9.0, dtype=torch.bfloat16, device=cuda_device)
        got = call(s, out=out[1:-1])
        assert int(s["status"]) == 0
        check_two_terms(s, got)
        assert bool((out[[0, -1]] == 9).all())
        again = call(s)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


# ------------------------------------------------------------------ caches as long as kv_lens can say
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("kv", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 100])
def test_lengths_next_to_31_bits(cuda_device, kv, shared):
    """Every key weighs 1 but the last, whose weight is about that of all others together; behind it lies one that would outweigh
    everything.  All pages but the last are the same one.  Sums of ones are exact (2^24 a piece), so the outputs are off by their
    own rounding, 2^-8, and the joins', 2^-16 at most."""
    hq, d, n, last, far = 2, 64, 5, 5.0, 400.0
    seqs = 4 if shared else 1
    pages = -(-kv // 16)
    kc, vc = torch.zeros(2, 1, 16, d, device=cuda_device).bfloat16(), torch.ones(2, 1, 16, d, device=cuda_device).bfloat16()
    place = (kv - 1) % 16
    kc[1, 0, place, 0], vc[1, 0, place] = 172.0, last  # score 21.5
    kc[1, 0, place + 1:, 0], vc[1, 0, place + 1:] = far, 100.0
    table = torch.zeros(seqs, pages, dtype=torch.int32, device=cuda_device)
    table[:, -1] = 1
    whole = (kv - n) // 16 * 16 if shared else 0
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=cuda_device)
    s = dict(q=torch.ones(seqs * n, hq, d, device=cuda_device).bfloat16(), kc=kc, vc=vc, table=table, cu=n * torch.arange(seqs + 1, dtype=torch.int32, device=cuda_device),
             kv=i32(*[kv] * seqs), cg=i32(0, seqs), shared=i32(whole), max_q=n, max_group=seqs * n, max_kv=kv, status=i32(0))
    out, lse = call(s)
    assert int(s["status"]) == 0
    ones, w = float(kv - 1), np.exp(21.5)
    want = torch.ones(n, dtype=torch.float64)
    want[-1] = (ones + last * w) / (ones + w)
    total = torch.tensor([np.log(kv - n + 1.0 + i) for i in range(n - 1)] + [np.log(ones + w)])
    err = (out.double().cpu().view(seqs, n, hq, d) - want[None, :, None, None]).abs()
    assert bool((err <= (2.0 ** -8 + 2.0 ** -16) * want[None, :, None, None]).all()), err.amax((0, 2, 3))
    assert bool(((lse.double().cpu().view(seqs, n, hq) - total[None, :, None]).abs() <= 2.0 ** -13 + 2.0 ** -20 * total[-1]).all())


# ------------------------------------------------------------------ the SM budget
@pytest.mark.parametrize("name", ["mixed", "several_tokens"])
def test_the_sm_budget_changes_no_bit(cuda_device, name):
    s = make(GROUPS[name], 28, 4, 128, cuda_device)
    want = call(s)
    before = rpx.get_sm_budget()
    try:
        for budget in (1, 40, 147):
            rpx.set_sm_budget(budget)
            got = call(s)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    finally:
        rpx.set_sm_budget(before)


# ------------------------------------------------------------------ data that does not fit, in every form
BATCH = [(500, [(40, 1), (60, 1), (5, 1)]), (64, [(9, 2), (200, 2)])]
FORMS = {"bf16": (torch.bfloat16, 0), "f32": (torch.float32, 0), "bf16_many": (torch.bfloat16, 1100)}  # type, sequences of their own behind


def _longer(s, key, first, behind):
    """The first entries of one of the batch's arrays replaced; those of the sequences behind as they were."""
    old = s[key]
    s[key] = torch.cat([torch.tensor(first, dtype=torch.int32, device=old.device), old[len(first):]])
    assert s[key].shape == old.shape and behind == old.shape[0] - len(first)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("change", [
    dict(cg=[0, 3, 2]), dict(cg=[-1, 3, 5]), dict(cg=[1, 0, 5]), dict(cg=[0, 2 ** 31 - 1, 5]), dict(cg=[0, -2 ** 31, 5]),
    dict(cg=[2 ** 31 - 1] * 3), dict(cg=[2 ** 31 - 20, 2 ** 31 - 20, 2 ** 31 - 1]), dict(cg=[-2 ** 31, -1, 5]), dict(shared=[-1, 64]),
    dict(shared=[505, 64]), dict(shared=[500, 2 ** 31 - 1]), dict(max_group=2), dict(shared=[500, 72])], ids=str)
def test_groups_that_do_not_fit(cuda_device, form, change):
    """Reported, and computed without sharing: whatever the form, the rows are right."""
    dtype, behind = FORMS[form]
    s = make(BATCH + [(0, [(3 + i % 30, 1)]) for i in range(behind)], 8, 2, 128, cuda_device, dtype=dtype)
    good = call(s)
    assert int(s["status"]) == 0
    for k, v in change.items():
        if k == "max_group":
            s[k] = v
        else:
            _longer(s, k, v, behind)
    got = call(s)
    assert int(s["status"]) == -8
    if dtype == torch.float32:
        assert torch.equal(got[0], good[0]) and torch.equal(got[1], good[1])  # (never shared)
    else:
        check_two_terms(s, got)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("change,gone", [
    (dict(kv=[540, 560, 505, 1, 264]), [3, 4]), (dict(kv=[540, -1, 505, 73, 264]), [1]), (dict(kv=[540, 2 ** 31 - 1, 505, 73, 264]), [1]),
    (dict(max_q=1), [3, 4, 5, 6]), (dict(cu=[-1, 1, 2, 3, 5, 7]), [0]), (dict(cu=[0, 1, 2, 3, 5, 8]), [5, 6, 7])], ids=str)
def test_sequences_that_do_not_fit(cuda_device, form, change, gone):
    """Reported, and their rows left as they were; the other sequences' are right."""
    dtype, behind = FORMS[form]
    s = make(BATCH + [(0, [(3 + i % 30, 1)]) for i in range(behind)], 8, 2, 128, cuda_device, dtype=dtype)
    want, lse = exact(s)[:2]
    for k, v in change.items():
        if k == "max_q":
            s[k] = v
        else:
            _longer(s, k, v, behind)
    out = torch.full_like(s["q"], 9.0)
    out_lse = torch.full(s["q"].shape[:2], 9.0, device=cuda_device)
    call(s, out=out, lse=out_lse)
    assert int(s["status"]) == -8
    gone = [t for t in gone if t < out.shape[0]]  # (the last sequence of the batch takes the next one's token, or one that is not there)
    kept = [t for t in range(out.shape[0]) if t not in gone]
    assert bool((out[gone] == 9).all()) and bool((out_lse[gone] == 9).all())
    # values of size 1 to 4: rounded to 2^-8 of themselves, and 2^-13 of the terms' sum
    assert float((out[kept].double() - want[kept]).abs().max()) < 0.03 and float((out_lse[kept].double() - lse[kept]).abs().max()) < 1e-3


def test_bounds_of_later_groups_that_do_not_fit(cuda_device):
    """More groups than the plan takes at a time, the later ones' bounds far behind the last sequence but ascending."""
    for first, last in ((1024, 2 ** 31 - 1), (1024, 2 ** 31 - 500), (1, 2 ** 31 - 1), (1030, 2 ** 31 - 1)):
        s = make(BATCH + [(0, [(3 + i % 30, 1)]) for i in range(1100)], 8, 2, 128, cuda_device)
        s["cg"][first:] = last
        got = call(s)
        assert int(s["status"]) == -8
        check_two_terms(s, got)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("cu", [[0, 1, 2, 3, 2, 7], [0, 1, 2 ** 31 - 1, 3, 5, 7], [0, 1, -2 ** 31, 3, 5, 7], [2, 1, 2, 3, 5, 7]], ids=str)
def test_offsets_that_run_backwards(cuda_device, form, cu):
    """A row's sequence is looked up in offsets that ascend: where they do not, no row is written."""
    dtype, behind = FORMS[form]
    s = make(BATCH + [(0, [(3 + i % 30, 1)]) for i in range(behind)], 8, 2, 128, cuda_device, dtype=dtype)
    _longer(s, "cu", cu, behind)
    out = torch.full_like(s["q"], 9.0)
    lse = torch.full(s["q"].shape[:2], 9.0, device=cuda_device)
    call(s, out=out, lse=lse)
    assert int(s["status"]) == -8
    assert bool((out == 9).all()) and bool((lse == 9).all())


# ------------------------------------------------------------------ outputs in the place of the queries
@pytest.mark.parametrize("name", list(GROUPS))
@pytest.mark.parametrize("hq,hkv,d,dtype", [(28, 4, 128, torch.bfloat16), (4, 2, 64, torch.bfloat16), (100, 1, 128, torch.bfloat16), (4, 2, 64, torch.float32)])
def test_outputs_in_the_place_of_the_queries(cuda_device, name, hq, hkv, d, dtype):
    s = make(GROUPS[name], hq, hkv, d, cuda_device, dtype=dtype)
    want = call(s)
    for _ in range(3):
        q = s["q"].clone()
        got = call(s, q=q, out=q)
        assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(got[1], want[1])
    assert int(s["status"]) == 0
