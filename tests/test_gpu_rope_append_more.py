"""Further GPU tests of norm + rotation with K and V stored on the way: what its first ones do not reach.

Tolerances as in test_gpu_rope_append.py; an angle of a position of 2^31 is off by 2^-21 in 64 bits, which is within its 2^-18.
"""
import pytest
import torch

import paper_2608_14498_b200 as rpx
from test_gpu_rope_append import HALF_STEP, PAGE, call, formula, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,norm,dtype", [(128, True, "bf16"), (64, False, "bf16"), (64, True, "f32")])
@pytest.mark.parametrize("cached", [2 ** 31 - 3, 2 ** 31 - 1, 2 ** 31 - 8, 2 ** 30 + 5])
def test_positions_next_to_31_bits(cuda_device, d, norm, dtype, cached):
    """The slots that cache_append stores into, behind a sequence as long as cached_lens can say (a table row of 2^27 pages)."""
    new = 21
    s = make([4, new], [3, 0], 4, 2, d, d, 1, dtype, norm, cuda_device, spare=8)
    first = (cached // PAGE) - 1
    table = torch.full((2, (cached + new) // PAGE + 2), -1, dtype=torch.int32, device=cuda_device)
    table[0, :4] = s["table"][0, :1]
    pages = torch.randperm(s["kc"].shape[0], dtype=torch.int32)[:5]
    pages[pages == int(s["table"][0, 0])] = -1
    table[1, first:first + 4] = pages[:4].to(cuda_device)
    s["table"], s["lens"] = table, torch.tensor([3, cached], dtype=torch.int32, device=cuda_device)
    kc, vc = s["kc"].clone(), s["vc"].clone()
    q_two, k_two = rpx.qk_norm_rope(s["q"], s["k"], s["pos"], s["inv"], q_weight=s["w"][0], k_weight=s["w"][1], pair_axis=s["axis"], eps=1e-6)
    status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    rpx.cache_append(k_two, s["v"].contiguous(), s["cu"], s["lens"], s["max_new"], (kc, vc, table), device_status=status)
    q = call(s)
    assert torch.equal(q, q_two) and torch.equal(s["kc"], kc) and torch.equal(s["vc"], vc)
    assert int(s["status"]) == int(status)
    # a token's place as its position
    place = torch.cat([3 + torch.arange(4), cached + torch.arange(new)])[None]
    got = call(s, positions=None, pair_axis=None)
    ref, size = formula(s["q"], s["w"][0], place, s["inv"], [0] * (d // 2))
    assert bool(((got.double().cpu() - ref).abs() <= HALF_STEP[got.dtype] * ref.abs() + 2.0 ** -18 * size).all())
