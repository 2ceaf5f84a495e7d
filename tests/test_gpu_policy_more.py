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
