"""Attention over the 8-bit cache: what values, scales and weights far apart may do to a result, and what may not."""
import numpy as np
import pytest
import torch

import heads_ref as R
from paper_2604_03957_amd import binding as B
from test_gpu_cache_attention import DEV, filled, i32, run

pytestmark = pytest.mark.gpu
f16, b16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("lens,new,max_len", [([300, 260], [1, 1], 300), ([300, 260], [1, 1], 30000), ([300, 260], [40, 3], 300), ([1300, 260], [90, 3], 1300),
                                              ([300, 260], [40, 3], 30000)])
def test_a_scale_that_nobody_names_decides_no_bit(lens, new, max_len):
    """Scales of a block that no sequence has, near the others' and far from them, where the first block of a sequence, or one in
    its middle, is not there: the same bits."""
    g = torch.Generator().manual_seed(26)
    ref, table = filled(g, lens, 2, 64, 64)
    table[0, 1], table[1, 0] = -1, 1 << 30
    free = [p for p in range(ref.sizes[0]) if p not in table.tolist()[0] + table.tolist()[1]]
    swap = table.clone()  # block 0 is one of those that nobody names
    swap[table == 0] = free[0]
    for x in (ref.k, ref.v, ref.ke, ref.ve):
        x[free[0]] = x[0]
    Q = torch.randn((sum(new), 4, 64), generator=g).half()
    got = []
    for fill in (1.0, *(2.0 ** e for e in range(-12, 0)), float("nan"), float("inf"), 0.0, -1.0, 2.0 ** 100):
        cache = ref.device(B)
        for i in (2, 3):
            cache.tensors[i][0] = fill
        got.append(run(ref, cache, Q, swap, lens, new, 4, 0.125, True, 0, max_len=max_len))
    want = R.attention(ref, Q.double().numpy(), swap, lens, got[0][2], 2, 0.125, True, 0)
    assert (np.abs(got[0][0].double().cpu().numpy() - want[0]) <= R.attention_tolerance(f16, *want)[0]).all()
    for other in got[1:]:
        assert torch.equal(other[0], got[0][0]) and torch.equal(other[1], got[0][1])
