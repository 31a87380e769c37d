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


def layout(M, heads, kv, dim, batch, max_new, max_len, window=0):
    """How the work of a call is laid out, from the size of its parts: each row whole, in parts, or in equal shares of all steps."""
    max_new = min(max_new, M)
    if window and window < max_len:
        max_len = min(max_len, window + max_new + 62)
    n = B.cache_attention_workspace_bytes(M=M, heads=heads, kv_heads=kv, dim=dim, batch=batch, max_new=max_new, max_len=max_len)
    rows = max_new * (heads // kv)
    tile = 16 if rows <= 16 else 32 if rows <= 32 and dim < 256 else 128
    counts = (batch + 1) * 4 if tile < 128 else 16 << 9
    shares = [-(-(((2 * tile) << log2) * (dim + 2) * 4 + counts) // 256) * 256 for log2 in (range(11) if tile < 128 else (9,))]
    return "whole" if n == 0 else "shares" if n in shares else "parts"


@pytest.mark.parametrize("lens,new,heads,kv,dim,max_len,how", [
    ([5], [1], 2, 1, 64, 5, "whole"), ([700, 1], [1, 1], 20, 1, 128, 700, "whole"), ([2000], [1], 2, 1, 64, 2000, "parts"), ([2000], [1], 2, 1, 256, 131072, "parts"),
    ([40, 0, 130] * 100, [1, 0, 1] * 100, 4, 2, 64, 20000, "shares"), ([70, 300], [70, 150], 2, 1, 64, 300, "whole"), ([1100], [1100], 1, 1, 128, 1100, "parts"),
    ([1100, 200], [100, 200], 2, 1, 256, 9000, "parts"), ([90, 700, 0] * 18, [70, 70, 0] * 18, 6, 3, 64, 5000, "shares")])
def test_values_at_the_end_of_the_range_stay_finite(lens, new, heads, kv, dim, max_len, how):
    """fp16's largest value is held as 256 * 2^8, which fp16 does not have, and infinities as more: an average of them is fp16's
    largest, as reading gives it."""
    batch, total = len(lens), sum(lens)
    assert layout(sum(new), heads, kv, dim, batch, max(new), max_len) == how
    g = torch.Generator().manual_seed(31)
    wide = -(-max_len // 64)
    need = [-(-n // 64) for n in lens]
    at = np.concatenate(([0], np.cumsum(need)))
    table = torch.full((batch, wide), -1, dtype=torch.int32)
    for b in range(batch):
        table[b, :need[b]] = torch.arange(at[b], at[b + 1])
    ref = R.Cache(int(at[-1]), kv, 64, dim)
    K, V = (torch.randn((total, kv, dim), generator=g).half() for _ in range(2))
    V[:, :, 0], V[:, :, 1], V[:, :, 2], V[:, :, 3] = 65504.0, -65504.0, float("inf"), -float("inf")
    ref.write(K.double().numpy(), V.double().numpy(), table, lens, np.concatenate(([0], np.cumsum(lens))), batch)
    Q = torch.randn((sum(new), heads, dim), generator=g).half()
    out, lse, _ = run(ref, ref.device(B), Q, table, lens, new, heads, dim ** -0.5, True, 0, max_len=max_len)
    out = out.cpu()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for c, v in enumerate((65504.0, -65504.0, 65504.0, -65504.0)):
        assert (out[:, :, c] == v).all()
    assert (out[:, :, 4:].abs() < 65504).all()
