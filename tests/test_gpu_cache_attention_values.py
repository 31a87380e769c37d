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


def held(g, n, kv, dim, dtype, nats, big):
    """n tokens of which the 100th rules: its score is `nats` above the others', its value 0 but for the last channel, where it is `big`.
    -> reference cache and table"""
    K, V = torch.randn((n, kv, dim), generator=g) * 0.5, 1.0 + 0.5 * torch.randn((n, kv, dim), generator=g)
    K[:, :, 0], K[100, :, 0], K[100, :, 1] = 0.0, nats, 0.0
    V[100], V[100, :, dim - 1] = 0.0, big
    blocks = -(-n // 64)
    table = torch.randperm(blocks, generator=g).to(torch.int32)[None]
    ref = R.Cache(blocks, kv, 64, dim)
    ref.write(K.to(dtype).double().numpy(), V.to(dtype).double().numpy(), table, [n], [0, n], 1)
    return ref, table


def bounded(k, v, size, q, alpha, dtype):
    """(out, its bound, lse, its bound) of one query over all of a head's n keys and values, size[j] the scale of v[j].  A weight times
    scale is rounded to 2^-11 of itself or 2^-36 of the row's largest; scores are off by ds as everywhere; fp32 sums of 16 keys
    at a time, n / 16 of them, by 2^-24 each; then one rounding."""
    n = len(k)
    s = alpha * (k @ q)
    w = np.exp(s - s.max())
    W = w.sum()
    out = w @ v / W
    ds = float((alpha * (np.abs(k) @ np.abs(q))).max()) * 2.0 ** -16 + 2.0 ** -20
    each = 2.0 ** -11 + 2 * ds + n / 16 * 2.0 ** -24
    small = 2.0 ** -36 * (w * size).max() * (np.abs(v) / size[:, None]).sum(0) / W
    eps = torch.finfo(dtype).eps / 2
    return out, 1.01 * ((w @ np.abs(v)) / W * each + small) + eps * np.abs(out) + eps * float(torch.finfo(dtype).smallest_normal), s.max() + np.log(W), ds + 2.0 ** -19 + n / 16 * 2.0 ** -24


@pytest.mark.parametrize("dtype,nats,big", [(f16, 15.0, 0.0), (f16, 18.0, 64.0), (b16, 26.0, 0.0), (b16, 15.0, 4096.0)])
@pytest.mark.parametrize("n,batch,new,heads,kv,dim,how", [
    (20000, 1, 1, 2, 1, 128, "parts"), (20000, 64, 1, 8, 8, 64, "shares"), (16000, 32, 3, 16, 2, 64, "parts"), (20000, 1, 40, 2, 1, 64, "parts"),
    (16000, 1, 8400, 2, 2, 128, "whole"), (16000, 1, 8400, 8, 4, 64, "whole"), (131072, 1, 17000, 2, 1, 64, "shares"), (30000, 2, 4200, 2, 1, 256, "whole")])
def test_the_tail_behind_a_key_that_rules(n, batch, new, heads, kv, dim, how, dtype, nats, big):
    """A result that many small weights make, next to one that is 2^22 to 2^38 times as large: rows whose keys one wavefront goes over
    alone, and in parts and shares."""
    assert layout(batch * new, heads, kv, dim, batch, new, n) == how
    g = torch.Generator().manual_seed(51)
    ref, table = held(g, n, kv, dim, dtype, nats, big)
    some = torch.zeros((8, dim), dtype=dtype)  # eight queries, all rows and heads have one of them
    some[:, 0], some[:, 1] = 1.0, torch.randn(8, generator=g).to(dtype)
    rows = torch.arange(batch * new) % 8
    Q = some[rows][:, None].expand(-1, heads, -1).contiguous()
    out, lse, _ = run(ref, ref.device(B), Q, table.expand(batch, -1).contiguous(), [n] * batch, [new] * batch, heads, 1.0, False, 0, max_len=n)
    K, V, _ = ref.rows(table, 0, n)
    group = heads // kv
    for h in range(kv):
        for i in range(min(8, batch * new)):
            size = np.repeat(2.0 ** ref.ve[table[0].numpy(), h].astype(float), 64)[:n]
            want, tol, log, tol_log = bounded(K[:, h], V[:, h], size, some[i].double().numpy(), 1.0, dtype)
            mine = (rows == i).to(DEV)
            err = np.abs(out[mine][:, h * group:(h + 1) * group].double().cpu().numpy() - want)
            assert (err <= tol).all(), (h, i, (err / tol).max())
            assert (np.abs(lse[mine][:, h * group:(h + 1) * group].double().cpu().numpy() - log) <= tol_log).all()


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -12, 1.0, 2.0 ** 30])
@pytest.mark.parametrize("batch,new,heads,kv,dim,max_len,how", [(60, 1, 2, 1, 64, 700, "whole"), (20, 1, 4, 2, 128, 3000, "parts"), (300, 1, 4, 2, 64, 20000, "shares"), (140, 140, 1, 1, 64, 700, "whole"),
                                                                (140, 140, 1, 1, 256, 700, "whole"), (3, 70, 2, 1, 128, 5000, "parts"), (52, 70, 6, 3, 64, 5000, "shares")])
def test_log_sums_of_exact_scores_are_rounded_once(batch, new, heads, kv, dim, max_len, how, size):
    """Scores that are whole numbers of bits, so weights and their sums are exact: the logarithm is off by its own rounding, 2^-24 of it,
    and by that of a fraction's logarithm and of ln 2, less than 2^-22 together, whatever the values' scale is."""
    alpha = np.float32(1) / np.float32(1.44269504088896340736)
    assert np.float32(alpha * np.float32(1.44269504088896340736)) == 1
    assert layout(batch * new, heads, kv, dim, batch, new, max_len) == how
    g = torch.Generator().manual_seed(71)
    n = 700
    blocks = -(-n // 64)
    K, V = torch.zeros((n, kv, dim)), torch.randn((n, kv, dim), generator=g) * size
    K[:, :, 0] = -torch.randint(0, 13, (n, kv), generator=g).float()
    table = torch.randperm(blocks, generator=g).to(torch.int32)[None]
    ref = R.Cache(blocks, kv, 64, dim)
    ref.write(K.double().numpy(), V.bfloat16().double().numpy(), table, [n], [0, n], 1)
    lens = [int(torch.randint(1, n + 1, (1,), generator=g)) for _ in range(batch)]
    Q = torch.zeros((batch * new, heads, dim), dtype=b16)
    Q[:, :, 0] = 1.0
    wide = torch.cat([table, torch.full((1, -(-max_len // 64) - blocks), -1, dtype=torch.int32)], dim=1) if max_len > n else table
    lse = run(ref, ref.device(B), Q, wide.expand(batch, -1).contiguous(), lens, [new] * batch, heads, float(alpha), False, 0, max_len=max_len)[1].double().cpu().numpy()
    sums = np.cumsum(2.0 ** K[:, :, 0].double().numpy(), axis=0)  # exact
    want = np.log(sums[np.array(lens) - 1])[:, None, :, None]  # the same for a sequence's rows and a key head's queries
    got = lse.reshape(batch, new, kv, heads // kv)
    assert (np.abs(got - want) <= 2.0 ** -23 * np.abs(want) + 2.0 ** -22).all(), np.abs(got - want).max()
