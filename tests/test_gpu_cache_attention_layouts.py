"""Attention over the 8-bit cache in each layout of its work, which the size of its parts tells: tests that reach equal shares of all
steps say so, for many rows and for few, with windows, without rows, and with fewer steps than workgroups."""
import numpy as np
import pytest
import torch

import heads_ref as R
from paper_2604_03957_amd import binding as B
from test_gpu_cache_attention import DEV, check, filled, i32, run
from test_gpu_cache_attention_values import layout

pytestmark = pytest.mark.gpu
f16, b16 = torch.float16, torch.bfloat16


def compact(g, lens, heads, block, dim):
    """A reference cache of as many blocks as the sequences need and two, their tokens written, and its table."""
    need = [-(-n // block) for n in lens]
    order = torch.randperm(sum(need) + 2, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32)
    at = np.concatenate(([0], np.cumsum(need)))
    for b in range(len(lens)):
        table[b, :need[b]] = order[at[b]:at[b + 1]]
    ref = R.Cache(sum(need) + 2, heads, block, dim)
    cu = np.concatenate(([0], np.cumsum(lens)))
    K, V = (torch.randn((int(cu[-1]), heads, dim), generator=g) * torch.exp2(torch.randint(-2, 3, (int(cu[-1]), 1, 1), generator=g).float()) for _ in range(2))
    ref.write(K.half().double().numpy(), V.half().double().numpy(), table, lens, cu, len(lens))
    return ref, table


def padded(seed, lens, new, heads, kv, dim, dtype, how, M, max_new, max_len, causal=True, window=0, block=64):
    """The rows of all sequences and, behind them, rows of none up to M, which max_new may not exceed."""
    assert M >= max(max_new, sum(new))
    assert layout(M, heads, kv, dim, len(lens), max_new, max_len, window) == how
    g = torch.Generator().manual_seed(seed)
    ref, table = compact(g, lens, kv, block, dim)
    Q = torch.randn((M, heads, dim), generator=g).to(dtype)
    got = run(ref, ref.device(B), Q, table, lens, new, heads, dim ** -0.5, causal, window, max_new=max_new, max_len=max_len)
    check(ref, Q, table, lens, new, heads, dim ** -0.5, causal, window, got)
    return got


@pytest.mark.parametrize("lens,new", [([1100], [100]), ([60], [3]), ([64], [64]), ([1], [1]), ([5900], [7])])
@pytest.mark.parametrize("dim,dtype", [(64, f16), (128, b16)])
def test_shares_of_one_sequence(lens, new, dim, dtype):
    """A tile of rows that is many workgroups', and fewer steps than workgroups."""
    padded(61, lens, new, 40, 40, dim, dtype, "shares", 1000, 1000, 6000, block=128)


@pytest.mark.parametrize("batch,heads,kv,dim,M,max_new,max_len,how", [
    (50, 6, 3, 128, 200, 100, 5000, "shares"), (1, 40, 40, 64, 1000, 1000, 6000, "shares"), (2, 2, 1, 64, 50, 50, 20000, "parts"), (2, 2, 1, 256, 50, 50, 20000, "parts"),
    (300, 4, 2, 64, 4, 1, 20000, "shares"), (1030, 2, 1, 128, 8, 1, 20000, "shares"), (40, 4, 2, 64, 300, 300, 300, "whole")])
def test_no_rows_at_all(batch, heads, kv, dim, M, max_new, max_len, how):
    """Dense rows of which no sequence has any are left as they are."""
    assert layout(M, heads, kv, dim, batch, max_new, max_len) == how
    g = torch.Generator().manual_seed(62)
    ref, table = filled(g, [90] * batch, kv, 64, dim)
    Q = torch.randn((M, heads, dim), generator=g).half()
    out, lse, _ = run(ref, ref.device(B), Q, table, [90] * batch, [0] * batch, heads, 0.1, True, 0, max_new=max_new, max_len=max_len)
    assert (out == 33).all() and (lse == 33).all()


@pytest.mark.parametrize("dim,group,dtype,window", [(128, 2, f16, 4100), (64, 3, b16, 4200), (64, 2, f16, 6000), (128, 2, b16, 0)])
def test_shares_of_many_rows_behind_a_window(dim, group, dtype, window):
    """Sequences longer than the window beside shorter and empty ones."""
    g = torch.Generator().manual_seed(dim + group)
    batch, kv, max_new = 52, 3, 70
    lens = [int(torch.randint(0, 40, (1,), generator=g)) * int(torch.randint(0, 5, (1,), generator=g)) for _ in range(batch)]
    lens[0], lens[20], lens[21], lens[51] = 0, 6500, 0, 4300
    new = [int(torch.randint(0, 12, (1,), generator=g)) for _ in range(batch)]
    new[0], new[20], new[21], new[33], new[51] = 3, max_new, 0, 0, max_new
    padded(71 + dim + group, lens, new, kv * group, kv, dim, dtype, "shares", sum(new) + 3, max_new, 9000, window=window)


@pytest.mark.parametrize("batch,kv,group,dim,dtype,window", [(300, 2, 2, 128, f16, 2100), (300, 2, 20, 64, b16, 2100), (520, 1, 1, 256, b16, 2500), (300, 2, 4, 64, f16, 4096), (1030, 1, 1, 64, f16, 2200),
                                                             (300, 2, 2, 128, f16, 0)])
def test_shares_of_few_rows_behind_a_window(batch, kv, group, dim, dtype, window):
    """So many sequences that workgroups share all steps, some longer than the window."""
    g = torch.Generator().manual_seed(batch + window)
    lens = [int(torch.randint(0, 20, (1,), generator=g)) * int(torch.randint(0, 3, (1,), generator=g)) for _ in range(batch)]
    lens[batch // 3], lens[batch // 2], lens[batch - 2] = 5000, 2100, 200
    most = 1 if group > 16 else 2
    new = [min(n, most, 1 + b % 2) for b, n in enumerate(lens)]
    padded(81 + batch, lens, new, kv * group, kv, dim, dtype, "shares", sum(new) + 1, most, 20000, window=window)


@pytest.mark.parametrize("extra,how", [(1, "whole"), (40, "whole"), (700, "whole")])
def test_larger_bounds_on_new_tokens(extra, how):
    """As many dense rows as the bound on a sequence's new tokens: few rows, one tile of many, several."""
    padded(21, [400, 190], [7, 2], 4, 2, 64, f16, how, 800, 7 + extra, 448)


@pytest.mark.parametrize("rows,how", [(8, "few"), (40, "many")])
def test_lengths_and_offsets_outside_their_bounds(rows, how):
    """A length above max_len counts as max_len, one below 0 as 0; offsets are kept inside the rows: each sequence's rows against what
    they are then.  (Row 2 belongs to two sequences: either's result.)"""
    g = torch.Generator().manual_seed(23)
    ref, table = filled(g, [128, 128, 128], 1, 64, 64)
    Q = torch.randn((rows, 2, 64), generator=g).half()
    lens, cu = [10 ** 9, -3, 128], [-5, 3, 2, 1000]
    seq = dict(M=rows, batch=3, max_new=rows, max_len=128)
    out, lse = torch.full((rows, 2, 64), 33.0, dtype=f16, device=DEV), torch.full((rows, 2), 33.0, device=DEV)
    ws = torch.empty(max(256, B.cache_attention_workspace_bytes(heads=2, kv_heads=1, dim=64, **seq)), dtype=torch.uint8, device=DEV)
    B.bwta_cache_attention(ref.device(B), Q.to(DEV), out, lse, table.to(DEV), i32(lens), i32(cu), ws, heads=2, alpha=0.125, **seq)
    torch.cuda.synchronize()
    # sequence 0 has rows 0 to 2, positions 125 to 127; sequence 1 has none (its end is before its beginning); sequence 2 has rows 2 to
    # the last, of as many positions up to 127
    for b, first, last, sure in ((0, 0, 3, slice(0, 2)), (2, 2, rows, slice(3, rows))):
        want = R.attention(ref, Q.double().numpy()[first:last], table[b:b + 1], [128], [0, last - first], 1, 0.125, True, 0)
        tol, tol_lse = R.attention_tolerance(f16, *want)
        at = slice(sure.start - first, sure.stop - first)
        assert (np.abs(out[sure].double().cpu().numpy() - want[0][at]) <= tol[at]).all()
        assert (np.abs(lse[sure].double().cpu().numpy() - want[1][at]) <= tol_lse[at]).all()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
