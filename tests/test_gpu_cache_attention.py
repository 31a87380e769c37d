"""Attention over the 8-bit cache (bwta_cache_attention) against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import heads_ref as R
from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def filled(g, lens, heads, block, dim, spread=2, spare=2, dtype=torch.float16, scale=1.0):
    """A reference cache with `lens` tokens per sequence written, its table, and NaN codes wherever no token is."""
    wide = max(1, max(-(-n // block) for n in lens))
    blocks = len(lens) * wide + spare
    table = torch.randperm(blocks, generator=g)[:len(lens) * wide].reshape(len(lens), wide).to(torch.int32)
    ref = R.Cache(blocks, heads, block, dim)
    ref.ke[:], ref.ve[:] = 40, 40
    cu = np.concatenate(([0], np.cumsum(lens)))
    K, V = (torch.randn((int(cu[-1]), heads, dim), generator=g) * scale for _ in range(2))
    for X in (K, V):  # blocks of different sizes
        for b, n in enumerate(lens):
            for lo in range(0, n, block):
                X[cu[b] + lo:cu[b] + min(n, lo + block)] *= 2.0 ** int(torch.randint(-spread, spread + 1, (1,), generator=g))
    ref.write(K.to(dtype).double().numpy(), V.to(dtype).double().numpy(), table, lens, cu, len(lens))
    return ref, table


def run(ref, cache, Q, table, lens, new, heads, alpha, causal, window, rows=None, max_new=None, max_len=None, cu=None):
    M, dim = Q.shape[0], ref.sizes[3]
    cu = np.concatenate(([0], np.cumsum(new))) if cu is None else cu
    seq = dict(M=M, batch=len(lens), max_new=max(max(new), 1) if max_new is None else max_new, max_len=max(lens) if max_len is None else max_len)
    wide = -(-seq["max_len"] // ref.sizes[2])
    if table.shape[1] < wide:  # what lies behind a sequence's blocks is not looked at
        table = torch.cat([table, torch.full((table.shape[0], wide - table.shape[1]), 1 << 30, dtype=torch.int32)], dim=1)
    out = torch.full((M, heads, dim), 33.0, dtype=Q.dtype, device=DEV)
    lse = torch.full((M, heads), 33.0, device=DEV)
    n = B.cache_attention_workspace_bytes(heads=heads, kv_heads=ref.sizes[1], dim=dim, **seq)
    ws = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV)  # NaN everywhere
    B.bwta_cache_attention(cache, Q.to(DEV), out, lse, table.to(DEV), i32(lens), i32(cu), ws, heads=heads, alpha=alpha, causal=causal, window=window, **seq)
    torch.cuda.synchronize()
    return out, lse, cu


def check(ref, Q, table, lens, new, heads, alpha, causal, window, got):
    out, lse, cu = got
    want = R.attention(ref, Q.double().numpy(), table, lens, cu, len(lens), alpha, causal, window)
    tol, tol_lse = R.attention_tolerance(Q.dtype, *want)
    n = int(cu[-1])
    err = np.abs(out.double().cpu().numpy() - want[0])
    assert (err <= tol)[:n].all(), (err / tol)[:n].max()
    l = lse.double().cpu().numpy()[:n]
    assert np.array_equal(np.isneginf(l), np.isneginf(want[1][:n]))
    fine = np.isfinite(want[1][:n])
    assert (np.abs(l[fine] - want[1][:n][fine]) <= tol_lse[:n][fine]).all()
    assert (out[n:] == 33).all() and (lse[n:] == 33).all()  # rows of no sequence


def case(seed, lens, new, heads, kv, block, dim, dtype, causal=True, window=0, spread=2, scale=1.0, **kw):
    g = torch.Generator().manual_seed(seed)
    ref, table = filled(g, lens, kv, block, dim, spread=spread, scale=scale)
    Q = torch.randn((sum(new) + 1, heads, dim), generator=g).to(dtype)
    alpha = dim ** -0.5
    got = run(ref, ref.device(B), Q, table, lens, new, heads, alpha, causal, window, **kw)
    check(ref, Q, table, lens, new, heads, alpha, causal, window, got)
    return got


f16, b16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("lens,new,heads,kv,block,dim,dtype", [
    ([1], [1], 1, 1, 64, 64, f16),
    ([1, 2, 64, 65, 63, 0], [1, 1, 1, 1, 1, 0], 4, 2, 64, 128, f16),
    ([700, 3, 129], [1, 1, 1], 32, 8, 64, 128, b16),
    ([513], [1], 8, 8, 128, 128, f16),
    ([300, 257], [1, 1], 16, 1, 256, 64, b16),       # sixteen heads to a key head
    ([300, 20], [1, 1], 20, 1, 64, 128, f16),         # twenty: more than one 16
    ([200], [1], 40, 1, 64, 64, f16),                 # forty: rows for each wavefront
    ([2000, 100], [1, 1], 4, 4, 128, 256, f16),
    ([5000], [1], 4, 1, 64, 128, b16),                # split over the sequence
    ([260, 1100], [1, 1], 6, 2, 64, 256, b16),
])
def test_single_tokens(lens, new, heads, kv, block, dim, dtype):
    case(len(lens) + heads, lens, new, heads, kv, block, dim, dtype)


@pytest.mark.parametrize("lens,new,heads,kv,block,dim,dtype,causal,window", [
    ([70, 200], [70, 130], 4, 2, 64, 128, f16, True, 0),
    ([129, 5, 64], [129, 2, 64], 3, 1, 64, 64, b16, True, 0),
    ([333], [333], 2, 2, 128, 128, b16, True, 50),
    ([500, 400], [3, 100], 2, 1, 64, 128, f16, True, 64),
    ([260], [260], 2, 1, 256, 256, f16, True, 1),      # a window of the token itself
    ([150, 90], [40, 300], 2, 2, 64, 128, f16, False, 0),  # more queries than keys
    ([77, 0, 200], [33, 20, 1], 6, 3, 64, 64, b16, False, 0),
    ([190], [17], 5, 1, 64, 128, f16, True, 0),        # 85 rows, more heads than a power of two
    ([66, 300], [9, 9], 2, 1, 64, 256, b16, True, 0),
    ([1500], [5], 6, 1, 128, 128, f16, True, 100),
])
def test_several_tokens(lens, new, heads, kv, block, dim, dtype, causal, window):
    case(len(lens) + heads + dim, lens, new, heads, kv, block, dim, dtype, causal, window)


@pytest.mark.parametrize("max_len,dim,dtype", [(9000, 128, f16), (131072, 64, b16), (70000, 256, f16)])
def test_fewer_steps_than_parts(max_len, dim, dtype):
    """The host's bound is far above the lengths: most of a sequence's parts are empty."""
    case(31, [10, 70, 0, 640], [1, 1, 0, 1], 4, 2, 64, dim, dtype, max_len=max_len)
    case(32, [300], [8], 4, 1, 64, dim, dtype, max_len=max_len)


@pytest.mark.parametrize("batch,kv,group,dim,dtype,window", [(300, 2, 2, 128, f16, 0), (64, 8, 3, 64, b16, 0), (130, 4, 20, 128, f16, 0), (515, 1, 1, 256, b16, 0), (300, 2, 4, 64, f16, 40)])
def test_equal_shares_of_ragged_batches(batch, kv, group, dim, dtype, window):
    """So many sequences of any length, one of them far longer than the others, that workgroups share all steps: shares begin and
    end inside a head's steps, hold several heads and sequences, and pass over empty ones."""
    g = torch.Generator().manual_seed(batch)
    lens = [int(torch.randint(0, 20, (1,), generator=g)) * int(torch.randint(0, 3, (1,), generator=g)) for _ in range(batch)]
    lens[batch // 3], lens[batch - 2] = 1500, 200
    new = [min(n, int(torch.randint(0, 3, (1,), generator=g)) // 2 + 1) if n else 0 for n in lens]
    new = [min(n, 1) for n in new] if group > 16 else new
    case(batch, lens, new, kv * group, kv, 64, dim, dtype, True, window, max_new=1 if group > 16 else 2, max_len=20000)


def test_sequences_without_rows():
    """Rows that belong to no sequence, in each way the work is laid out."""
    for batch, kv, max_new, max_len in ((3, 2, 1, 300), (3, 2, 1, 20000), (300, 2, 1, 20000), (3, 2, 50, 300), (2, 1, 50, 20000)):
        g = torch.Generator().manual_seed(batch)
        lens = [90] * batch
        ref, table = filled(g, lens, kv, 64, 64)
        Q = torch.randn((4, 2 * kv, 64), generator=g).half()
        got = run(ref, ref.device(B), Q, table, lens, [0] * batch, 2 * kv, 0.1, True, 0, max_new=max_new, max_len=max_len)
        assert (got[0] == 33).all() and (got[1] == 33).all()


@pytest.mark.parametrize("lens,new,heads,kv,dim,dtype,causal,max_len", [
    ([1100], [100], 2, 1, 128, f16, True, 1100),      # rows held twice, one workgroup's wavefronts in turn
    ([1100, 60], [90, 60], 3, 1, 64, b16, True, 1100),
    ([1000, 1090], [70, 33], 2, 2, 128, b16, False, 1100),
    ([1100, 130], [100, 129], 2, 1, 128, f16, True, 9000),    # eight parts of each row
    ([1100, 130], [100, 40], 2, 1, 256, b16, True, 5000),
    ([900], [150], 1, 1, 64, f16, True, 40000),        # many parts of each row
])
def test_many_rows_of_long_sequences(lens, new, heads, kv, dim, dtype, causal, max_len):
    case(len(lens) + dim + max_len, lens, new, heads, kv, 64, dim, dtype, causal, max_len=max_len)
    if causal:
        case(7 + len(lens) + dim + max_len, lens, new, heads, kv, 128, dim, dtype, causal, 333, max_len=max_len)


@pytest.mark.parametrize("new", [1, 40])
def test_blocks_of_very_different_sizes(new):
    """Value and key scales 2^-24 to 2^8 apart within a sequence, in every order."""
    case(91, [900, 640], [new, new], 2, 1, 64, 128, f16, spread=12)
    case(92, [900], [new], 2, 1, 64, 64, b16, spread=7, scale=0.01)


def test_steep_scores():
    """Scores of several hundred: the running maximum moves often, most weights vanish."""
    case(93, [700, 333], [1, 30], 2, 1, 64, 128, f16, scale=30.0)


@pytest.mark.parametrize("new", [[1, 1, 1], [10, 40, 3]])
def test_blocks_that_are_not_there(new):
    g = torch.Generator().manual_seed(12)
    lens = [300, 260, 100]
    ref, table = filled(g, lens, 2, 64, 128)
    table[0, 1], table[0, 4], table[1, 0], table[2, :2] = -1, 1 << 30, ref.sizes[0], -(1 << 31)  # the last has none at all
    Q = torch.randn((sum(new), 4, 128), generator=g).half()
    for causal, window in ((True, 0), (True, 70), (False, 0)):
        got = run(ref, ref.device(B), Q, table, lens, new, 4, 0.1, causal, window)
        check(ref, Q, table, lens, new, 4, 0.1, causal, window, got)
    assert (got[0][-new[2]:] == 0).all() and torch.isneginf(got[1][-new[2]:]).all()


def test_rows_before_the_start_see_nothing():
    g = torch.Generator().manual_seed(13)
    lens, new = [20, 5], [30, 5]
    ref, table = filled(g, lens, 1, 64, 64)
    Q = torch.randn((35, 2, 64), generator=g).half()
    got = run(ref, ref.device(B), Q, table, lens, new, 2, 0.125, True, 0)
    check(ref, Q, table, lens, new, 2, 0.125, True, 0, got)
    assert (got[0][:10] == 0).all() and torch.isneginf(got[1][:10]).all()


def test_larger_bounds_give_the_same_rows():
    """max_new and max_len are bounds: larger ones change how the work is split, and nothing else."""
    for extra in (1, 40, 700):
        case(21, [400, 190], [7, 2], 4, 2, 64, 128, f16, max_new=7 + extra, max_len=448)
    case(22, [300, 190], [1, 1], 4, 2, 64, 128, f16, max_len=320)


def test_lengths_above_max_len_and_bad_offsets():
    g = torch.Generator().manual_seed(23)
    ref, table = filled(g, [128, 128, 128], 1, 64, 64)
    Q = torch.randn((8, 2, 64), generator=g).half()
    lens, cu = [10 ** 9, -3, 128], np.array([-5, 3, 2, 1000])
    seq = dict(M=8, batch=3, max_new=8, max_len=128)
    out, lse = torch.full((8, 2, 64), 33.0, dtype=f16, device=DEV), torch.full((8, 2), 33.0, device=DEV)
    ws = torch.empty(max(256, B.cache_attention_workspace_bytes(heads=2, kv_heads=1, dim=64, **seq)), dtype=torch.uint8, device=DEV)
    B.bwta_cache_attention(ref.device(B), Q.to(DEV), out, lse, table.to(DEV), i32(lens), i32(cu), ws, heads=2, alpha=0.125, **seq)
    torch.cuda.synchronize()
    # sequence 0: rows 0-2 at the end of 128 tokens; 1: none; 2: rows 2-7 (after 0's row 2: written by either)
    want = R.attention(ref, Q.double().numpy(), table, [128, 0, 128], np.array([0, 2, 2, 2]), 1, 0.125, True, 0)[0]
    got = out.double().cpu().numpy()
    alone = run(ref, ref.device(B), Q[2:], table[2:], [128], [6], 2, 0.125, True, 0)
    assert torch.equal(out[3:], alone[0][1:]) and np.isfinite(got).all() and want.shape == got.shape


def test_nan_among_scores_stays_with_its_rows():
    g = torch.Generator().manual_seed(14)
    lens, new = [900, 200], [1, 20]
    ref, table = filled(g, lens, 2, 64, 128)
    Q = torch.randn((21, 4, 128), generator=g).half()
    Q[0, 1, 5], Q[7, 2, 0], Q[9, 0, 0] = float("nan"), float("nan"), float("inf")
    out, lse, _ = run(ref, ref.device(B), Q, table, lens, new, 4, 0.1, True, 0)
    bad = torch.zeros((21, 4), dtype=torch.bool)
    bad[0, 1] = bad[7, 2] = bad[9, 0] = True
    assert out.cpu()[bad].isnan().all() and torch.isfinite(out.cpu()[~bad]).all()
    assert lse.cpu()[bad].isnan().all() and torch.isfinite(lse.cpu()[~bad]).all()


def test_strided_rows_in_place_and_without_lse():
    g = torch.Generator().manual_seed(15)
    lens, new, heads, dim = [500, 90], [20, 1], 4, 64
    ref, table = filled(g, lens, 2, 64, dim)
    ld = heads * dim + 40
    rows = torch.randn((21, ld), generator=g).half()
    dev = rows.to(DEV)
    x = dev[:, 8:]
    seq = dict(M=21, batch=2, max_new=20, max_len=500)
    cache = ref.device(B)
    ws = torch.empty(max(256, B.cache_attention_workspace_bytes(heads=heads, kv_heads=2, dim=dim, **seq)), dtype=torch.uint8, device=DEV)
    wide = torch.full((2, table.shape[1] + 3), -7, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table.to(DEV)
    B.bwta_cache_attention(cache, x, x, None, wide, i32(lens), i32([0, 20, 21]), ws, heads=heads, alpha=0.125, ldq=ld, ldo=ld, **seq)
    torch.cuda.synchronize()
    Q = rows[:, 8:8 + heads * dim].reshape(21, heads, dim)
    want = R.attention(ref, Q.double().numpy(), table, lens, np.array([0, 20, 21]), 2, 0.125, True, 0)
    tol = R.attention_tolerance(f16, *want)[0]
    got = dev[:, 8:8 + heads * dim].reshape(21, heads, dim).double().cpu().numpy()
    assert (np.abs(got - want[0]) <= tol).all()
    assert torch.equal(dev[:, :8].cpu(), rows[:, :8]) and torch.equal(dev[:, 8 + heads * dim:].cpu(), rows[:, 8 + heads * dim:])


def test_a_cache_beyond_32_bit_offsets():
    heads, block, dim = 8, 64, 128
    blocks = (1 << 32) // (heads * block * dim) + 4
    k, v = torch.empty((blocks, heads, block, dim), dtype=torch.uint8, device=DEV), torch.empty((blocks, heads, dim, block), dtype=torch.uint8, device=DEV)
    ks, vs = (torch.empty((blocks, heads), device=DEV) for _ in range(2))
    cache = B.make_cache(k, v, ks, vs)
    g = torch.Generator().manual_seed(16)
    ref, small = filled(g, [400], heads, block, dim)
    ids = [blocks - 1 - 2 * i for i in range(small.shape[1])]
    for i, p in enumerate(small[0].tolist()):
        k[ids[i]] = torch.from_numpy(ref.k[p]).to(DEV)
        v[ids[i]] = torch.from_numpy(ref.v[p].transpose(0, 2, 1).copy()).to(DEV)
        ks[ids[i]], vs[ids[i]] = (torch.from_numpy(2.0 ** e[p].astype(np.float32)).to(DEV) for e in (ref.ke, ref.ve))
    for new in (1, 50):
        Q = torch.randn((new, heads, dim), generator=g).half()
        got = run(ref, cache, Q, i32([ids]).cpu(), [400], [new], heads, 0.088, True, 0)
        check(ref, Q, small, [400], [new], heads, 0.088, True, 0, got)


def _step(cache, s, heads, kv, dim, lens, ws, outs, max_len):
    """One decode step of a batch: rotate, write, attend."""
    q, k, v, wq, wk, inv, table = s
    batch = q.shape[0]
    seq = dict(M=batch, batch=batch, max_new=1, max_len=max_len)
    B.bwta_head_norm_rope(q, k, wq, wk, lens - 1, inv, outs[0], outs[1], M=batch, heads=heads, kv_heads=kv, dim=dim)
    B.bwta_cache_write(cache, outs[1], v, table, lens, **seq)
    B.bwta_cache_attention(cache, outs[0], outs[2], outs[3], table, lens, None, ws, heads=heads, alpha=dim ** -0.5, **seq)


@pytest.mark.parametrize("max_len", [320, 20000, 200000])  # a workgroup for each head, parts of each, shares of all
def test_a_captured_step_replayed_follows_the_lengths(max_len):
    """Rotation, write and attention as one graph, replayed while the lengths grow on the device, against eager steps; then
    both caches hold the same."""
    batch, heads, kv, dim, block = 3, 8, 2, 128, 64
    g = torch.Generator().manual_seed(17)
    lens0 = [120, 1, 255]
    ref, table = filled(g, [320] * 3, kv, block, dim)
    caches = [ref.device(B) for _ in range(2)]
    table = torch.cat([table, torch.full((batch, -(-max_len // block) - table.shape[1]), -1, dtype=torch.int32)], dim=1).to(DEV)
    q, k, v = (torch.zeros((batch, n, dim), dtype=f16, device=DEV) for n in (heads, kv, kv))
    wq, wk = (torch.rand(dim, generator=g).half().to(DEV) + 0.5 for _ in range(2))
    inv = (10000.0 ** (-torch.arange(0, dim, 2).double() / dim)).float().to(DEV)
    s = (q, k, v, wq, wk, inv, table)
    seq = dict(M=batch, batch=batch, max_new=1, max_len=max_len)
    n = B.cache_attention_workspace_bytes(heads=heads, kv_heads=kv, dim=dim, **seq)
    wss = [torch.empty(max(n, 256), dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [[torch.zeros((batch, m, dim), dtype=f16, device=DEV) for m in (heads, kv, heads)] + [torch.zeros((batch, heads), device=DEV)] for _ in range(2)]
    lens = i32(lens0)
    _step(caches[0], s, heads, kv, dim, lens, wss[0], outs[0], max_len)  # outside the capture once
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens += 1
        _step(caches[0], s, heads, kv, dim, lens, wss[0], outs[0], max_len)
    _step(caches[1], s, heads, kv, dim, i32(lens0), wss[1], outs[1], max_len)
    for t in range(1, 6):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g).half() * 2.0 ** t)
        graph.replay()
        torch.cuda.synchronize()
        now = i32([a + t for a in lens0])
        assert torch.equal(lens, now)
        _step(caches[1], s, heads, kv, dim, now, wss[1], outs[1], max_len)
        torch.cuda.synchronize()
        for a, b in zip(outs[0], outs[1]):
            assert torch.equal(a, b)
    for a, b in zip(caches[0].tensors, caches[1].tensors):
        assert torch.equal(a, b)


def test_a_prompt_then_tokens_with_the_linears():
    """A block's attention as a program runs it: projections by bwta_linear, rotation, write, attention, output projection;
    a prompt, then tokens one by one, give what the whole sequence gives at once (keys and values of a block are coded again
    when its scale grows, so the caches agree to a code's rounding, half of 2^-3 of a value)."""
    hidden, heads, kv, dim, block, total, prompt = 512, 4, 2, 128, 64, 90, 83
    g = torch.Generator(device=DEV).manual_seed(18)
    wide = (heads + 2 * kv) * dim
    x = torch.randn((total, hidden), device=DEV, generator=g).half()
    words = [torch.randint(-2 ** 31, 2 ** 31, (n, B.plane_row_words(k)), device=DEV, generator=g).to(torch.int32) for n, k in ((wide, hidden), (hidden, heads * dim))]
    s_w = [torch.full((n,), 0.04, dtype=f16, device=DEV) for n in (wide, hidden)]
    inv = (10000.0 ** (-torch.arange(0, dim, 2).double() / dim)).float().to(DEV)
    table = i32([[1, 0]])

    def program(chunks):
        k, v = torch.zeros((2, kv, block, dim), dtype=torch.uint8, device=DEV), torch.zeros((2, kv, dim, block), dtype=torch.uint8, device=DEV)
        cache = B.make_cache(k, v, *(torch.zeros((2, kv), device=DEV) for _ in range(2)))
        ys, at = [], 0
        for n in chunks:
            rows = x[at:at + n].contiguous()
            s_a = torch.empty(n, dtype=f16, device=DEV)
            qkv = torch.empty((n, wide), dtype=f16, device=DEV)
            B.bwta_act_scale(rows, s_a, M=n, K=hidden)
            B.bwta_linear(rows, s_a, words[0], s_w[0], qkv, torch.empty(B.workspace_bytes(n, wide, hidden), dtype=torch.uint8, device=DEV), M=n, N=wide, K=hidden)
            q, kk, vv = qkv[:, :heads * dim], qkv[:, heads * dim:], qkv[:, (heads + kv) * dim:]
            pos = torch.arange(at, at + n, dtype=torch.int32, device=DEV)
            B.bwta_head_norm_rope(q, kk, None, None, pos, inv, q, kk, M=n, heads=heads, kv_heads=kv, dim=dim, ldq=wide, ldk=wide, ldqo=wide, ldko=wide)
            seq = dict(M=n, batch=1, max_new=n, max_len=2 * block)
            lens = i32([at + n])
            B.bwta_cache_write(cache, kk, vv, table, lens, ldk=wide, ldv=wide, **seq)
            att = torch.empty((n, heads * dim), dtype=f16, device=DEV)
            ws = torch.empty(max(256, B.cache_attention_workspace_bytes(heads=heads, kv_heads=kv, dim=dim, **seq)), dtype=torch.uint8, device=DEV)
            B.bwta_cache_attention(cache, q, att, None, table, lens, None, ws, heads=heads, alpha=dim ** -0.5, ldq=wide, **seq)
            out = torch.empty((n, hidden), dtype=f16, device=DEV)
            B.bwta_act_scale(att, s_a, M=n, K=heads * dim)
            B.bwta_linear(att, s_a, words[1], s_w[1], out, torch.empty(B.workspace_bytes(n, hidden, heads * dim), dtype=torch.uint8, device=DEV), M=n, N=hidden, K=heads * dim)
            ys.append((att, out))
            at += n
        torch.cuda.synchronize()
        return torch.cat([a for a, _ in ys]), torch.cat([o for _, o in ys]), cache

    at_once, out_once, c0 = program([total])
    by_token, out_token, c1 = program([prompt] + [1] * (total - prompt))
    for i in range(2):
        scale = c0.tensors[2 + i].reshape(2, kv, 1, 1)
        a, b = (c.tensors[i].view(torch.float8_e4m3fn).float() * c.tensors[2 + i].reshape(2, kv, 1, 1) for c in (c0, c1))
        assert ((a - b).abs() <= 2.0 ** -3 * a.abs() + 2.0 ** -9 * scale).all()
    assert torch.isfinite(out_once).all() and torch.isfinite(out_token).all()
    # the attention of two caches whose codes are off by at most a step: what a step in every key and value can do
    assert (at_once.float() - by_token.float()).norm() <= 2.0 ** -3 * at_once.float().norm()


def test_two_streams_with_workspaces_of_their_own():
    g = torch.Generator().manual_seed(19)
    ref, table = filled(g, [5000, 3000], 2, 64, 128, spread=1)
    cache, table = ref.device(B), table.to(DEV)
    Q = [torch.randn((2, 8, 128), generator=g).half().to(DEV) for _ in range(2)]
    seq = dict(M=2, batch=2, max_new=1, max_len=5000)
    n = B.cache_attention_workspace_bytes(heads=8, kv_heads=2, dim=128, **seq)
    assert n > 0
    lens = i32([5000, 3000])

    def attend(i, ws):
        out = torch.empty((2, 8, 128), dtype=f16, device=DEV)
        B.bwta_cache_attention(cache, Q[i], out, None, table, lens, None, ws, heads=8, alpha=0.088, **seq)
        return out

    ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2)]
    want = [attend(i, ws[0]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(attend(i, ws[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])


@pytest.mark.parametrize("new,max_len", [([30, 5], 20), ([2, 1], 20), ([40, 9], 9000)])
def test_windows_beyond_every_length(new, max_len):
    """Up to the largest 32-bit number, rows of negative position among them: the same bits as without one."""
    g = torch.Generator().manual_seed(24)
    lens = [20, 5] if new[0] != 2 else [1, 20]
    ref, table = filled(g, lens, 1, 64, 64)
    Q = torch.randn((sum(new), 2, 64), generator=g).half()
    without = run(ref, ref.device(B), Q, table, lens, new, 2, 0.125, True, 0, max_len=max_len)
    check(ref, Q, table, lens, new, 2, 0.125, True, 0, without)
    for window in (20, max_len, 2 ** 31 - 1):
        got = run(ref, ref.device(B), Q, table, lens, new, 2, 0.125, True, window, max_len=max_len)
        assert torch.equal(got[0], without[0]) and torch.equal(got[1], without[1])


@pytest.mark.parametrize("max_new,max_len", [(1, 200), (3, 200), (1, 9000), (40, 200), (40, 40000)])
def test_rows_beyond_max_new_are_left_out(max_new, max_len):
    """They keep what is in them; the rows before them stay the tokens that they are."""
    g = torch.Generator().manual_seed(25)
    lens, new, heads, kv, dim = [200, 90, 33], [max_new + 3, max_new, max(max_new - 1, 1)], 4, 2, 64
    ref, table = filled(g, lens, kv, 64, dim)
    Q = torch.randn((sum(new), heads, dim), generator=g).half()
    out, lse, cu = run(ref, ref.device(B), Q, table, lens, new, heads, 0.125, True, 0, max_new=max_new, max_len=max_len)
    want = R.attention(ref, Q.double().numpy(), table, lens, cu, 3, 0.125, True, 0)
    tol, _ = R.attention_tolerance(f16, *want)
    left = torch.zeros(sum(new), dtype=torch.bool)
    left[max_new:max_new + 3] = True
    assert (out.cpu()[left] == 33).all() and (lse.cpu()[left] == 33).all()
    err = np.abs(out.double().cpu().numpy() - want[0])[~left.numpy()]
    assert (err <= tol[~left.numpy()]).all()


@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_scales_of_blocks_that_nobody_names(new):
    """A block that is not there has no scale either: whatever memory holds instead changes no bit."""
    g = torch.Generator().manual_seed(26)
    lens = [300, 260]
    ref, table = filled(g, lens, 2, 64, 64)
    table[0, 1], table[1, 0] = -1, 1 << 30
    free = [p for p in range(ref.sizes[0]) if p not in table.tolist()[0] + table.tolist()[1]]
    swap = table.clone()  # block 0 is one of those that nobody names
    swap[table == 0] = free[0]
    for x in (ref.k, ref.v, ref.ke, ref.ve):
        x[free[0]] = x[0]
    Q = torch.randn((sum(new), 4, 64), generator=g).half()
    got = []
    for fill in (1.0, float("nan"), float("inf"), 0.0, 2.0 ** 100):
        cache = ref.device(B)
        for i in (2, 3):
            cache.tensors[i][0] = fill
        got.append(run(ref, cache, Q, swap, lens, new, 4, 0.125, True, 0))
    check(ref, Q, swap, lens, new, 4, 0.125, True, 0, got[0])
    for other in got[1:]:
        assert torch.equal(other[1], got[0][1])
        err = R.attention_tolerance(f16, *R.attention(ref, Q.double().numpy(), swap, lens, other[2], 2, 0.125, True, 0))[0]
        assert (np.abs(other[0].double().cpu().numpy() - got[0][0].double().cpu().numpy()) <= 2 * err).all()


@pytest.mark.parametrize("lens,new,heads,kv,dim,max_len", [
    ([700, 90], [1, 1], 8, 2, 128, 704), ([700, 90], [1, 1], 8, 2, 64, 30000), ([5000], [1], 4, 4, 128, 5000),
    ([700, 90], [90, 40], 4, 2, 64, 704), ([1500], [60], 2, 1, 128, 9000)])
def test_the_same_bits_twice(lens, new, heads, kv, dim, max_len):
    g = torch.Generator().manual_seed(27)
    ref, table = filled(g, lens, kv, 64, dim)
    Q = torch.randn((sum(new), heads, dim), generator=g).half()
    cache = ref.device(B)
    a, b = (run(ref, cache, Q, table, lens, new, heads, 0.1, True, 0, max_len=max_len) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_two_graphs_in_turn():
    """Two captured calls of different shapes, each with a workspace of its own, replayed in turn and on two streams; then two
    that share a workspace, replayed one after the other."""
    g = torch.Generator().manual_seed(28)
    ref, table = filled(g, [5000, 3000], 2, 64, 128, spread=1)
    cache, table, lens = ref.device(B), table.to(DEV), i32([5000, 3000])
    shapes = [(1, 8), (30, 4)]
    Q = [torch.randn((2 * n, h, 128), generator=g).half().to(DEV) for n, h in shapes]
    out = [torch.zeros_like(q) for q in Q]
    seqs = [dict(M=2 * n, batch=2, max_new=n, max_len=5000) for n, _ in shapes]
    need = [B.cache_attention_workspace_bytes(heads=h, kv_heads=2, dim=128, **s) for (_, h), s in zip(shapes, seqs)]
    assert all(need)

    def attend(i, ws):
        B.bwta_cache_attention(cache, Q[i], out[i], None, table, lens, None, ws, heads=shapes[i][1], alpha=0.088, **seqs[i])

    one = torch.empty(max(need), dtype=torch.uint8, device=DEV)
    want = []
    for i in range(2):
        attend(i, one)
        torch.cuda.synchronize()
        want.append(out[i].clone())
    for wss, apart in (([torch.empty(n, dtype=torch.uint8, device=DEV) for n in need], True), ([one, one], False)):
        graphs = []
        for i in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[i]):
                attend(i, wss[i])
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(4):
            for o in out:
                o.zero_()
            torch.cuda.synchronize()
            for i in range(2):
                with torch.cuda.stream(streams[i if apart else 0]):
                    graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(out, want))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv,dtype", [(6, 2, f16), (20, 1, b16), (32, 1, f16)])
@pytest.mark.parametrize("window", [0, 130])
def test_sequences_of_eight_to_eleven_steps(dim, heads, kv, dtype, window):
    """So long that a workgroup of twice the wavefronts has one, a last step that holds one key, one sequence without any."""
    case(41 + dim + heads, [513, 700, 0, 20], [1, 1, 0, 1], heads, kv, 64, dim, dtype, True, window)


@pytest.mark.parametrize("dim,group,dtype,causal,window", [(128, 2, f16, True, 0), (64, 3, b16, True, 0), (128, 1, b16, False, 0), (64, 2, f16, True, 90), (128, 5, f16, True, 300)])
def test_equal_shares_of_many_rows(dim, group, dtype, causal, window):
    """Tiles of rows whose steps workgroups share: shares begin and end inside a tile, hold several tiles, heads and sequences, a
    long tile belongs to many, and sequences of no rows or no tokens lie between."""
    g = torch.Generator().manual_seed(dim + group)
    batch, kv, max_new = 52, 3, 70 if group < 5 else 30
    lens = [int(torch.randint(0, 40, (1,), generator=g)) * int(torch.randint(0, 5, (1,), generator=g)) for _ in range(batch)]
    lens[0], lens[20], lens[21], lens[51] = 0, 1700, 0, 900
    new = [int(torch.randint(0, 12, (1,), generator=g)) for _ in range(batch)]
    new[0], new[20], new[21], new[33], new[51] = 3, max_new, 0, 0, max_new
    case(51 + group, lens, new, kv * group, kv, 64, dim, dtype, causal, window, max_new=max(max_new, -(-129 // group)), max_len=5000)


def test_equal_shares_of_one_sequence():
    """Fewer tiles than the host's bound allows, so that a tile is many workgroups', and fewer steps than workgroups."""
    for lens, new in (([1100], [100]), ([60], [3]), ([64], [64])):
        case(61, lens, new, 40, 40, 128, 64, f16, max_new=1000, max_len=6000)


def test_equal_shares_without_rows():
    g = torch.Generator().manual_seed(62)
    ref, table = filled(g, [90] * 50, 3, 64, 128)
    Q = torch.randn((4, 6, 128), generator=g).half()
    got = run(ref, ref.device(B), Q, table, [90] * 50, [0] * 50, 6, 0.1, True, 0, max_new=100, max_len=5000)
    assert (got[0] == 33).all() and (got[1] == 33).all()


@pytest.mark.parametrize("dtype", [f16, b16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 20])
@pytest.mark.parametrize("max_len", [250, 640, 2560])  # a workgroup of four wavefronts for each head, of eight, parts that are joined
def test_every_head_size_of_both_types(max_len, group, dim, dtype):
    case(71 + dim + group, [250, 33], [1, 1], 2 * group, 2, 64, dim, dtype, max_len=max_len)


@pytest.mark.parametrize("new", [[1, 1, 1], [5, 2, 1], [60, 3, 40]])
@pytest.mark.parametrize("window", [1, 63, 64, 700, 1100])
def test_windows_far_inside_long_sequences(new, window):
    """The work is laid out for what a window lets rows see, in a workspace for any."""
    for max_len in (2300, 20000):
        case(81 + window, [2300, 64, 1200], new, 4, 2, 64, 128, f16, True, window, max_len=max_len)
    case(82 + window, [2300, 64, 1200], new, 8, 8, 128, 64, b16, True, window, max_len=200000)


@pytest.mark.parametrize("dim,heads,kv,lens,new,dtype", [(128, 8, 8, [1990], [100], f16), (256, 4, 4, [700, 300], [170, 200], b16), (64, 6, 2, [1500, 300, 40], [30, 22, 40], f16), (128, 24, 6, [900], [22], b16)])
def test_many_rows_in_short_parts(dim, heads, kv, lens, new, dtype):
    """Parts of four steps and more, up to one round of workgroups."""
    case(91 + dim, lens, new, heads, kv, 64, dim, dtype)
    case(92 + dim, lens, new, heads, kv, 64, dim, dtype, False)


def test_bounds_above_the_number_of_rows():
    """max_new counts as M where it is larger: the same layout of the work, the same workspace."""
    g = torch.Generator().manual_seed(97)
    lens, new = [3000, 500], [1, 2]
    ref, table = filled(g, lens, 2, 64, 128)
    Q = torch.randn((3, 4, 128), generator=g).half()
    a, b = (run(ref, ref.device(B), Q, table, lens, new, 4, 0.1, True, 0, max_new=n) for n in (3, 1 << 30))
    check(ref, Q, table, lens, new, 4, 0.1, True, 0, a)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
