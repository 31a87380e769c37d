"""The 8-bit cache: writing keys and values into it, and reading them back."""
import numpy as np
import pytest
import torch

import heads_ref as R
from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def same_codes(a, b):
    """Equal bytes, but for the sign of zero and of NaN."""
    return (a == b) | ((a & 0x7F == b & 0x7F) & np.isin(a & 0x7F, (0, 0x7F)))


def check(ref, cache):
    got = ref.back(cache)
    assert np.array_equal(got.ke, ref.ke) and np.array_equal(got.ve, ref.ve)
    assert same_codes(got.k, ref.k).all() and same_codes(got.v, ref.v).all()


def some_rows(g, M, heads, dim, dtype, spread=3):
    x = torch.randn((M, heads, dim), generator=g) * torch.exp2(torch.randint(-spread, spread, (M, heads, 1), generator=g).float())
    return x.to(dtype)


CASES = [  # block, dim, heads, dtype, [(tokens before, tokens of each call)...] per sequence
    (64, 128, 2, torch.float16, [(0, [1, 1, 1]), (0, [64, 1, 63]), (0, [5, 0, 130])]),
    (64, 64, 3, torch.bfloat16, [(0, [65, 2, 3]), (0, [0, 1, 4]), (0, [63, 1, 1])]),
    (128, 128, 1, torch.bfloat16, [(0, [300, 7, 1]), (0, [16, 16, 16])]),
    (256, 256, 2, torch.float16, [(0, [255, 1, 1]), (0, [3, 400, 5])]),
    (64, 256, 1, torch.float16, [(0, [1, 1, 1])]),
    (128, 64, 4, torch.float16, [(0, [20, 100, 9]), (0, [129, 127, 200]), (0, [0, 0, 3]), (0, [1, 2, 60])]),
]


@pytest.mark.parametrize("block,dim,heads,dtype,seqs", CASES)
def test_writes_in_a_row_and_reads(block, dim, heads, dtype, seqs):
    """Codes and scales to the bit, each call behind what earlier ones wrote, no token where none is."""
    g = torch.Generator().manual_seed(block + dim)
    batch = len(seqs)
    wide = max(-(-(b + sum(c)) // block) for b, c in seqs)
    blocks = batch * wide + 3
    table = torch.randperm(blocks, generator=g)[:batch * wide].reshape(batch, wide).to(torch.int32)
    ref = R.Cache(blocks, heads, block, dim)
    cache = ref.device(B)
    lens = [b for b, _ in seqs]
    for call in range(len(seqs[0][1])):
        new = [c[call] for _, c in seqs]
        lens = [a + n for a, n in zip(lens, new)]
        cu = np.concatenate(([0], np.cumsum(new)))
        M = int(cu[-1]) + 2  # rows of no sequence
        K, V = (some_rows(g, M, heads, dim, dtype) for _ in range(2))
        ld = heads * dim + 8
        kd = torch.zeros((M, ld), dtype=dtype)
        kd[:, :heads * dim] = K.reshape(M, -1)
        ref.write(K.double().numpy(), V.double().numpy(), table, lens, cu, batch)
        seq = dict(M=M, batch=batch, max_new=max(new), max_len=max(lens) + 5 * (wide * block >= max(lens) + 5))
        B.bwta_cache_write(cache, kd.to(DEV), V.to(DEV), table.to(DEV), i32(lens), i32(cu), ldk=ld, **seq)
        torch.cuda.synchronize()
        check(ref, cache)
        kb, vb = (torch.full((M, heads, dim), 55.0, dtype=dtype, device=DEV) for _ in range(2))
        B.bwta_cache_read(cache, kb, vb, table.to(DEV), i32(lens), i32(cu), **seq)
        torch.cuda.synchronize()
        for b in range(batch):
            k, v, _ = ref.rows(table, b, lens[b])
            for back, want in ((kb, k), (vb, v)):
                got = back[cu[b]:cu[b + 1]].cpu()
                assert torch.equal(got, torch.from_numpy(want[lens[b] - new[b]:]).to(dtype))
        assert (kb[cu[-1]:] == 55).all() and (vb[cu[-1]:] == 55).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_code_and_every_rounding(dtype):
    """All finite 16-bit values of a binade range beside a fixed largest one: each code is the nearest, and reading gives its
    value.  Then a larger token: the codes that are there are rounded again."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16)
    x = bits.view(dtype)
    x = x[torch.isfinite(x) & (x.abs() <= 3.5) & ((x == 0) | (x.abs() >= 2.0 ** -14))]
    x = torch.cat([x, torch.zeros(-len(x) % 128, dtype=dtype)]).reshape(-1, 1, 128)  # one head of 128
    x = torch.cat([x, x[:5]]) if x.shape[0] % 64 == 0 else x  # the last block has a slot left
    M = x.shape[0]
    x[::63, 0, 0] = 3.5  # in every block: 448 * 2^-7
    table = torch.arange(-(-(M + 1) // 64) + 1, dtype=torch.int32)[None]
    ref = R.Cache(table.shape[1], 1, 64, 128)
    cache = ref.device(B)
    seq = dict(batch=1, max_new=M, max_len=table.shape[1] * 64)
    ref.write(x.double().numpy(), -x.double().numpy(), table, [M], [0, M], 1)
    B.bwta_cache_write(cache, x.to(DEV), (-x).to(DEV), table.to(DEV), i32([M]), i32([0, M]), M=M, **seq)
    check(ref, cache)
    big = torch.full((1, 1, 128), 3.5 * 2.0 ** 9, dtype=dtype)
    ref.write(big.double().numpy(), big.double().numpy(), table, [M + 1], [0, 1], 1)
    B.bwta_cache_write(cache, big.to(DEV), big.to(DEV), table.to(DEV), i32([M + 1]), None, M=1, batch=1, max_new=1, max_len=table.shape[1] * 64)
    torch.cuda.synchronize()
    check(ref, cache)


@pytest.mark.parametrize("dtype,values", [
    (torch.float16, [float("nan"), float("inf"), float("-inf"), 65504.0, 6e-8, 0.0, -0.0, 448.0, 449.0, 464.0, 480.0]),
    (torch.bfloat16, [float("nan"), float("inf"), float("-inf"), 3e38, 1e-38, 1e-45, 0.0, 448.0 * 2.0 ** 40, 450.0 * 2.0 ** 40]),
])
def test_special_values(dtype, values):
    """Each value alone in a block, beside ones, and a block of it."""
    n = len(values)
    x = torch.zeros((3 * n, 1, 64), dtype=dtype)
    for i, v in enumerate(values):
        x[3 * i, 0, 7] = v
        x[3 * i + 1] = 1.0
        x[3 * i + 1, 0, 9] = v
        x[3 * i + 2] = v
    table = torch.arange(3 * n, dtype=torch.int32)[:, None]
    ref = R.Cache(3 * n, 1, 64, 64)
    cache = ref.device(B)
    with np.errstate(invalid="ignore", over="ignore"):
        ref.write(x.double().numpy(), -x.double().numpy(), table, [1] * (3 * n), np.arange(3 * n + 1), 3 * n)
    B.bwta_cache_write(cache, x.to(DEV), (-x).to(DEV), table.to(DEV), i32([1] * (3 * n)), M=3 * n, batch=3 * n, max_new=1, max_len=64)
    torch.cuda.synchronize()
    check(ref, cache)
    kb, vb = (torch.empty((3 * n, 1, 64), dtype=dtype, device=DEV) for _ in range(2))
    B.bwta_cache_read(cache, kb, vb, table.to(DEV), i32([1] * (3 * n)), M=3 * n, batch=3 * n, max_new=1, max_len=64)
    most = float(torch.finfo(dtype).max)
    for b in range(3 * n):
        want = torch.from_numpy(np.clip(ref.rows(table, b, 1)[0], -most, most)).to(dtype)
        assert torch.equal(kb[b:b + 1].cpu(), want) and torch.equal(vb[b:b + 1].cpu(), -want) and torch.isfinite(kb[b]).all()


def test_blocks_that_are_not_there_and_rows_before_the_start():
    block, dim, heads = 64, 64, 2
    g = torch.Generator().manual_seed(3)
    table = torch.tensor([[0, -1, 2], [7, 5, 1 << 30], [3, 4, 6]], dtype=torch.int32)  # 7 blocks: 7 and 2^30 are none
    lens, new = [150, 140, 20], [150, 100, 30]  # the last sequence's first ten rows are before its start
    cu = np.concatenate(([0], np.cumsum(new)))
    M = int(cu[-1])
    K, V = (some_rows(g, M, heads, dim, torch.float16) for _ in range(2))
    ref = R.Cache(7, heads, block, dim)
    cache = ref.device(B)
    seq = dict(M=M, batch=3, max_new=150, max_len=192)
    ref.write(K.double().numpy(), V.double().numpy(), table, lens, cu, 3)
    B.bwta_cache_write(cache, K.to(DEV), V.to(DEV), table.to(DEV), i32(lens), i32(cu), **seq)
    torch.cuda.synchronize()
    check(ref, cache)
    kb, vb = (torch.full((M, heads, dim), 9.0, dtype=torch.float16, device=DEV) for _ in range(2))
    B.bwta_cache_read(cache, kb, vb, table.to(DEV), i32(lens), i32(cu), **seq)
    kb, vb = kb.cpu(), vb.cpu()
    for b in range(3):
        k, v, there = ref.rows(table, b, lens[b])
        first = max(0, new[b] - lens[b])
        for back, want in ((kb, k), (vb, v)):
            assert (back[cu[b]:cu[b] + first] == 9).all()
            got = back[cu[b] + first:cu[b + 1]]
            assert torch.equal(got, torch.from_numpy(want[max(0, lens[b] - new[b]):]).half())  # 0 where not there


def test_lengths_and_offsets_outside_their_bounds_stay_inside_memory():
    """Lengths above max_len count as max_len, negative ones as 0, offsets are kept inside the rows."""
    block, dim, heads = 64, 64, 1
    g = torch.Generator().manual_seed(4)
    K, V = (some_rows(g, 8, heads, dim, torch.float16) for _ in range(2))
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32)
    ref = R.Cache(6, heads, block, dim)
    cache = ref.device(B)
    ref.write(K.double().numpy(), V.double().numpy(), table, [128, 0, 0], [0, 3, 3, 3], 3)
    B.bwta_cache_write(cache, K.to(DEV), V.to(DEV), table.to(DEV), i32([1000000, -5, 2 ** 31 - 1]), i32([-4, 3, 2, 1]), M=8, batch=3, max_new=8, max_len=128)
    torch.cuda.synchronize()
    got = ref.back(cache)
    assert same_codes(got.k, ref.k).all() and same_codes(got.v, ref.v).all()


def test_a_cache_beyond_32_bit_offsets():
    """Blocks whose codes lie more than 4 GiB into the cache."""
    heads, block, dim = 8, 64, 128
    blocks = (1 << 32) // (heads * block * dim) + 4
    k, v = torch.empty((blocks, heads, block, dim), dtype=torch.uint8, device=DEV), torch.empty((blocks, heads, dim, block), dtype=torch.uint8, device=DEV)
    ks, vs = (torch.empty((blocks, heads), device=DEV) for _ in range(2))
    cache = B.make_cache(k, v, ks, vs)
    ids = [blocks - 1, 2, blocks - 3]
    table = i32(ids)[None].contiguous()
    g = torch.Generator().manual_seed(6)
    K, V = (some_rows(g, 150, heads, dim, torch.float16) for _ in range(2))
    ref = R.Cache(3, heads, block, dim)
    ref.write(K.double().numpy(), V.double().numpy(), torch.arange(3)[None], [150], [0, 150], 1)
    seq = dict(M=150, batch=1, max_new=150, max_len=150)
    B.bwta_cache_write(cache, K.to(DEV), V.to(DEV), table, i32([150]), **seq)
    kb, vb = (torch.empty((150, heads, dim), dtype=torch.float16, device=DEV) for _ in range(2))
    B.bwta_cache_read(cache, kb, vb, table, i32([150]), **seq)
    want_k, want_v, _ = ref.rows(torch.arange(3)[None], 0, 150)
    assert torch.equal(kb.cpu(), torch.from_numpy(want_k).half()) and torch.equal(vb.cpu(), torch.from_numpy(want_v).half())
    for i, p in enumerate(ids):
        n = min(64, 150 - 64 * i)
        assert same_codes(k[p, :, :n].cpu().numpy(), ref.k[i, :, :n]).all() and same_codes(v[p, :, :, :n].cpu().numpy().transpose(0, 2, 1), ref.v[i, :, :n]).all()


@pytest.mark.parametrize("max_new", [1, 40, 70])
def test_rows_beyond_max_new_are_left_out(max_new):
    """Written: the first max_new rows, as the tokens that they are; read: only they."""
    block, dim, heads, lens, new = 64, 64, 2, [200, 130], [max_new + 9, max_new]
    g = torch.Generator().manual_seed(7)
    cu = np.concatenate(([0], np.cumsum(new)))
    M = int(cu[-1])
    K, V = (some_rows(g, M, heads, dim, torch.float16) for _ in range(2))
    table = torch.randperm(8, generator=g).reshape(2, 4).to(torch.int32)
    ref = R.Cache(8, heads, block, dim)
    before = [max(0, n - m) for n, m in zip(lens, new)]  # what is there before
    K0, V0 = (some_rows(g, sum(before), heads, dim, torch.float16) for _ in range(2))
    ref.write(K0.double().numpy(), V0.double().numpy(), table, before, np.concatenate(([0], np.cumsum(before))), 2)
    cache = ref.device(B)
    kept = [lens[0] - 9, lens[1]]  # the same tokens as a call of max_new rows each
    rows = [*range(max_new), *range(max_new + 9, M)]
    ref.write(K[rows].double().numpy(), V[rows].double().numpy(), table, kept, [0, max_new, 2 * max_new], 2)
    seq = dict(M=M, batch=2, max_new=max_new, max_len=200)
    B.bwta_cache_write(cache, K.to(DEV), V.to(DEV), table.to(DEV), i32(lens), i32(cu), **seq)
    torch.cuda.synchronize()
    check(ref, cache)
    kb, vb = (torch.full((M, heads, dim), 9.0, dtype=torch.float16, device=DEV) for _ in range(2))
    B.bwta_cache_read(cache, kb, vb, table.to(DEV), i32(lens), i32(cu), **seq)
    kb, vb = kb.cpu(), vb.cpu()
    k, v, _ = ref.rows(table, 0, kept[0])
    for back, want in ((kb, k), (vb, v)):
        assert torch.equal(back[:max_new], torch.from_numpy(want[kept[0] - max_new:]).half())
        assert (back[max_new:max_new + 9] == 9).all() and (back[max_new + 9:] != 9).any()


def test_the_same_bits_twice():
    g = torch.Generator().manual_seed(8)
    K, V = (some_rows(g, 300, 2, 128, torch.bfloat16).to(DEV) for _ in range(2))
    ref = R.Cache(6, 2, 64, 128)
    caches = [ref.device(B) for _ in range(2)]
    table, lens = i32([[5, 0, 3, 1, 2]]), i32([300])
    for cache in caches:
        B.bwta_cache_write(cache, K, V, table, lens, M=300, batch=1, max_new=300, max_len=300)
        B.bwta_cache_write(cache, 64 * K[:9], V[:9], table, lens + 9, M=9, batch=1, max_new=9, max_len=309)
    torch.cuda.synchronize()
    for a, b in zip(caches[0].tensors, caches[1].tensors):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [64, 128, 256])
def test_every_block_and_head_size_of_both_types(block, dim, dtype):
    """A prompt that ends inside a block, tokens one by one over the block's end, a chunk."""
    test_writes_in_a_row_and_reads(block, dim, 2, dtype, [(0, [block + 3, 1, 7]), (0, [block - 1, 1, block])])
    test_writes_in_a_row_and_reads(block, dim, 1, dtype, [(0, [1, 1]), (0, [1, 1])])
