"""Norm of heads and rotation by position (bwta_head_norm_rope) against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import heads_ref as R
from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _close(got, want, size, dtype):
    """One rounding of the result, and fp32 arithmetic on the pair: the sum of up to 256 squares, root, quotient, weight, a
    cosine and a sine of 2^-22 (the reduced angle is rounded once, times 2 pi), two products and a sum: at most
    (64 + 32) * 2^-24 of |y_a| + |y_b|."""
    eps = torch.finfo(dtype).eps / 2
    tol = eps * np.abs(want) * 1.0001 + 96 * 2.0 ** -24 * size + float(torch.finfo(dtype).smallest_normal) * eps
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err / tol).max()


CASES = [  # M, heads, kv_heads, dim, rot, interleaved, norm, dtype
    (1, 32, 32, 128, 128, False, True, torch.float16),
    (1, 1, 1, 16, 16, False, True, torch.bfloat16),
    (3, 5, 1, 64, 64, True, True, torch.float16),
    (7, 8, 2, 96, 48, False, True, torch.bfloat16),      # a head of six lanes, half of it rotated
    (5, 3, 2, 112, 112, True, True, torch.float16),      # seven lanes
    (130, 12, 12, 64, 32, True, False, torch.float16),
    (33, 10, 2, 256, 256, False, True, torch.bfloat16),
    (9, 4, 4, 240, 16, False, True, torch.float16),
    (2, 7, 0, 32, 32, False, True, torch.float16),        # queries alone
    (2, 0, 3, 48, 0, False, True, torch.float16),         # keys alone, norm alone
    (4100, 2, 1, 128, 128, False, True, torch.float16),
]


@pytest.mark.parametrize("M,heads,kv,dim,rot,inter,norm,dtype", CASES)
def test_against_64_bits(M, heads, kv, dim, rot, inter, norm, dtype):
    g = torch.Generator().manual_seed(M + dim)
    lead, pad = 8, 24  # a row has something before and behind the heads
    ld = lead + (heads + kv) * dim + pad
    rows = (torch.randn((M, ld), generator=g) * torch.exp2(torch.randint(-6, 6, (M, 1), generator=g).float())).to(dtype)
    w = [(1 + 0.3 * torch.randn(dim, generator=g)).to(dtype) for _ in range(2)]
    pos = torch.randint(0, 1 << 20, (M,), generator=g, dtype=torch.int32)
    pos[0] = -3
    inv = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float()
    dev = rows.to(DEV)
    q, k = dev[:, lead:lead + heads * dim], dev[:, lead + heads * dim:]
    qo, ko = (torch.full((M + 1, n * dim + 8), 77.0, dtype=dtype, device=DEV) for n in (heads, kv))
    B.bwta_head_norm_rope(q if heads else None, k if kv else None, w[0].to(DEV), w[1].to(DEV), pos.to(DEV), inv.to(DEV), qo, ko, M=M, heads=heads, kv_heads=kv, dim=dim,
                          rot_dim=rot, eps=1e-5, norm=norm, interleaved=inter, ldq=ld, ldk=ld, ldqo=heads * dim + 8, ldko=kv * dim + 8)
    torch.cuda.synchronize()
    assert torch.equal(dev.cpu(), rows)
    for out, n, at, wt in ((qo, heads, lead, w[0]), (ko, kv, lead + heads * dim, w[1])):
        if not n:
            continue
        x = rows[:, at:at + n * dim].reshape(M, n, dim)
        want, size = R.rope(x, wt, pos, inv, rot, inter, 1e-5, norm)
        _close(out[:M, :n * dim].reshape(M, n, dim), want, size, dtype)
        assert (out[M] == 77).all() and (out[:, n * dim:] == 77).all()  # behind the last row and between the rows


def test_in_place_without_weights_and_far_positions():
    M, heads, kv, dim = 65, 4, 2, 128
    g = torch.Generator().manual_seed(5)
    rows = torch.randn((M, (heads + kv) * dim), generator=g).half()
    pos = (2 ** 31 - 1 - torch.arange(M)).to(torch.int32)
    inv = (1e6 ** (-torch.arange(0, dim, 2).double() / dim)).float()
    dev = rows.to(DEV)
    q, k = dev[:, :heads * dim], dev[:, heads * dim:]
    ld = dev.stride(0)
    B.bwta_head_norm_rope(q, k, None, None, pos.to(DEV), inv.to(DEV), q, k, M=M, heads=heads, kv_heads=kv, dim=dim, ldq=ld, ldk=ld, ldqo=ld, ldko=ld)
    torch.cuda.synchronize()
    want, size = R.rope(rows.reshape(M, heads + kv, dim), None, pos, inv, dim, False, 1e-6, True)
    _close(dev.reshape(M, heads + kv, dim), want, size, torch.float16)


def test_special_values_and_zero_heads():
    x = torch.zeros((4, 2, 64), dtype=torch.float16)
    x[1, 0, 3] = float("nan")
    x[2, 1, 5] = float("inf")
    x[3] = 60000.0
    inv = torch.ones(32)
    out = torch.empty_like(x).to(DEV)
    B.bwta_head_norm_rope(x.to(DEV), None, None, None, torch.zeros(4, dtype=torch.int32, device=DEV), inv.to(DEV), out, None, M=4, heads=2, kv_heads=0, dim=64, eps=0.0 + 1e-6)
    out = out.cpu()
    assert (out[0] == 0).all() and out[1, 0].isnan().all() and (out[1, 1] == 0).all()
    assert out[2, 1, 5].isnan() and (out[2, 0] == 0).all()  # inf / inf
    assert (out[3] - 1).abs().max() <= 2.0 ** -11


def test_many_heads_are_spread_and_many_tokens_are_not():
    """The same rows in one call and token by token: the same bits, whatever a wavefront has of a token."""
    M, heads, kv, dim = 6000, 9, 3, 64
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k = (torch.randn((M, n, dim), device=DEV, generator=g).bfloat16() for n in (heads, kv))
    pos = torch.arange(M, device=DEV, dtype=torch.int32) * 17
    inv = (10000.0 ** (-torch.arange(0, dim, 2).double() / dim)).float().to(DEV)
    whole, single = ([torch.empty_like(q), torch.empty_like(k)] for _ in range(2))
    kw = dict(heads=heads, kv_heads=kv, dim=dim)
    B.bwta_head_norm_rope(q, k, None, None, pos, inv, *whole, M=M, **kw)
    for m in range(0, M, 997):
        B.bwta_head_norm_rope(q[m:m + 1], k[m:m + 1], None, None, pos[m:m + 1], inv, single[0][m:m + 1], single[1][m:m + 1], M=1, **kw)
    torch.cuda.synchronize()
    for m in range(0, M, 997):
        assert torch.equal(whole[0][m], single[0][m]) and torch.equal(whole[1][m], single[1][m])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 128, 256])
def test_every_head_size_of_both_types_and_orders(dim, inter, dtype):
    test_against_64_bits(17, 3, 2, dim, dim // 32 * 16 or 16, inter, True, dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_norm_alone_needs_no_positions(dtype):
    g = torch.Generator().manual_seed(6)
    x, w = torch.randn((9, 3, 80), generator=g).to(dtype), (1 + torch.rand(80, generator=g)).to(dtype)
    out = torch.empty((9, 3, 80), dtype=dtype, device=DEV)
    B.bwta_head_norm_rope(x.to(DEV), None, w.to(DEV), None, None, None, out, None, M=9, heads=3, kv_heads=0, dim=80, rot_dim=0)
    torch.cuda.synchronize()
    want, size = R.rope(x, w, None, None, 0, False, 1e-6, True)
    _close(out, want, size, dtype)
