"""The rotation's cosines and sines, seen through results of one product each."""
import pytest
import torch

from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("far", [0, 1 << 20, (1 << 31) - (1 << 15)])
def test_cosines_and_sines_to_the_last_bit_of_fp32(far, interleaved):
    """Pairs (1, 0) come out as (cos t, sin t): off from the angle in 64 bits by half a step of fp16 and an ulp of fp32, 2^-24, with a
    third of one for what is left of the angle and the products' rounding, and by the roundings of the angle in 64 bits, 2^-53 of it each:
    one product here, two in the kernel (4 * 2^-24 in all at 2^31).  (An angle rounded to fp32 may be off by pi 2^-25 alone.)"""
    M, dim = 1 << 14, 128
    q = torch.zeros((M, dim), dtype=torch.float16, device=DEV)
    first = slice(0, None, 2) if interleaved else slice(0, dim // 2)
    second = slice(1, None, 2) if interleaved else slice(dim // 2, None)
    q[:, first] = 1.0
    pos = far + torch.arange(M, dtype=torch.int32, device=DEV)
    inv = (10000.0 ** (-torch.arange(0, dim, 2).double() / dim)).float().to(DEV)
    out = torch.empty_like(q)
    B.bwta_head_norm_rope(q, None, None, None, pos, inv, out, None, M=M, heads=1, kv_heads=0, dim=dim, norm=False, interleaved=interleaved)
    t = pos.double().cpu()[:, None] * inv.double().cpu()
    for at, want in ((first, torch.cos(t)), (second, torch.sin(t))):
        got = out[:, at].double().cpu()
        _, e = torch.frexp(want)
        step = torch.exp2((e - 11).clamp(min=-24).double())
        over = (got - want).abs() - step / 2 - 3 * 2.0 ** -53 * t.abs()
        assert (over <= 1.34 * 2.0 ** -24).all(), (over * 2.0 ** 24).max()
