"""bwta_head_norm_rope where operands lie close to its results, but not in them."""
import pytest
import torch

from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_operands_between_and_beside_the_rows_of_results():
    """Weights, positions and frequencies in the gaps of the rows that are written, right before the first and right behind the last."""
    M, H, D, gap = 5, 3, 32, 64
    ld = H * D + gap
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn((M, H * D), device=DEV, generator=g).half()
    w, inv, pos = torch.rand(D, device=DEV, generator=g).half(), torch.rand(D // 2, device=DEV, generator=g), torch.arange(M, device=DEV, dtype=torch.int32) * 7
    want = torch.empty_like(q)
    B.bwta_head_norm_rope(q, None, w, None, pos, inv, want, None, M=M, heads=H, kv_heads=0, dim=D)
    room = torch.zeros(64 + M * ld + 64, dtype=torch.float16, device=DEV)
    out = room[64:64 + M * ld].view(M, ld)

    def put(x, at):  # x's bytes at element `at` of the room
        n = x.numel() * x.element_size() // 2
        room[at:at + n] = x.view(torch.float16)
        return room.data_ptr() + 2 * at

    between, before, behind = 64 + ld + H * D + 8, 64, 64 + (M - 1) * ld + H * D
    for w_at, inv_at, pos_at in ((between, before - D, between + 2 * ld), (behind, between, before - 2 * M), (before - D, between + ld, behind)):
        room.zero_()
        B.bwta_head_norm_rope(q, None, put(w, w_at), None, put(pos, pos_at), put(inv, inv_at), out, None, M=M, heads=H, kv_heads=0, dim=D, ldqo=ld, dtype=B.DTYPE_FP16)
        torch.cuda.synchronize()
        assert torch.equal(out[:, :H * D], want)
