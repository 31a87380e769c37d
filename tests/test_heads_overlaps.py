"""Results of bwta_head_norm_rope over the operands that are no rows: refused on the host (no GPU needed)."""
import pytest

from paper_2604_03957_amd import binding as B

P = [0x7F0000000000 + i * (1 << 32) for i in range(8)]  # addresses that are never read
M, H, K, D = 6, 4, 2, 64
QOUT, KOUT, LDQ, LDK = P[6], P[7], H * D + 32, K * D + 16  # rows with room between them


@pytest.mark.parametrize("kw", [
    dict(wq=QOUT), dict(wk=QOUT + 2 * LDQ), dict(wq=KOUT + 16), dict(wk=KOUT + 2 * (M - 1) * LDK + 2 * K * D - 16), dict(wq=QOUT - 2 * D + 16),
    dict(wq=QOUT + 2 * H * D),  # 128 bytes from a gap of 64 on
    dict(positions=QOUT + 2 * LDQ + 8), dict(positions=KOUT - 4 * M + 4), dict(positions=QOUT + 2 * (M - 1) * LDQ + 2 * H * D - 4),
    dict(inv_freq=KOUT), dict(inv_freq=QOUT - 4 * D // 2 + 4), dict(inv_freq=KOUT + 2 * K * D, rot_dim=32),  # 64 bytes from a gap of 32 on
])
def test_results_over_weights_positions_or_frequencies(kw):
    d = dict(Q=P[0], K=P[1], wq=P[2], wk=P[3], positions=P[4], inv_freq=P[5], Qout=QOUT, Kout=KOUT, M=M, heads=H, kv_heads=K, dim=D, ldqo=LDQ, ldko=LDK,
             dtype=B.DTYPE_FP16, stream=0)
    with pytest.raises(B.BwtaError) as e:
        B.bwta_head_norm_rope(**dict(d, **kw))
    assert e.value.code == B.ERR_UNSUPPORTED
