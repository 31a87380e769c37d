"""The operators on heads on parts of wider rows, as the tensors say where they are; whoever marshals the call."""
import ctypes

import pytest
import torch

from paper_2604_03957_amd import binding as B
from test_gpu_heads_binding import _calls

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, K, D, BLK = 4, 2, 64, 64


def forms(name):
    """The call as it is, marshalled natively without its Python form, and in its Python form."""
    def no_fallback(*a, **k):
        raise AssertionError("%s fell back to its Python form" % name)
    native = B._native.bind(name, ctypes.cast(getattr(B.raw(), name), ctypes.c_void_p).value, no_fallback)
    call = getattr(B, name)
    return [call, native, lambda *a, **k: call(*a, **k, stream=torch.cuda.current_stream())]  # a given stream: the Python form


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def fused(tokens, dtype=torch.float16):
    """The rows of one projection: [tokens, H + 2 K heads, D], and its queries, keys and values."""
    g = torch.Generator(device=DEV).manual_seed(tokens)
    qkv = torch.randn((tokens, H + 2 * K, D), device=DEV, generator=g).to(dtype)
    return qkv, qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_parts_of_a_fused_projection(dtype):
    """Rotation in place, write, read and attention on views of one projection's rows, against the same on rows of their own."""
    lens, cu, table = i32([90, 5]), i32([0, 7, 10]), i32([[2, 0], [1, 3]])
    seq = dict(M=10, batch=2, max_new=7, max_len=128)
    pos, inv = torch.arange(10, device=DEV, dtype=torch.int32), torch.rand(D // 2, device=DEV)
    results = []
    for how in range(4):
        _, q, k, v = fused(10, dtype)
        if how == 3:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        rope, write, read, attend = (forms(n)[how % 3] for n in ("bwta_head_norm_rope", "bwta_cache_write", "bwta_cache_read", "bwta_cache_attention"))
        codes = [torch.zeros(s, dtype=torch.uint8, device=DEV) for s in ((4, K, BLK, D), (4, K, D, BLK))]
        cache = B.make_cache(*codes, *(torch.full((4, K), 0.25, device=DEV) for _ in range(2)))
        rope(q, k, None, None, pos, inv, q, k, M=10, heads=H, kv_heads=K, dim=D)
        write(cache, k, v, table, lens, cu, **seq)
        back = torch.full((10, 2 * K + 1, D), 7.0, dtype=dtype, device=DEV)
        read(cache, back[:, :K], back[:, K:2 * K], table, lens, cu, **seq)
        out = torch.full((2, 5, H * D + 8), 7.0, dtype=dtype, device=DEV)[:, :, 8:]  # two times five rows, with something before each
        attend(cache, q, out, None, table, lens, cu, torch.empty(1 << 20, dtype=torch.uint8, device=DEV), heads=H, alpha=0.125, **seq)
        torch.cuda.synchronize()
        assert (back[:, 2 * K:] == 7).all()
        results.append([q.clone(), k.clone(), *codes, *cache.tensors[2:], back.clone(), out.clone()])
    for r in results[:3]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[3]))


def test_rows_that_are_none_are_refused_by_the_calls():
    qkv, q, k, v = fused(10)
    pos, inv = torch.arange(10, device=DEV, dtype=torch.int32), torch.rand(D // 2, device=DEV)
    out = torch.full((10, H, D), 7.0, dtype=torch.float16, device=DEV)
    for bad in (qkv[:, ::2], qkv[:, :H].transpose(0, 1)):
        with pytest.raises(ValueError):
            B.bwta_head_norm_rope(bad, None, None, None, pos, inv, out, None, M=10, heads=H, kv_heads=0, dim=D)
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_a_table_of_one_row_of_any_stride():
    g = torch.Generator(device=DEV).manual_seed(3)
    codes = [torch.randint(0, 127, s, device=DEV, generator=g).to(torch.uint8) for s in ((5, K, BLK, D), (5, K, D, BLK))]
    cache = B.make_cache(*codes, *(torch.full((5, K), 0.25, device=DEV) for _ in range(2)))
    q = torch.randn((1, H, D), device=DEV, generator=g).half()
    ids = i32([[3], [1], [4]])
    seq = dict(M=1, batch=1, max_new=1, max_len=190)
    ws, got = torch.empty(1 << 20, dtype=torch.uint8, device=DEV), []
    for table in (ids.view(1, 3), ids.T, ids.view(-1)):
        for call in forms("bwta_cache_attention"):
            out = torch.zeros_like(q)
            call(cache, q, out, None, table, i32([190]), None, ws, heads=H, alpha=0.125, **seq)
            torch.cuda.synchronize()
            got.append(out)
    assert all(torch.equal(x, got[0]) for x in got) and got[0].abs().max() > 0


def test_short_tensors_are_refused_before_anything_is_launched():
    """Whoever marshals: one row, entry or length where the call's sizes say more."""
    for name, make, kw, written in _calls(torch.float16):
        for i, x in enumerate(make()):
            if not isinstance(x, torch.Tensor) or (name == "bwta_cache_attention" and i == 7):
                continue
            for how in (0, 2):
                a = make()
                whole = a[i]
                a[i] = whole[:1]
                before = [a[j].clone() for j in written if isinstance(a[j], torch.Tensor)] + [whole.clone()]
                with pytest.raises(ValueError):
                    forms(name)[how](*a, **kw)
                torch.cuda.synchronize()
                assert all(torch.equal(b, y) for b, y in zip(before, [a[j] for j in written if isinstance(a[j], torch.Tensor)] + [whole]))


def test_a_given_type_that_is_not_the_tensors_is_refused():
    for name, make, kw, written in _calls(torch.float16):
        for how in (0, 2):
            a = make()
            before = [a[j].clone() for j in written if isinstance(a[j], torch.Tensor)]
            with pytest.raises(TypeError):
                forms(name)[how](*a, **dict(kw, dtype=B.DTYPE_BF16))
            torch.cuda.synchronize()
            assert all(torch.equal(b, a[j]) for b, j in zip(before, [j for j in written if isinstance(a[j], torch.Tensor)]))
        for call in forms(name):
            assert call(*make(), **dict(kw, dtype=B.DTYPE_FP16)) is None
    torch.cuda.synchronize()


def test_a_workspace_that_is_not_there_is_refused():
    name, make, kw, _ = [c for c in _calls(torch.float16) if c[0] == "bwta_cache_attention" and len(c[1]()) == 8][0]
    for how in (0, 2):
        for ws, more in ((torch.zeros(1, dtype=torch.uint8, device=DEV).expand(1 << 20), {}), (torch.zeros(4096, dtype=torch.uint8, device=DEV), dict(workspace_bytes=1 << 20))):
            a = make()
            a[7] = ws
            with pytest.raises(ValueError):
                forms(name)[how](*a, **kw, **more)
            torch.cuda.synchronize()
            assert (a[2] == 3).all() and (ws == 0).all()
