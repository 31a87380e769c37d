"""The natively marshalled operators on heads on the GPU: the ordinary form of each reaches the C entry point with the same
arguments as the Python form, on the current stream, and raises the same errors; others are the Python form's."""
import ctypes

import pytest
import torch

from paper_2604_03957_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _native_only(name):
    """The native function with a fallback that fails the test."""
    def no_fallback(*a, **k):
        raise AssertionError("%s fell back to its Python form" % name)
    return B._native.bind(name, ctypes.cast(getattr(B.raw(), name), ctypes.c_void_p).value, no_fallback)


def _calls(dtype):
    """(name, a maker of positional arguments, keywords, the places of what is written)"""
    M, H, K, D, blk = 5, 4, 2, 64, 64
    g = torch.Generator(device=DEV).manual_seed(8)
    q, k, v = (torch.randn((M, n * D + 16), device=DEV, generator=g).to(dtype) for n in (H, K, K))
    w = torch.rand(D, device=DEV, generator=g).to(dtype)
    pos, lens, cu = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (list(range(M)), [70, 3], [0, 3, 5]))
    inv = torch.rand(D // 2, device=DEV, generator=g)
    table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device=DEV)
    codes = [torch.randint(0, 127, s, device=DEV, generator=g).to(torch.uint8) for s in ((4, K, blk, D), (4, K, D, blk))]
    out = lambda n: torch.full((M, n * D + 16), 3.0, dtype=dtype, device=DEV)  # noqa: E731
    seq = dict(M=M, batch=2, max_new=3, max_len=128)

    def cache():
        return B.make_cache(*(c.clone() for c in codes), *(torch.full((4, K), 0.25, device=DEV) for _ in range(2)))

    ws = lambda: torch.zeros(max(256, B.cache_attention_workspace_bytes(heads=H, kv_heads=K, dim=D, **seq)), dtype=torch.uint8, device=DEV)  # noqa: E731
    ld = dict(ldq=H * D + 16, ldk=K * D + 16, ldqo=H * D + 16, ldko=K * D + 16)
    return [
        ("bwta_head_norm_rope", lambda: [q, k, w, None, pos, inv, out(H), out(K)], dict(M=M, heads=H, kv_heads=K, dim=D, **ld), (6, 7)),
        ("bwta_head_norm_rope", lambda: [q, None, None, None, pos, inv, out(H), None],
         dict(M=M, heads=H, kv_heads=0, dim=D, rot_dim=32, eps=1e-5, norm=False, interleaved=True, ldq=H * D + 16, ldqo=H * D + 16), (6,)),
        ("bwta_cache_write", lambda: [cache(), k, v, table, lens, cu], dict(seq, ldk=K * D + 16, ldv=K * D + 16), (0,)),
        ("bwta_cache_read", lambda: [cache(), out(K), out(K), table, lens, cu], dict(seq, ldk=K * D + 16, ldv=K * D + 16, ldt=2), (1, 2)),
        ("bwta_cache_read", lambda: [cache(), out(K), out(K), table, lens], dict(seq, max_new=2), (1, 2)),
        ("bwta_cache_attention", lambda: [cache(), q, out(H), torch.zeros((M, H), device=DEV), table, lens, cu, ws()],
         dict(seq, heads=H, alpha=0.125, ldq=H * D + 16, ldo=H * D + 16), (2, 3)),
        ("bwta_cache_attention", lambda: [cache(), q, out(H), None, table, lens], dict(seq, max_new=2, heads=H, alpha=0.5, causal=True, window=7, ldq=H * D + 16), (2,)),
    ]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_native_calls_match_the_python_forms(dtype):
    other = torch.cuda.Stream()
    for name, make, kw, written in _calls(dtype):
        print("native call", name, kw, flush=True)
        results = []
        for how in range(3):
            a = make()
            torch.cuda.synchronize()
            if how == 0:
                getattr(B, name)(*a, **kw, stream=torch.cuda.current_stream())  # a given stream: the Python form
            elif how == 1:
                assert _native_only(name)(*a, **kw) is None
            else:
                with torch.cuda.stream(other):
                    _native_only(name)(*a, **kw)
                other.synchronize()
            torch.cuda.synchronize()
            results.append([x for i in written for x in (a[i].tensors if isinstance(a[i], B.Cache) else (a[i],))])
        for r in results[1:]:
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(r, results[0])), name
        assert any(not torch.equal(x, make()[i]) for x, i in zip(results[0], written) if not isinstance(make()[i], B.Cache)) or written == (0,), name


def test_native_calls_raise_the_same_errors():
    for name, make, kw, _ in _calls(torch.float16):
        f = _native_only(name)
        with pytest.raises(B.BwtaError) as e:
            f(*make(), **dict(kw, M=-1))
        assert e.value.code == B.ERR_SHAPE
        with pytest.raises(B.BwtaError) as e:
            f(*make(), **dict(kw, dtype=B.DTYPE_INT8))
        assert e.value.code == B.ERR_UNSUPPORTED


def test_other_forms_are_the_python_forms():
    for name, make, kw, written in _calls(torch.float16):
        a = make()
        tensors = [i for i, x in enumerate(a) if isinstance(x, torch.Tensor)]
        a[tensors[0]] = a[tensors[0]].cpu()
        with pytest.raises(ValueError):
            getattr(B, name)(*a, **kw)
        a = make()
        i = 1 if name.startswith("bwta_cache") else 0
        a[i] = a[i].float()
        with pytest.raises(TypeError):
            getattr(B, name)(*a, **kw)


def test_tensors_of_other_types_or_strides_are_refused():
    """Whoever marshals: 64-bit lengths, rows of two types, elements apart, a table's columns."""
    for name, make, kw, written in _calls(torch.float16):
        for i, x in enumerate(make()):
            if not isinstance(x, torch.Tensor) or (name == "bwta_cache_attention" and i == 7):
                continue
            bad = [x.double() if x.is_floating_point() else x.long()]
            if x.numel() > 1:
                bad.append(torch.stack([x, x], dim=-1)[..., 0])
            if x.dtype == torch.float16 and i != (1 if name.startswith("bwta_cache") else 0):
                bad.append(x.bfloat16())
            for y in bad:
                a = make()
                a[i] = y
                before = [a[j].clone() for j in written if isinstance(a[j], torch.Tensor)]
                with pytest.raises((TypeError, ValueError)):
                    getattr(B, name)(*a, **kw)
                torch.cuda.synchronize()
                assert all(torch.equal(b, a[j]) for b, j in zip(before, [j for j in written if isinstance(a[j], torch.Tensor)]))
