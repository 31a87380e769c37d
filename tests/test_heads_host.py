"""Host-side checks of the operators on heads that need no GPU: what they refuse, and with which code, before anything could
be enqueued; their sizes; the Python forms' own checks."""
import ctypes

import pytest
import torch

from paper_2604_03957_amd import binding as B

FAKE = 0x7F0000000000  # 16-byte aligned addresses that are never read
P = [FAKE + i * (1 << 32) for i in range(16)]
INF, NAN = float("inf"), float("nan")


def cache(**kw):
    d = dict(k=P[0], v=P[1], k_scale=P[2], v_scale=P[3], blocks=8, kv_heads=2, block=64, dim=128)
    d.update(kw)
    return B.Cache(d["k"], d["v"], d["k_scale"], d["v_scale"], d["blocks"], d["kv_heads"], d["block"], d["dim"])


def rope(**kw):
    d = dict(Q=P[0], K=P[1], wq=P[2], wk=P[3], positions=P[4], inv_freq=P[5], Qout=P[6], Kout=P[7], M=3, heads=4, kv_heads=2, dim=64, dtype=B.DTYPE_FP16, stream=0)
    d.update(kw)
    B.bwta_head_norm_rope(**d)


def rows(call, **kw):
    d = dict(cache=cache(), K=P[4], V=P[5], table=P[6], lens=P[7], cu=P[8], M=10, batch=2, max_new=5, max_len=200, ldt=4, dtype=B.DTYPE_BF16, stream=0)
    d.update(kw)
    call(**d)


def attend(**kw):
    d = dict(cache=cache(), Q=P[4], out=P[5], lse=P[6], table=P[7], lens=P[8], cu=P[9], workspace=P[10], M=10, batch=2, max_new=5, max_len=200, ldt=4, heads=4,
             alpha=0.1, workspace_bytes=1 << 40, dtype=B.DTYPE_FP16, stream=0)
    d.update(kw)
    B.bwta_cache_attention(**d)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=B.DTYPE_INT8), B.ERR_UNSUPPORTED), (dict(dtype=9), B.ERR_UNSUPPORTED),
    (dict(dim=40), B.ERR_UNSUPPORTED), (dict(dim=272), B.ERR_UNSUPPORTED), (dict(dim=0), B.ERR_UNSUPPORTED),
    (dict(rot_dim=24), B.ERR_UNSUPPORTED), (dict(rot_dim=80), B.ERR_UNSUPPORTED), (dict(rot_dim=-16), B.ERR_UNSUPPORTED),
    (dict(eps=-1e-6), B.ERR_UNSUPPORTED), (dict(eps=NAN), B.ERR_UNSUPPORTED), (dict(eps=INF), B.ERR_UNSUPPORTED),
    (dict(M=-1), B.ERR_SHAPE), (dict(heads=-1), B.ERR_SHAPE), (dict(ldq=255), B.ERR_SHAPE), (dict(ldko=120), B.ERR_SHAPE),
    (dict(heads=1 << 20), B.ERR_TOO_LARGE), (dict(M=1 << 26), B.ERR_TOO_LARGE),
    (dict(Q=None), B.ERR_NULL), (dict(Kout=None), B.ERR_NULL), (dict(positions=None), B.ERR_NULL), (dict(inv_freq=None), B.ERR_NULL),
    (dict(Q=P[0] + 8), B.ERR_ALIGN), (dict(ldk=132), B.ERR_ALIGN), (dict(wq=P[2] + 2), B.ERR_ALIGN), (dict(positions=P[4] + 2), B.ERR_ALIGN),
    (dict(Qout=P[0] + 128), B.ERR_UNSUPPORTED), (dict(Qout=P[0], ldqo=264), B.ERR_UNSUPPORTED),  # rows over their operand, not the same ones
    (dict(Kout=P[0], ldko=256), B.ERR_UNSUPPORTED), (dict(Kout=P[6] + 256, ldko=256), B.ERR_UNSUPPORTED),
    (dict(Qout=P[1], ldk=256), B.ERR_UNSUPPORTED),
])
def test_rope_refusals(kw, code):
    with pytest.raises(B.BwtaError) as e:
        rope(**kw)
    assert e.value.code == code


def test_rope_empty_calls():
    rope(M=0, Q=None, K=None, Qout=None, Kout=None)
    rope(heads=0, kv_heads=0, Q=None, K=None)


@pytest.mark.parametrize("call", [B.bwta_cache_write, B.bwta_cache_read])
@pytest.mark.parametrize("kw,code", [
    (dict(cache=cache(block=32)), B.ERR_UNSUPPORTED), (dict(cache=cache(block=512)), B.ERR_UNSUPPORTED), (dict(cache=cache(dim=96)), B.ERR_UNSUPPORTED),
    (dict(dtype=B.DTYPE_INT8), B.ERR_UNSUPPORTED), (dict(cache=cache(blocks=0)), B.ERR_SHAPE), (dict(cache=cache(kv_heads=0)), B.ERR_SHAPE),
    (dict(batch=-1), B.ERR_SHAPE), (dict(M=-1), B.ERR_SHAPE), (dict(max_new=-1), B.ERR_SHAPE), (dict(max_len=-1), B.ERR_SHAPE),
    (dict(ldt=3), B.ERR_SHAPE), (dict(cu=None, M=9), B.ERR_SHAPE), (dict(ldk=248), B.ERR_SHAPE),
    (dict(lens=None), B.ERR_NULL), (dict(table=None), B.ERR_NULL), (dict(K=None), B.ERR_NULL), (dict(V=None), B.ERR_NULL),
    (dict(cache=cache(k=None)), B.ERR_NULL), (dict(cache=cache(v_scale=None)), B.ERR_NULL),
    (dict(cache=cache(v=P[1] + 8)), B.ERR_ALIGN), (dict(cache=cache(k_scale=P[2] + 2)), B.ERR_ALIGN), (dict(K=P[4] + 2), B.ERR_ALIGN),
    (dict(ldv=260), B.ERR_ALIGN), (dict(cu=P[8] + 1), B.ERR_ALIGN), (dict(table=P[6] + 2), B.ERR_ALIGN), (dict(lens=P[7] + 2), B.ERR_ALIGN),
    (dict(batch=1 << 24), B.ERR_TOO_LARGE), (dict(batch=2 ** 31 - 1, max_new=2 ** 31 - 1), B.ERR_TOO_LARGE), (dict(cache=cache(kv_heads=1 << 15)), B.ERR_TOO_LARGE),
])
def test_cache_row_refusals(call, kw, code):
    with pytest.raises(B.BwtaError) as e:
        rows(call, **kw)
    assert e.value.code == code


def test_reading_over_itself_is_refused():
    with pytest.raises(B.BwtaError) as e:
        rows(B.bwta_cache_read, V=P[4])
    assert e.value.code == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,code", [
    (dict(heads=3), B.ERR_SHAPE), (dict(heads=0), B.ERR_SHAPE), (dict(heads=1 << 15), B.ERR_TOO_LARGE),
    (dict(alpha=0.0), B.ERR_UNSUPPORTED), (dict(alpha=-1.0), B.ERR_UNSUPPORTED), (dict(alpha=INF), B.ERR_UNSUPPORTED), (dict(alpha=NAN), B.ERR_UNSUPPORTED),
    (dict(window=-1), B.ERR_UNSUPPORTED), (dict(window=5, causal=False), B.ERR_UNSUPPORTED),
    (dict(ldq=504), B.ERR_SHAPE), (dict(ldo=504), B.ERR_SHAPE), (dict(Q=None), B.ERR_NULL), (dict(out=None), B.ERR_NULL), (dict(lens=None), B.ERR_NULL),
    (dict(out=P[5] + 4), B.ERR_ALIGN), (dict(lse=P[6] + 2), B.ERR_ALIGN), (dict(out=P[4] + 128), B.ERR_UNSUPPORTED), (dict(out=P[4], ldo=520), B.ERR_UNSUPPORTED),
    (dict(max_len=100000, ldt=2000, workspace=None), B.ERR_WORKSPACE), (dict(max_len=100000, ldt=2000, workspace_bytes=1024), B.ERR_WORKSPACE),
    (dict(max_len=100000, ldt=2000, workspace=P[10] + 128), B.ERR_ALIGN),
    (dict(batch=1 << 23, max_new=1000), B.ERR_TOO_LARGE), (dict(batch=2 ** 31 - 1, max_new=2 ** 31 - 1), B.ERR_TOO_LARGE),
])
def test_attention_refusals(kw, code):
    with pytest.raises(B.BwtaError) as e:
        attend(**kw)
    assert e.value.code == code


def test_empty_calls():
    for kw in (dict(M=0), dict(batch=0), dict(max_new=0)):
        rows(B.bwta_cache_write, **kw)
        attend(**kw)
    with pytest.raises(B.BwtaError) as e:
        B._check(B.raw().bwta_cache_write(None, P[0], 256, P[1], 256, 0, P[2], 4, P[3], P[4], 1, 1, 1, 64, None))
    assert e.value.code == B.ERR_NULL


def test_workspace_sizes():
    f = B.cache_attention_workspace_bytes
    kw = dict(heads=32, kv_heads=8, dim=128)
    assert f(M=0, batch=1, max_new=1, max_len=1000, **kw) == 0 and f(M=1, batch=1, max_new=1, max_len=0, **kw) == 0
    assert f(M=1, batch=1, max_new=1, max_len=64, **kw) == 0           # one step: nothing to split
    assert f(M=8192, batch=1, max_new=8192, max_len=8192, **kw) == 0   # enough rows
    n = f(M=1, batch=1, max_new=1, max_len=131072, **kw)
    assert n > 0 and n % 256 == 0 and n >= 2 * 32 * 130 * 4
    m = f(M=300, batch=1, max_new=300, max_len=131072, **kw)           # many rows: parts of each
    assert m % 256 == 0 and m >= 2 * 300 * 32 * 130 * 4
    assert f(M=1, batch=1, max_new=1, max_len=1000, heads=3, kv_heads=2, dim=128) == 0


def test_python_forms_check_types_and_caches():
    with pytest.raises(TypeError):
        rope(dtype=None)  # addresses have no dtype
    k, v = torch.zeros((3, 2, 64, 128), dtype=torch.uint8), torch.zeros((3, 2, 128, 64), dtype=torch.uint8)
    s = torch.zeros((3, 2))
    c = B.make_cache(k, v, s, s.clone())
    assert (c.blocks, c.kv_heads, c.block, c.dim) == (3, 2, 64, 128) and c.k == k.data_ptr()
    assert ctypes.sizeof(B.Cache) >= 48 and B.Cache.place.offset == 48 and c.place == 0  # the C struct comes first; host tensors
    for bad in ((k, k, s, s), (k, v, s[:2], s), (k, v, s, torch.zeros((2, 3)).T), (k[0], v, s, s), (k.transpose(2, 3), v.transpose(2, 3), s, s)):
        with pytest.raises(ValueError):
            B.make_cache(*bad)
    with pytest.raises(ValueError):
        B.make_cache(k, v, s, s, blocks=4)
    for bad in ((k.short(), v, s, s), (k, v, s.half(), s)):
        with pytest.raises(TypeError):
            B.make_cache(*bad)
    assert B.make_cache(P[0], P[1], P[2], P[3], blocks=1, kv_heads=1, block=64, dim=64).dim == 64


def test_native_marshalling_knows_the_python_forms():
    """Each call is marshalled with the Python form's parameters, in its order, and hands it what is not the ordinary form."""
    import inspect
    table = B._native.head_parameters()
    assert set(table) == {"bwta_head_norm_rope", "bwta_cache_write", "bwta_cache_read", "bwta_cache_attention"}
    for name, (positional, params) in table.items():
        sig = inspect.signature(getattr(B, name))
        assert [p.name for p in sig.parameters.values()] == params, name
        assert sum(p.kind is p.POSITIONAL_OR_KEYWORD for p in sig.parameters.values()) == positional, name
        seen = []
        f = B._native.bind(name, 0, lambda *a, **k: seen.append((a, k)))  # no address: it must not be called
        required = {p.name: 1 for p in sig.parameters.values() if p.kind is p.KEYWORD_ONLY and p.default is p.empty}
        host = torch.zeros(4)
        for args, kw in (((host,) * positional, required), ((P[0],) * positional, required), ((), {}), ((None,) * (positional + 1), required),
                         ((None,) * positional, dict(required, M=1.5)), ((None,) * positional, dict(required, stream=0)), ((None,) * positional, dict(required, nothing=1)),
                         ((bytes(64),) + (None,) * (positional - 1), required)):
            f(*args, **kw)
            assert len(seen) == 1 and all(x is y for x, y in zip(seen[0][0], args)) and seen[0][1] == kw
            seen.clear()


def test_host_tensors_are_refused():
    x = torch.zeros((3, 4, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        rope(Q=x, dtype=None)
    with pytest.raises(ValueError):
        rows(B.bwta_cache_write, K=x, dtype=None)
    with pytest.raises(ValueError):
        attend(lens=torch.zeros(2, dtype=torch.int32))
