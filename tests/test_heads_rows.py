"""Where the Python forms of the operators on heads look for the rows of a tensor (no GPU needed)."""
import pytest
import torch

from paper_2604_03957_amd import binding as B


def test_rows_are_as_far_apart_as_the_tensors():
    wide = torch.zeros((5, 12, 64), dtype=torch.float16)  # a fused projection: 4 + 4 + 4 heads of 64
    width = 4 * 64
    for x in (wide[:, :4], wide[:, 4:8], wide, wide.view(5, -1), wide.view(5, -1)[:, 64:], wide[:, :4].unsqueeze(1), wide.view(5, 1, -1)):
        assert B._apart(x, None, width) == 12 * 64
    assert B._apart(wide[::2, :4], None, width) == 24 * 64
    assert B._apart(torch.zeros((2, 5, 12, 64))[:, :, :4], None, width) == 12 * 64  # [batch, tokens, heads, dim]
    dense = torch.zeros((5, 4, 64))
    for x in (dense, dense.view(5, -1), dense.view(-1), dense.view(20, 64), dense[:1], wide[:1, :4], dense.view(5, 2, 2, 64), dense[:0], None, 1 << 20, torch.zeros((2, 5, 256))):
        assert B._apart(x, None, width) == width
    assert B._apart(torch.zeros((5, 1, 64)), None, 64) == 64 and B._apart(torch.zeros((5, 3, 64))[:, :1], None, 64) == 192
    assert B._apart(wide, 999, width) == 999 and B._apart(None, 999, width) == 999 and B._apart(wide, None, 0) == 0


def test_rows_that_are_none_are_refused():
    wide = torch.zeros((5, 12, 64), dtype=torch.float16)
    for x in (wide[:, ::2], wide.transpose(0, 1), wide[:, :4].transpose(1, 2), wide[:, 0]):  # every second head, heads first, elements apart, one head of rows of four
        for ld in (None, 12 * 64):
            with pytest.raises(ValueError):
                B._apart(x, ld, 4 * 64)
    uneven = torch.zeros((2, 7, 4, 64))[:, :5]
    with pytest.raises(ValueError):
        B._apart(uneven, None, 4 * 64)
    assert B._apart(uneven, 256, 4 * 64) == 256


def test_a_table_of_one_row():
    t = torch.zeros((7, 1), dtype=torch.int32)
    assert B._ldt(t.T, None, 1) == 7 and B._ldt(t.view(-1), None, 1) == 7 and B._ldt(t.view(1, 7), None, 1) == 7
    assert B._ldt(torch.zeros((3, 9), dtype=torch.int32)[:, :7], None, 3) == 9 and B._ldt(t, None, 7) == 1 and B._ldt(t, 5, 1) == 5
    assert B._ldt(None, None, 1) == 0 and B._ldt(4096, 6, 1) == 6
    with pytest.raises(TypeError):
        B._ldt(t.long(), None, 1)


def test_short_tensors_are_refused():
    """What a call would read or write behind a tensor's last element."""
    x = torch.zeros((5, 4, 64), dtype=torch.float16)
    for t, apart, rows, width in ((x, 256, 5, 256), (x, 256, 0, 256), (x, 256, -1, 256), (x, 512, 3, 256), (x[:, :2], 256, 5, 128), (x[1:], 256, 4, 256), (x[:0], 256, 5, 0),
                                  (None, 256, 9, 256), (4096, 256, 9, 256)):
        B._holds(t, apart, rows, width, 2)
    for t, apart, rows, width in ((x, 256, 6, 256), (x, 264, 5, 256), (x, 256, 5, 257), (x[:, :2], 256, 5, 129), (x[:, 1:], 256, 5, 256), (x[:0], 256, 1, 256), (x[1:], 256, 5, 256),
                                  (x.view(torch.uint8)[:, :, :64], 256, 5, 256)):
        with pytest.raises(ValueError):
            B._holds(t, apart, rows, width, 2)


def test_short_lengths_offsets_and_tables_are_refused():
    cache = B.Cache(4096, 4096, 4096, 4096, 8, 2, 64, 128)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    good = dict(table=i32(3, 4), ldt=4, lens=i32(3), cu=i32(4), M=9, batch=3, max_new=3, max_len=250)
    B._sequences_hold(cache, **good)
    B._sequences_hold(cache, **dict(good, table=i32(3, 7)[:, 2:6], ldt=7, cu=None))
    for empty in (dict(M=0), dict(batch=0), dict(max_new=0)):
        B._sequences_hold(cache, **dict(good, lens=i32(0), **empty))
    for bad in (dict(lens=i32(2)), dict(cu=i32(3)), dict(table=i32(2, 4)), dict(max_len=257), dict(table=i32(3, 3)), dict(table=i32(3, 7)[:, 4:], ldt=7)):
        with pytest.raises(ValueError):
            B._sequences_hold(cache, **dict(good, **bad))


def test_a_given_type_is_the_tensors():
    half, brain, bits = torch.zeros(4, dtype=torch.float16), torch.zeros(4, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int16)
    for dtype, xs in ((B.DTYPE_FP16, (half, half)), (B.DTYPE_BF16, (brain, None)), (B.DTYPE_FP16, (bits, 4096)), (B.DTYPE_BF16, (bits, brain)), (B.DTYPE_FP16, (None, 4096)),
                      (B.DTYPE_INT8, (half, brain)), (9, (half,))):  # the last two are the library's to refuse
        assert B._dtype(dtype, *xs) == dtype
    for dtype, xs in ((B.DTYPE_FP16, (brain,)), (B.DTYPE_BF16, (half,)), (B.DTYPE_FP16, (half, brain)), (B.DTYPE_FP16, (half.float(),)), (B.DTYPE_BF16, (None, brain.view(torch.uint8)))):
        with pytest.raises(TypeError):
            B._dtype(dtype, *xs)


def test_a_workspace_is_in_its_tensor():
    ws = torch.zeros(512, dtype=torch.uint8)
    assert B._room(ws, None) == 512 and B._room(ws, 256) == 256 and B._room(None, None) == 0 and B._room(4096, 1 << 30) == 1 << 30 and B._room(ws.view(torch.float32)[64:], None) == 256
    for x, n in ((ws, 513), (ws[::2], None), (ws[:1].expand(1 << 20), None), (ws[:1].expand(1 << 20), 1)):
        with pytest.raises(ValueError):
            B._room(x, n)


def test_the_quick_form_of_the_checks_is_the_same_checks():
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    wide = half(5, 12, 64)
    tensors = [wide, wide[:, :4], wide[:, 4:8], wide[:, ::2], wide.view(5, -1), wide.view(5, -1)[:, 64:], wide[:1], wide[:1, :4], wide[::2, :4], half(5, 4, 64), half(20, 64), half(1280), half(2, 5, 4, 64),
               half(5, 1, 256), half(5, 300), half(0, 256), wide[:, :4].transpose(0, 1), half(1, 256).expand(5, 256), half(5, 4, 64).float(), None, 4096]
    for x in tensors:
        for M in (-1, 0, 1, 2, 5, 6):
            for width in (0, 64, 256, 320):
                for given in (None, 256, 300, 768):
                    def both():
                        apart = B._apart(x, given, width)
                        B._holds(x, apart, M, width, 2)
                        return apart
                    results = []
                    for f in (both, lambda: B._rows(x, given, M, width)):
                        try:
                            results.append(f())
                        except ValueError:
                            results.append("refused")
                    assert results[0] == results[1], (x if x is None or isinstance(x, int) else (x.shape, x.stride()), M, width, given)
