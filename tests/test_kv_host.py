"""The calls around the key/value cache, as far as they go without a GPU: sizes, and what they refuse before anything is launched."""
import ctypes

import numpy as np
import pytest

import kv_reference as ref

M = pytest.importorskip("paper_2511_13061_amd")
kv = pytest.importorskip("paper_2511_13061_amd.kv")

INVALID, UNSUPPORTED = -1, -3
A = 1 << 20          # an address that is aligned and never followed


def cache(pages=4, page_size=16, kv_heads=2, head_dim=64, data=A):
    return kv._CCache(data, pages, page_size, kv_heads, head_dim)


@pytest.mark.parametrize("pages,page,heads,dim", [(0, 16, 1, 32), (1, 16, 1, 32), (7, 64, 8, 128), (3, 4096, 5, 224), (100000, 256, 40, 256)])
def test_size_of_a_pool(pages, page, heads, dim):
    c = cache(pages, page, heads, dim, None)
    assert M.load_library().macko_kv_cache_bytes(ctypes.byref(c)) == pages * heads * ref.piece_bytes(page, dim)


@pytest.mark.parametrize("change,status", [
    (dict(pages=-1), INVALID), (dict(page_size=0), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=-32), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED),
    (dict(head_dim=288), UNSUPPORTED), (dict(kv_heads=65537), UNSUPPORTED), (dict(pages=2 ** 27), UNSUPPORTED)])
def test_geometries_that_are_refused(change, status):
    c = cache(**change)
    lib = M.load_library()
    assert lib.macko_kv_cache_bytes(ctypes.byref(c)) == status
    assert lib.macko_kv_read(ctypes.byref(c), 1, A, 0, A, 128, 64, A, 128, 64, None) == status
    assert lib.macko_kv_append(ctypes.byref(c), ctypes.byref(append()), None) == status
    assert lib.macko_kv_attention(ctypes.byref(c), ctypes.byref(attention()), None, 0, None) == status
    assert lib.macko_kv_cache_bytes(None) == INVALID


def rotation(positions=A, table=A, table_rows=10, rot=64, interleaved=0, eps=1e-6):
    return kv._CRotation(positions, table, table_rows, rot, interleaved, eps)


def append(r=None, **change):
    a = kv._CAppend(3, 4, 0, A, 256, 64, A, 256, 64, A, 128, 64, A, 128, 64, A, None, None, r or rotation())
    for name, value in change.items():
        setattr(a, name, value)
    return a


def attention(**change):
    a = kv._CAttention(3, 4, 0, 3, A, 256, 64, A, 256, 64, None, A, 8, 8, A, None, 1, 0, 100, 0.125)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(heads=-1), INVALID), (dict(type=2), INVALID), (dict(k=None), INVALID), (dict(v=A + 1), INVALID), (dict(q=None), INVALID),
    (dict(q_out=A + 1), INVALID), (dict(slots=None), INVALID), (dict(slots=A + 2), INVALID), (dict(k_token=-1), INVALID), (dict(v_head=-64), INVALID),
    (dict(q_weight=A + 1), INVALID), (dict(k_token=2 ** 40), INVALID), (dict(tokens=2 ** 31), UNSUPPORTED), (dict(heads=65537), UNSUPPORTED),
    (dict(r=rotation(positions=None)), INVALID), (dict(r=rotation(table=None)), INVALID), (dict(r=rotation(table=A + 4)), INVALID), (dict(r=rotation(rot=128)), INVALID),
    (dict(r=rotation(rot=-16)), INVALID), (dict(r=rotation(rot=24)), UNSUPPORTED), (dict(r=rotation(table_rows=-1)), INVALID)])
def test_appends_that_are_refused(change, status):
    r = change.pop("r", None)
    assert M.load_library().macko_kv_append(ctypes.byref(cache()), ctypes.byref(append(r, **change)), None) == status


def test_memory_that_is_missing():
    lib = M.load_library()
    for data in (None, A + 8):
        c = cache(data=data)
        assert lib.macko_kv_append(ctypes.byref(c), ctypes.byref(append()), None) == INVALID
        assert lib.macko_kv_read(ctypes.byref(c), 1, A, 0, A, 128, 64, A, 128, 64, None) == INVALID
        assert lib.macko_kv_attention(ctypes.byref(c), ctypes.byref(attention()), A, 1 << 30, None) == INVALID
    assert lib.macko_kv_append(ctypes.byref(cache()), None, None) == INVALID
    assert lib.macko_kv_attention(ctypes.byref(cache()), None, None, 0, None) == INVALID


@pytest.mark.parametrize("args", [(-1, A, 0, A, A), (1, None, 0, A, A), (1, A + 1, 0, A, A), (1, A, 3, A, A), (1, A, 0, A + 1, A)])
def test_reads_that_are_refused(args):
    tokens, slots, kind, k, v = args
    assert M.load_library().macko_kv_read(ctypes.byref(cache()), tokens, slots, kind, k, 128, 64, v, 128, 64, None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(type=5), INVALID), (dict(batch=-1), INVALID), (dict(batch=2), INVALID),
    (dict(q=None), INVALID), (dict(out=A + 1), INVALID), (dict(q_token=-5), INVALID), (dict(sums=A + 2), INVALID), (dict(tables=None), INVALID), (dict(tables=A + 1), INVALID),
    (dict(lengths=None), INVALID), (dict(lengths=A + 1), INVALID), (dict(start=A + 2), INVALID), (dict(table_width=-1), INVALID), (dict(table_stride=-1), INVALID),
    (dict(most_queries=0), INVALID), (dict(window=-1), INVALID), (dict(longest=-1), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(tokens=2 ** 31, start=A), UNSUPPORTED), (dict(tokens=2 ** 30, start=A), UNSUPPORTED), (dict(heads=2 ** 17), UNSUPPORTED), (dict(longest=2 ** 31), UNSUPPORTED),
    (dict(tokens=65536, batch=65536), UNSUPPORTED), (dict(heads=65536), UNSUPPORTED)])
def test_attention_that_is_refused(change, status):
    lib = M.load_library()
    c = cache() if change != dict(heads=65536) else cache(kv_heads=1)
    assert lib.macko_kv_attention(ctypes.byref(c), ctypes.byref(attention(**change)), A, 1 << 40, None) == status
    if status == UNSUPPORTED:
        assert lib.macko_kv_attention_workspace(ctypes.byref(c), ctypes.byref(attention(**change))) == status


def test_workspace_of_attention():
    lib = M.load_library()
    size = lambda **c: lib.macko_kv_attention_workspace(ctypes.byref(cache(kv_heads=8, head_dim=128)), ctypes.byref(attention(heads=32, **c)))  # noqa: E731
    assert size(longest=1) == 0 and size(longest=100) == 0 and size(tokens=0) == 0 and size(batch=0) == 0
    long = size(longest=131072, tokens=1, batch=1)
    splits, rest = divmod(long - 4 * 32, 32 * 4 * (128 + 2))       # maximum, sum and the unnormalised result of every row and part; how many parts a row has
    assert rest == 0 and 2 <= splits <= 256
    # too little of it, none of it, and some that is not aligned
    a = attention(heads=32, longest=131072, tokens=1, batch=1)
    for workspace, given in ((A, long - 1), (None, long), (A + 4, long)):
        assert lib.macko_kv_attention(ctypes.byref(cache(kv_heads=8, head_dim=128)), ctypes.byref(a), workspace, given, None) == INVALID
    for batch in (1, 3, 64, 1000):
        for longest in (1, 500, 4096, 10 ** 6, 2 ** 31 - 1):
            for queries in (1, 5, 17, 1000):
                for window in (0, 1000):
                    n = size(batch=batch, tokens=batch * queries, longest=longest, most_queries=queries, window=window, start=A)
                    assert n >= 0 and (n == 0 or (n - 4 * batch * queries * 32) % (batch * queries * 32 * 4 * 130) == 0)


@pytest.mark.parametrize("args", [
    (-1, 4, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A), (0, -4, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A), (0, 4, 63, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A),
    (0, 4, 0, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A), (0, 4, 258, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A), (0, 4, 64, 0.0, 1.0, 0.0, 1.0, 32.0, 1.0, A),
    (0, 4, 64, float("nan"), 1.0, 0.0, 1.0, 32.0, 1.0, A), (0, 4, 64, 1e4, -2.0, 0.0, 1.0, 32.0, 1.0, A), (0, 4, 64, 1e4, 1.0, float("inf"), 1.0, 32.0, 1.0, A),
    (0, 4, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None), (0, 4, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, A + 2)])
def test_tables_that_are_refused(args):
    assert M.load_library().macko_rope_table(*args, None) == INVALID


def test_rotations_that_are_refused():
    lib = M.load_library()
    r = rotation()
    call = lambda tokens=3, heads=2, dim=64, kind=0, x=A, w=None, out=A, rot=r: lib.macko_rotate(  # noqa: E731
        tokens, heads, dim, kind, x, 128, 64, None if rot is None else ctypes.byref(rot), w, out, 128, 64, None)
    assert call(rot=None) == INVALID and call(tokens=-1) == INVALID and call(heads=-1) == INVALID and call(kind=9) == INVALID and call(x=None) == INVALID
    assert call(out=A + 1) == INVALID and call(w=A + 1) == INVALID and call(dim=0) == INVALID and call(dim=48) == UNSUPPORTED and call(dim=320) == UNSUPPORTED
    assert call(rot=rotation(rot=96)) == INVALID and call(rot=rotation(rot=40)) == UNSUPPORTED and call(rot=rotation(table=None)) == INVALID
    assert call(tokens=2 ** 31) == UNSUPPORTED and call(heads=2 ** 17) == UNSUPPORTED
    assert call(tokens=0) == 0 and call(heads=0, x=None, out=None) == 0


def test_nearest_values_of_the_reference():
    """The reference's rounding, by hand: the middle between two codes goes to the even one, above 7 the factor doubles."""
    x = np.zeros((1, 32))
    x[0, :12] = [7, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.001, -0.2501, 6.9, 0.0]
    assert ref.nearest(x)[0, :12].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -6, -0.5, 6, 0]
    x[0, 0] = 7.0001
    assert ref.nearest(x)[0, :8].tolist() == [8, 4, 4, 2, 2, 1, 1, 0]       # in steps of 1, 2, 3, 4, 6, 8 and 12 now
    x[0, 0] = np.inf
    assert np.isnan(ref.nearest(x)).all()
