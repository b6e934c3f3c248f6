"""The calls around the 8-bit key/value cache, as far as they go without a GPU: sizes, what they refuse before anything is launched, the reference itself."""
import ctypes

import numpy as np
import pytest

import kv8_reference as ref

M = pytest.importorskip("paper_2511_13061_amd")
kv = pytest.importorskip("paper_2511_13061_amd.kv")

INVALID, UNSUPPORTED = -1, -3
A = 1 << 20          # an address that is aligned and never followed


def cache(pages=4, page_size=16, kv_heads=2, head_dim=64, codes=A, scales=A):
    return kv._CCache8(codes, scales, pages, page_size, kv_heads, head_dim)


def rotation(positions=A, table=A, table_rows=10, rot=64, interleaved=0, eps=1e-6):
    return kv._CRotation(positions, table, table_rows, rot, interleaved, eps)


def append(r=None, **change):
    a = kv._CAppend8(3, 4, 0, 3, A, 256, 64, A, 256, 64, A, 128, 64, A, 128, 64, A, 8, 8, A, None, None, None, r or rotation())
    for name, value in change.items():
        setattr(a, name, value)
    return a


def attention(**change):
    a = kv._CAttention(3, 4, 0, 3, A, 256, 64, A, 256, 64, None, A, 8, 8, A, None, 1, 0, 100, 0.125)
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("pages,page,heads,dim", [(0, 16, 1, 32), (1, 16, 1, 32), (7, 64, 8, 128), (3, 4096, 5, 224), (100000, 256, 40, 256)])
def test_size_of_a_pool(pages, page, heads, dim):
    scales = ctypes.c_int64(-1)
    lib = M.load_library()
    assert lib.macko_kv8_cache_bytes(ctypes.byref(cache(pages, page, heads, dim, None, None)), ctypes.byref(scales)) == pages * page * heads * dim * 2
    assert scales.value == pages * page // 16 * heads * 2


@pytest.mark.parametrize("change,status", [
    (dict(pages=-1), INVALID), (dict(page_size=0), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=-32), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED),
    (dict(head_dim=288), UNSUPPORTED), (dict(kv_heads=65537), UNSUPPORTED), (dict(pages=2 ** 27), UNSUPPORTED)])
def test_geometries_that_are_refused(change, status):
    c = cache(**change)
    lib = M.load_library()
    assert lib.macko_kv8_cache_bytes(ctypes.byref(c), None) == status
    assert lib.macko_kv8_read(ctypes.byref(c), 1, A, 0, A, 128, 64, A, 128, 64, None) == status
    assert lib.macko_kv8_append(ctypes.byref(c), ctypes.byref(append()), None) == status
    assert lib.macko_kv8_attention(ctypes.byref(c), ctypes.byref(attention()), None, 0, None) == status
    assert lib.macko_kv8_cache_bytes(None, None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(heads=-1), INVALID), (dict(type=2), INVALID), (dict(batch=-1), INVALID), (dict(batch=2), INVALID), (dict(k=None), INVALID),
    (dict(v=A + 1), INVALID), (dict(q=None), INVALID), (dict(q_out=A + 1), INVALID), (dict(tables=None), INVALID), (dict(tables=A + 2), INVALID), (dict(lengths=None), INVALID),
    (dict(lengths=A + 1), INVALID), (dict(start=A + 2), INVALID), (dict(table_width=-1), INVALID), (dict(table_stride=-1), INVALID), (dict(k_token=-1), INVALID),
    (dict(v_head=-64), INVALID), (dict(q_weight=A + 1), INVALID), (dict(k_token=2 ** 40), INVALID), (dict(tokens=2 ** 31 - 1, start=A), UNSUPPORTED),
    (dict(heads=65537), UNSUPPORTED), (dict(r=rotation(positions=None)), INVALID), (dict(r=rotation(table=None)), INVALID), (dict(r=rotation(rot=128)), INVALID),
    (dict(r=rotation(rot=24)), UNSUPPORTED)])
def test_appends_that_are_refused(change, status):
    r = change.pop("r", None)
    assert M.load_library().macko_kv8_append(ctypes.byref(cache()), ctypes.byref(append(r, **change)), None) == status


@pytest.mark.parametrize("missing", [dict(codes=None), dict(codes=A + 8), dict(scales=None), dict(scales=A + 1)])
def test_memory_that_is_missing(missing):
    lib = M.load_library()
    c = cache(**missing)
    assert lib.macko_kv8_append(ctypes.byref(c), ctypes.byref(append()), None) == INVALID
    assert lib.macko_kv8_read(ctypes.byref(c), 1, A, 0, A, 128, 64, A, 128, 64, None) == INVALID
    assert lib.macko_kv8_attention(ctypes.byref(c), ctypes.byref(attention()), A, 1 << 30, None) == INVALID
    assert lib.macko_kv8_append(ctypes.byref(cache()), None, None) == INVALID
    assert lib.macko_kv8_attention(ctypes.byref(cache()), None, None, 0, None) == INVALID


@pytest.mark.parametrize("args", [(-1, A, 0, A, A), (1, None, 0, A, A), (1, A + 1, 0, A, A), (1, A, 3, A, A), (1, A, 0, A + 1, A)])
def test_reads_that_are_refused(args):
    tokens, slots, kind, k, v = args
    assert M.load_library().macko_kv8_read(ctypes.byref(cache()), tokens, slots, kind, k, 128, 64, v, 128, 64, None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(heads=3), INVALID), (dict(type=5), INVALID), (dict(batch=2), INVALID), (dict(q=None), INVALID), (dict(out=A + 1), INVALID),
    (dict(sums=A + 2), INVALID), (dict(tables=None), INVALID), (dict(lengths=None), INVALID), (dict(start=A + 2), INVALID), (dict(most_queries=0), INVALID),
    (dict(window=-1), INVALID), (dict(longest=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(tokens=2 ** 30, start=A), UNSUPPORTED),
    (dict(tokens=65536, batch=65536), UNSUPPORTED)])
def test_attention_that_is_refused(change, status):
    lib = M.load_library()
    c = cache()
    assert lib.macko_kv8_attention(ctypes.byref(c), ctypes.byref(attention(**change)), A, 1 << 40, None) == status
    if status == UNSUPPORTED:
        assert lib.macko_kv8_attention_workspace(ctypes.byref(c), ctypes.byref(attention(**change))) == status


def test_workspace_of_attention():
    lib = M.load_library()
    c = cache(kv_heads=8, head_dim=128)
    size = lambda **k: lib.macko_kv8_attention_workspace(ctypes.byref(c), ctypes.byref(attention(heads=32, **k)))  # noqa: E731
    assert size(longest=1) == 0 and size(tokens=0) == 0 and size(batch=0) == 0
    long = size(longest=131072, tokens=1, batch=1)
    splits, rest = divmod(long - 4 * 32, 32 * 4 * (128 + 2))       # maximum, sum and the unnormalised result of every row and part; how many parts a row has
    assert rest == 0 and 2 <= splits <= 256
    a = attention(heads=32, longest=131072, tokens=1, batch=1)
    for workspace, given in ((A, long - 1), (None, long), (A + 4, long)):
        assert lib.macko_kv8_attention(ctypes.byref(c), ctypes.byref(a), workspace, given, None) == INVALID
    for batch in (1, 3, 64, 1000):
        for longest in (1, 500, 4096, 10 ** 6, 2 ** 31 - 1):
            for queries in (1, 5, 17, 1000):
                for window in (0, 1000):
                    n = size(batch=batch, tokens=batch * queries, longest=longest, most_queries=queries, window=window, start=A)
                    assert n >= 0 and (n == 0 or (n - 4 * batch * queries * 32) % (batch * queries * 32 * 4 * 130) == 0)


@pytest.mark.parametrize("geometry", [(2 ** 64 + 4, 16, 2, 64), (4, 2 ** 32 + 16, 2, 64), (4, 16, 2 ** 32 + 2, 64), (4, 16, 2, 2 ** 32 + 64)])
def test_geometries_that_do_not_fit_the_interface(geometry):
    with pytest.raises(ValueError, match="does not fit"):
        M.KvCache8(*geometry)


def test_the_reference_by_hand():
    """Ties to the even code, subnormal codes, 448 at most, NaN; a block's byte; earlier tokens that are rounded again."""
    assert ref.nearest(np.array([1.0625, 1.1875, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 500.0, -1e9])).tolist() == [1.0, 1.25, 16.0, 20.0, 0.0, 2.0 ** -8, 448.0, -448.0]
    assert np.isnan(ref.nearest(np.array([np.nan, np.inf]))).all()
    assert [ref.byte_of(np.array([x])) for x in (448.0, 448.1, 224.0, 0.0, 1e-45, 3e38, np.inf)] == [127, 128, 126, 1, 1, 246, 1]
    held = [np.zeros((16, 1, 32)), np.zeros((16, 1, 32)), np.full((1, 1, 1, 2), 9, dtype=np.uint8)]
    k = np.full((3, 1, 32), 3.0)
    k[0, 0, 0], k[2, 0, 0] = 0.0137, 448.0 * 64
    table = np.zeros((1, 1), dtype=np.int64)
    assert ref.append(held, k[:2], k[:2], 16, table, [2], [0, 2], 1) == [0, 1]
    small = 0.013671875                                       # 1.75 * 2^-7, at a factor of 2^-7
    assert held[2].ravel().tolist() == [120, 120] and held[0][0, 0, 0] == small and held[0][1, 0, 1] == 3.0
    ref.append(held, k[2:], k[2:], 16, table, [3], [0, 1], 1)
    assert held[2].ravel().tolist() == [133, 133] and held[0][0, 0, 0] == 0.0 and held[0][1, 0, 1] == 3.0 and held[0][2, 0, 0] == 448 * 64
