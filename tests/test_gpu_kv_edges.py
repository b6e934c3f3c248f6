"""Attention over the 4-bit cache where its statistics, masks and launches are stretched, in both of its kernels, against 64 bits.

Tolerances as in test_gpu_kv.py: half a unit in the last place of a result, 2^-16 for a weight, and for a score a few roundings in 32 bits where its
products are few and exact."""
import math

import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import HALF, TINY, TYPES, attend_with_room, check_attention, fill, ints, normal, pool, rng, sequences

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
M = pytest.importorskip("paper_2511_13061_amd")

# rows of q (with very many the kernel for many rows is taken), and what is said of the longest sequence (1: it is in one part)
KERNELS = {"few": (0, None), "few, one part": (0, 1), "many": (2 ** 17, None)}


@pytest.fixture(autouse=True)
def named_kernel(request):
    """The kernel that a test's parameter names, whatever the estimates say."""
    kernel = getattr(request.node, "callspec", None) and request.node.callspec.params.get("kernel")
    M.set_tuning("attention_kernel", 0 if kernel is None else 2 if kernel == "many" else 1)
    yield
    M.set_tuning("attention_kernel", 0)


# ---- weights and their sums ----------------------------------------------------

GAPS = [(32768, 15.0), (32768, 22.25), (131072, 25.1), (32768, 26.0), (32768, 30.5), (32768, 44.0), (131072, 90.0)]
ASKED = 3


def one_ahead_of_many(tokens, gap, kernel, dtype, sums):
    """Attention to tokens of which the first is `gap` powers of two ahead of all others (of a second head half as many) and has no value: results are the
    others' alone, and each of them counts by a weight of 2^-gap.  Returns results, sums, and (first score, weight, tokens seen, sum of their values) of a row."""
    page, dim = 64, 64
    g = rng(int(gap))
    cache = pool(g, tokens // page, page, 1, dim)
    tables = sequences(g, cache, [tokens])
    slots = tables[0, np.arange(tokens) // page] * page + np.arange(tokens) % page
    k, v = normal(g, tokens, 1, dim), normal(g, tokens, 1, dim) + 1
    k[..., :32], v[0] = 0, 0
    k[0, 0, :32] = 1
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    q = torch.zeros((ASKED, 2, dim), dtype=dtype)
    q[:, 0, :32], q[:, 1, :32] = 1.0, 0.5
    scale = gap * math.log(2) / 32                               # the first token's score: 32 products that are 1, exactly
    room, longest = KERNELS[kernel]
    got = attend_with_room(M.KvCache.attend, cache, q.cuda(), ints(tables), ints([tokens]), room, longest=longest, start=ints([0, ASKED]), most_queries=ASKED,
                           scale=scale, sums=sums)
    got, total = got if sums else (got, None)
    values = ref.read(cache.data.cpu().numpy(), page, dim, slots)[1][:, 0]
    rows = {}
    for i in range(ASKED):
        p = tokens - ASKED + i
        for h in range(2):
            first = (32, 16)[h] * float(np.float32(scale))
            rows[i, h] = first, math.exp(-first), p, values[1:p + 1].sum(0)
    return ref.to_numpy(got), total if total is None else ref.to_numpy(total), rows


def off_of(first):
    """How far off a weight may be: scale times log2(e), the maximum and the difference from it are rounded to 32 bits."""
    return first * 2.0 ** -21 + 2.0 ** -16


@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("tokens,gap", GAPS)
def test_attention_one_token_ahead_of_many(tokens, gap, kernel, dtype, sums):
    got, _, rows = one_ahead_of_many(tokens, gap, kernel, dtype, sums)
    for (i, h), (first, w, p, seen) in rows.items():
        want = w * seen / (1 + w * p)
        assert np.linalg.norm(got[i, h] - want) <= (HALF[dtype] + off_of(first)) * np.linalg.norm(want) + TINY[dtype] * len(want) ** 0.5, (i, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("tokens,gap", GAPS)
def test_attention_sums_of_one_token_ahead_of_many(tokens, gap, kernel, dtype):
    """The others' weights are too small to be added to the first one's alone; what they come to together is not."""
    _, sums, rows = one_ahead_of_many(tokens, gap, kernel, dtype, True)
    for (i, h), (first, w, p, _) in rows.items():
        assert abs(sums[i, h] - (first + math.log1p(w * p))) <= first * 2.0 ** -21 + off_of(first) * w * p / (1 + w * p) + 2.0 ** -20, (i, h)


@pytest.mark.parametrize("scale", [1e-30, -1e-37, 1e-38, -2e-39, 1e-45])
@pytest.mark.parametrize("kernel", ["few", "many"])
def test_attention_of_scores_that_are_next_to_nothing(kernel, scale):
    page, dim, length = 16, 64, 300
    cache = pool(rng(1), 20, page, 2, dim)
    tables = sequences(rng(2), cache, [length])
    fill(rng(9), cache, tables, [length])
    q = normal(rng(3), 1, 4, dim)
    got, sums = attend_with_room(M.KvCache.attend, cache, q.cuda(), ints(tables), ints([length]), KERNELS[kernel][0] // 2, start=ints([0, 1]), most_queries=1,
                                 scale=scale, sums=True)
    want, total, reach, far = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, [length], [0, 1], scale=scale)
    check_attention(got, sums, want, total, reach, far, torch.float16)
    assert np.abs(total - math.log(length)).max() < 1e-20


# ---- what is not seen ----------------------------------------------------------

def spoil(cache, tables, tokens, byte):
    """Values of these tokens of sequence 0 get the largest code, of both signs, and this byte in every group."""
    page, dim = cache.page_size, cache.head_dim
    data = cache.data.cpu().numpy()
    for t in tokens:
        _, (codes, _), _, groups = ref.addresses(page, dim, t % page, np.arange(dim))
        data[tables[0, t // page]][:, codes], data[tables[0, t // page]][:, groups] = 0xF7, byte
    cache.data.copy_(torch.from_numpy(data))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("kernel", ["few", "many"])
@pytest.mark.parametrize("byte", [252, 253, 254, 255])
@pytest.mark.parametrize("dim", [64, 160])
def test_attention_values_beyond_the_range_have_no_effect_where_they_are_not_seen(dim, byte, kernel, window, dtype):
    """Values of 2^128 and more, infinities in 32 bits, in tokens that some rows see and others do not."""
    page, heads, kv_heads, length, asked = 16, 4, 2, 200, 120
    clean, dirty = (pool(rng(1), 16, page, kv_heads, dim) for _ in range(2))
    tables = sequences(rng(2), clean, [length])
    for c in (clean, dirty):
        fill(rng(9), c, tables, [length])
    q = normal(rng(3), asked, heads, dim, dtype=dtype)
    call = dict(start=ints([0, asked]), most_queries=asked, window=window, sums=True)
    ask = lambda c: attend_with_room(M.KvCache.attend, c, q.cuda(), ints(tables), ints([length]), KERNELS[kernel][0], **call)  # noqa: E731
    if kernel == "few":                                          # 8 queries with 2 heads of a cache head are one tile of rows
        call.update(start=ints([0, 8]), most_queries=8)
    first = length - (8 if kernel == "few" else asked)
    want, total = ask(clean)
    spots = (195, 130 if window else 198)
    spoil(dirty, tables, spots, byte)
    got, sums = ask(dirty)
    place = np.arange(first, length)
    free = [i for i, p in enumerate(place) if not any(t <= p and (not window or t > p - window) for t in spots)]
    assert 2 < len(free) < len(place)
    assert torch.equal(got[free], want[free]) and torch.equal(sums[free], total[free])
    assert torch.isfinite(got[free]).all()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 60, 2 ** 30, 2 ** 30 - 1])
@pytest.mark.parametrize("kernel", ["few", "many"])
@pytest.mark.parametrize("length,asked", [(57, 60), (200, 300), (1, 90), (0, 5)])
def test_attention_a_window_that_is_longer_than_any_sequence(length, asked, kernel, window):
    """It hides nothing, of queries before the first token's place (there are more queries than tokens) either."""
    page, dim = 16, 64
    cache = pool(rng(1), 14, page, 1, dim)
    tables = sequences(rng(2), cache, [length])
    fill(rng(9), cache, tables, [length])
    q = normal(rng(3), asked, 1, dim)
    got, sums = attend_with_room(M.KvCache.attend, cache, q.cuda(), ints(tables), ints([length]), 2 * KERNELS[kernel][0], start=ints([0, asked]), most_queries=asked,
                                 window=window, sums=True)
    want, total, reach, far = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, [length], [0, asked])
    check_attention(got, sums, want, total, reach, far, torch.float16)


# ---- the largest numbers -------------------------------------------------------

def test_the_largest_numbers_of_bf16_stay_numbers():
    """6 * 2^125 is the largest number that the cache holds: what is above is stored as that, not as 2^128, which is an infinity."""
    big = torch.finfo(torch.bfloat16).max
    x = torch.zeros((5, 1, 64), dtype=torch.float64)
    x[0, 0, :4] = torch.tensor([big, -big, 2.99e38, 2.0 ** 126])
    x[1, 0, :3] = torch.tensor([1.75 * 2.0 ** 127, -2.0 ** 127, 2.0 ** 124])      # 7 * 2^125, to the nearest of 6 and 8: as far as b = 252 goes
    x[2, 0, :2] = torch.tensor([1.5 * 2.0 ** 127, 2.0 ** 127])
    x[3, 0, 0], x[3, 0, 33] = float("inf"), big
    x[4, 0, 5] = -float("nan")
    x = x.bfloat16()
    cache = pool(rng(1), 1, 16, 1, 64)
    cache.append(None, x.cuda(), x.cuda(), None, ints(np.arange(5)))
    unit = 2.0 ** 125
    want = np.zeros((5, 64))
    want[0, :4] = 6 * unit, -6 * unit, 6 * unit, 2 * unit
    want[1, :3] = 6 * unit, -4 * unit, 0.5 * unit
    want[2, :2] = 6 * unit, 4 * unit
    want[3, :32], want[3, 33], want[4, :32] = np.nan, 6 * unit, np.nan
    for got in ref.read(cache.data.cpu().numpy(), 16, 64, np.arange(5)) + [ref.to_numpy(t) for t in cache.read(ints(np.arange(5)), torch.bfloat16)]:
        assert np.array_equal(got[:, 0], want, equal_nan=True)
    # a query that sees one token gets its values
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    assert np.array_equal(ref.to_numpy(cache.attend(q, ints([[0]]), ints([1])))[0, 0], want[0])


# ---- the calls -----------------------------------------------------------------

def test_results_are_allocated_on_the_stream_that_the_call_runs_on(monkeypatch):
    """Memory of another stream's may still be in use there."""
    side, empty, seen = torch.cuda.Stream(), torch.empty, []

    def noted(*args, **more):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **more)

    cache = M.KvCache(2, 16, 1, 64)
    tab, x, at, slots, tables = M.rope_table(8, 64), torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda"), ints([0]), ints([1]), ints([[0]])
    calls = [lambda: M.rope_table(40, 64, stream=side), lambda: M.rope_table(40, 64, device="cuda:0", stream=side.cuda_stream), lambda: M.rotate(x, at, tab, stream=side),
             lambda: cache.append(x, x, x, at, slots, tab, stream=side), lambda: cache.read(slots, stream=side), lambda: cache.attend(x, tables, ints([2]), sums=True, stream=side)]
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", noted)
    for i, call in enumerate(calls):
        seen.clear()
        call()
        assert seen and all(s == side.cuda_stream for s in seen), i
    side.synchronize()
    with pytest.raises(ValueError):
        M.rope_table(4, 64, device="cpu")


@pytest.mark.parametrize("native", [True, False])
def test_append_without_queries_returns_nothing(native, monkeypatch):
    if not native:
        monkeypatch.setattr(M.binding, "_native", None)
    cache = M.KvCache(2, 16, 1, 64)
    x = torch.ones((2, 1, 64), dtype=torch.float16, device="cuda")
    assert cache.append(None, x, x, None, ints([0, 1])) is None
    kept = torch.full_like(x, 3.0)
    assert cache.append(None, x, x, None, ints([0, 1]), q_out=kept) is None and (kept == 3).all()


@pytest.mark.parametrize("native", [True, False])
def test_numbers_that_do_not_fit_the_interface_are_refused(native, monkeypatch):
    """2^32 + 5 was a window of 5."""
    if not native:
        monkeypatch.setattr(M.binding, "_native", None)
    cache = M.KvCache(4, 16, 1, 64)
    cache.data.zero_()
    q, tables, lengths = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda"), ints([[0, 1]]), ints([20])
    for more in (dict(window=2 ** 32 + 5), dict(window=2 ** 31), dict(most_queries=2 ** 32 + 1), dict(most_queries=2 ** 31), dict(window=-1), dict(longest=-1)):
        with pytest.raises((ValueError, M.MackoError)):
            cache.attend(q, tables, lengths, **more)
    assert (cache.attend(q, tables, lengths, window=2 ** 31 - 1, most_queries=2 ** 31 - 1, longest=2 ** 31 - 1) == 0).all()


@pytest.mark.parametrize("native", [True, False])
def test_tables_of_one_page_that_lie_next_to_each_other(native, monkeypatch):
    """A table of one entry has no next one: its stride says nothing."""
    if not native:
        monkeypatch.setattr(M.binding, "_native", None)
    cache = pool(rng(1), 4, 16, 1, 64)
    tables, lengths = np.array([[2], [0], [3]]), [5, 16, 9]
    fill(rng(9), cache, tables, lengths)
    q = normal(rng(3), 3, 2, 64).cuda()
    want = cache.attend(q, ints(tables), ints(lengths))
    assert torch.equal(cache.attend(q, ints([2, 0, 3])[None].t(), ints(lengths)), want)
    with pytest.raises((ValueError, M.MackoError)):
        cache.attend(q, ints([[2, 0, 3], [0, 0, 0]]).t(), ints(lengths))
