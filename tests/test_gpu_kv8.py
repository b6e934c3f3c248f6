"""The 8-bit key/value cache and attention over it, on the GPU, against tests/kv8_reference.py (64 bits).

Tolerances.  A result of 16 bits is off by at most half a unit in the last place, 2^-11 (fp16) or 2^-8 (bf16) of it, from what was computed.  What was
computed: rotation and norm in 32 bits, some ten roundings, 2^-20 of the largest product that enters.  Attention: a score is a sum of up to 256 exact products in 32 bits, off
by 2^-16 of the sum of their magnitudes at most, so a weight by the same share of it times scale, numerator and denominator alike, and a weight
goes in with 16 bits (2^-16 for rounding, as much for the exponential and the sums), in calls of more than 64 rows of a sequence on a key/value head with 11 (2^-11)."""
import numpy as np
import pytest

import kv8_reference as ref
import kv_reference as ref4

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
M = pytest.importorskip("paper_2511_13061_amd")

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float16, torch.bfloat16]
to_numpy = ref4.to_numpy


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype=torch.float16, scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)


def ints(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()


def close(got, want, dtype, slack):
    """|got - want| <= half a unit in the last place and slack (an array or a number); NaN and infinities where they belong."""
    got = to_numpy(got)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bound = np.abs(want) * HALF[dtype] * (1 + 2.0 ** -10) + TINY[dtype] + slack
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - want) <= bound) & ~np.isnan(want) & ~(got == want)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the worst by {np.nanmax(np.where(bad, np.abs(got - want) / bound, 0)):.2f} of the bound"


def pool(g, pages, page, heads, dim):
    """A pool of random bytes: what nobody wrote has to have no effect."""
    blocks = (pages, heads, page // 16, 2)
    make = lambda *shape: torch.randint(0, 256, shape, generator=g, dtype=torch.uint8).cuda()  # noqa: E731
    return M.KvCache8(pages, page, heads, dim, data=make(*blocks, 16 * dim), scales=make(*blocks))


def content(cache):
    return cache.data.cpu().numpy(), cache.scales.cpu().numpy()


def sequences(g, cache, lengths):
    """Tables for these lengths; pages in random order, what is not used of the tables names no page."""
    order = torch.randperm(cache.pages, generator=g).tolist()
    width = max([-(-n // cache.page_size) for n in lengths] + [0]) + 2
    tables = np.full((len(lengths), width), -2 ** 31, dtype=np.int64)
    for b, n in enumerate(lengths):
        for i in range(-(-max(n, 0) // cache.page_size)):
            tables[b, i] = order.pop()
    return tables


def fill(g, cache, tables, lengths, dtype=torch.float16, scale=1.0):
    """Keys and values of all tokens, through append."""
    lengths = [max(n, 0) for n in lengths]
    k = normal(g, sum(lengths), cache.kv_heads, cache.head_dim, dtype=dtype, scale=scale)
    k[..., ::19] *= 4
    v = normal(g, sum(lengths), cache.kv_heads, cache.head_dim, dtype=dtype)
    cache.append(None, k.cuda(), v.cuda(), None, ints(tables), ints(lengths), start=ints(np.concatenate([[0], np.cumsum(lengths)])))
    return k, v


# ---- the cache ----------------------------------------------------------------

APPENDS = [
    # heads, kv heads, dim, page, rot, norm, interleaved, calls: (tokens of each sequence that are new) ...
    (4, 4, 128, 16, 128, False, False, [[1], [1], [1]]),
    (10, 2, 64, 32, 32, True, False, [[17, 0, 5], [1, 1, 1], [20, 3, 40], [1, 14, 0]]),
    (3, 3, 32, 16, 32, False, True, [[15, 16, 17, 1], [1, 1, 1, 1], [2, 33, 0, 16]]),
    (4, 1, 96, 64, 96, True, True, [[50], [14], [1], [64]]),
    (0, 2, 160, 16, 0, False, False, [[3, 30], [14, 1]]),
    (6, 3, 192, 128, 64, True, False, [[19, 120], [100, 20]]),
    (2, 1, 224, 16, 224, False, False, [[18], [18]]),
    (8, 8, 256, 16, 128, True, True, [[40, 2, 9], [8, 14, 1]]),
    # calls that go by 16 rows
    (4, 8, 128, 32, 128, True, False, [[700, 1, 0, 400], [9, 600, 1, 500]]), (2, 16, 64, 16, 32, False, True, [[5, 1100, 30], [900, 17, 250]]),
    (0, 40, 32, 64, 0, False, False, [[430, 440]]), (3, 6, 256, 16, 256, False, False, [[1400, 3], [16, 1390]]), (2, 8, 96, 128, 96, True, True, [[1] * 30 + [1100], [3] * 30 + [1000]]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_and_read(case, dtype):
    """Calls one after the other: blocks that fill up in several, whose scales grow; what is not written stays."""
    heads, kv_heads, dim, page, rot, norm, interleaved, calls = APPENDS[case]
    g = rng(case * 10 + 1)
    total = np.sum(calls, 0)
    cache = pool(g, sum(-(-n // page) for n in total) + 2, page, kv_heads, dim)
    cache.scales.clamp_(90, 160)                                     # values that are not written stay numbers to compare
    tables = sequences(g, cache, total)
    every = np.arange(cache.pages * page)
    tab = M.rope_table(300, rot) if rot else None
    wq, wk = (normal(g, dim, dtype=dtype) if norm else None for _ in range(2))
    w64 = [to_numpy(w) if norm else None for w in (wq, wk)]
    lengths = np.zeros(len(total), dtype=np.int64)
    for step, fresh in enumerate(calls):
        data, scales = content(cache)
        held = [x.copy() for x in ref.read(data, scales, page, every)] + [scales.copy()]
        lengths += fresh
        start = np.concatenate([[0], np.cumsum(fresh)])
        tokens = int(start[-1])
        fused = normal(g, tokens, heads + 2 * kv_heads, dim, dtype=dtype, scale=2.0 * 4.0 ** step)
        fused[:, heads:, 5] *= 0.001
        at = torch.randint(0, 300, (tokens,), generator=g).numpy()
        dev = fused.cuda()
        got = cache.append(dev[:, :heads] if heads else None, dev[:, heads:heads + kv_heads], dev[:, heads + kv_heads:], ints(at) if rot else None, ints(tables), ints(lengths),
                           start=ints(start), table=tab, q_weight=wq.cuda() if norm else None, k_weight=wk.cuda() if norm else None, eps=1e-5, interleaved=interleaved)
        t64 = tab.cpu().numpy() if rot else None
        if heads:
            want = ref4.rotate(to_numpy(fused[:, :heads]), at, t64, w64[0], 1e-5, interleaved)
            size = np.abs(ref4.rotate(np.abs(to_numpy(fused[:, :heads])), at, None, None if w64[0] is None else np.abs(w64[0]), 1e-5)).max(-1, keepdims=True)
            close(got, want, dtype, size * 2.0 ** -20)
        else:
            assert got is None
        turned = ref4.rotate(to_numpy(fused[:, heads:heads + kv_heads]), at, t64, w64[1], 1e-5, interleaved)
        before = [x.copy() for x in held[:2]]
        written = ref.append(held, turned, to_numpy(fused[:, heads + kv_heads:]), page, tables, lengths, start, cache.pages)
        assert len(written) == tokens
        data, scales = content(cache)
        keys, values = ref.read(data, scales, page, every)
        assert np.array_equal(scales[..., 1], held[2][..., 1]) and np.array_equal(values, held[1], equal_nan=True)
        # keys are rounded to 32 bits on the way: where that moves one over the edge between two codes, it is a step away, 2^-3 of it, or the least one
        assert np.array_equal(scales[..., 0], held[2][..., 0])
        unit = np.exp2(held[2][..., 0].astype(np.float64) - 127)[every // page, :, every % page // 16][..., None]
        same = (keys == held[0]) | np.isnan(keys) & np.isnan(held[0])
        others = np.setdiff1d(every, written)
        assert same[others].all() and same.mean() > 0.999
        near = np.abs(keys - held[0]) <= np.maximum(np.abs(held[0]) / 7, unit * 2.0 ** -9)
        assert (same | near).all()
        assert step == 0 or not np.array_equal(held[0][others], before[0][others], equal_nan=True) or (scales == held[2]).all()
    for out in TYPES:
        some = np.concatenate([every[::-1], [-1, cache.pages * page, 0, 1, 2, 3, 3, 2, 1, 0]])
        for x, y in zip(cache.read(ints(some), out), ref.read(data, scales, page, some)):
            assert x.dtype == out and torch.equal(x.cpu().nan_to_num(-77.0), torch.from_numpy(y).to(out).nan_to_num(-77.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 96, 256])
def test_read_of_every_byte_and_code(dim, dtype):
    """All factors with all codes, results beyond the type's range and below it included; slots in order, backwards and in pieces."""
    page = 32
    pages = 128
    data = (np.arange(pages * 2 * 2 * 16 * dim, dtype=np.int64) * 37 % 256).astype(np.uint8).reshape(pages, 1, 2, 2, 16 * dim)
    scales = (np.arange(pages * 4) // 2 % 247).astype(np.uint8).reshape(pages, 1, 2, 2)
    cache = M.KvCache8(pages, page, 1, dim, data=torch.from_numpy(data).cuda(), scales=torch.from_numpy(scales).cuda())
    for slots in (np.arange(pages * page), np.arange(pages * page)[::-1], np.arange(1, pages * page - 5), np.arange(0, pages * page, 4), np.array([7]), np.array([-1, 5, 6, 7, 8])):
        for x, y in zip(cache.read(ints(slots), dtype), ref.read(data, scales, page, slots)):
            want = torch.from_numpy(y).float().to(dtype)             # one rounding: every value is one of 32 bits
            assert torch.equal(x.cpu().nan_to_num(-77.0, posinf=6e4, neginf=-6e4), want.nan_to_num(-77.0, posinf=6e4, neginf=-6e4))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,heads", [(32, 4), (64, 3), (96, 2), (160, 5), (256, 1)])
def test_read_of_long_lists(dim, heads, dtype):
    """Entries four to a group of lanes: in order from every place of a block on, backwards, with gaps, twice, outside the pool, an odd number of them."""
    page, pages = 32, 20
    g = rng(dim)
    cache = pool(g, pages, page, heads, dim)
    cache.scales.clamp_(100, 140)
    every = np.arange(pages * page)
    slots = np.concatenate([every, every[1:], every[2:-1], every[3:], every[::-1], every[::4], every[1::2], [-1, -5, pages * page, 2 ** 31 - 1, -2 ** 31], np.repeat(every, 2),
                            torch.randperm(pages * page, generator=g).numpy()])
    slots = np.tile(slots, -(-140000 // (slots.size * heads * 4)))[:-2]
    assert slots.size * heads * 4 > 2 ** 17
    for x, y in zip(cache.read(ints(slots), dtype), ref.read(*content(cache), page, slots)):
        want = torch.from_numpy(y).float().to(dtype)                 # one rounding: every value is one of 32 bits
        assert torch.equal(x.cpu().nan_to_num(-77.0, posinf=6e4, neginf=-6e4), want.nan_to_num(-77.0, posinf=6e4, neginf=-6e4))


@pytest.mark.parametrize("dtype", TYPES)
def test_append_edges_of_codes_zeros_and_what_is_not_finite(dtype):
    """Values at the middle between two codes, the largest and smallest numbers, blocks of zeros, an infinity and a NaN among others."""
    steps = ref.STEPS
    rows = [np.concatenate([(steps[:-1] + steps[1:]) / 2, steps[-2:]])[:128], np.zeros(128), np.full(128, 3.5), np.linspace(-448, 448, 128)]
    big, small = torch.finfo(dtype).max, 2.0 ** (-24 if dtype == torch.float16 else -133)
    rows += [np.array([big, -big, big / 3] + [0.0] * 125), np.array([small, -small, 3 * small] + [0.0] * 125), np.array([np.inf, 1.0, -np.inf, np.nan] * 32), np.array([1e-3] * 127 + [65504.0])]
    n = len(rows)
    x = torch.from_numpy(np.stack(rows)).to(dtype).view(n, 1, 128)
    cache = pool(rng(1), n, 16, 1, 128)
    tables, lengths = np.arange(n)[:, None], np.ones(n, dtype=np.int64)     # a block for each
    cache.append(None, x.cuda(), x.cuda(), None, ints(tables), ints(lengths))
    data, scales = content(cache)
    keys, values = ref.read(data, scales, 16, np.arange(n) * 16)
    x64 = to_numpy(x)
    for i in range(n):
        byte = ref.byte_of(x64[i])
        assert (scales[i].ravel() == byte).all(), (i, scales[i].ravel(), byte)
        want = ref.nearest(x64[i] / 2.0 ** (byte - 127)) * 2.0 ** (byte - 127)
        assert np.array_equal(keys[i], want, equal_nan=True) and np.array_equal(values[i], want, equal_nan=True)


def test_append_of_what_has_no_place():
    """More rows than tokens, rows of no sequence, a length below zero, pages that are missing: stored nowhere, everything else stays; positions outside the table."""
    g = rng(4)
    page, dim = 16, 64
    cache = pool(g, 6, page, 2, dim)
    cache.scales[3] = 120                                            # of the block that a token joins below
    data, scales = (x.clone() for x in (cache.data, cache.scales))
    tables = np.array([[0, 1], [2, 9], [3, -1], [4, 5]])
    lengths, start = [2, 20, 18, -4], [1, 5, 9, 12, 14]               # row 0 and rows 14, 15 are no sequence's
    tab = M.rope_table(30, 64)
    q, k, v = (normal(g, 16, h, dim) for h in (3, 2, 2))
    at = np.arange(16)
    at[4], at[7] = 30, -1                                            # place 1 of sequence 0, a row of sequence 1 whose page is missing
    got = cache.append(q.cuda(), k.cuda(), v.cuda(), ints(at), ints(tables), ints(lengths), start=ints(start), table=tab)
    want = ref4.rotate(to_numpy(q), at, tab.cpu().numpy())
    close(got, want, torch.float16, np.abs(to_numpy(q)).max() * 2.0 ** -20)
    assert np.isnan(want[[4, 7]]).all()
    # sequence 0: rows 3, 4 at places 0, 1; sequence 1: rows 5 to 8 at places 16 to 19, page 9; sequence 2: rows 9 to 11 at places 15 (page 3), 16, 17 (page -1)
    d, s = content(cache)
    keys, values = ref.read(d, s, page, [0, 1, 3 * page + 15])
    assert np.isnan(keys[1]).all() and not np.isnan(keys[[0, 2]]).any()
    turned = ref4.rotate(to_numpy(k), at, tab.cpu().numpy())
    assert np.abs(keys[0] - turned[3]).max() < 0.2 and np.abs(values[1] - to_numpy(v)[4]).max() < 0.2 and np.abs(values[2] - to_numpy(v)[9]).max() < 0.5
    touched = torch.zeros(cache.scales.shape, dtype=torch.bool)
    touched[0, :, 0], touched[3, :, 0] = True, True
    assert torch.equal(cache.scales.cpu()[~touched], scales.cpu()[~touched])
    assert torch.equal(cache.data.cpu()[~touched], data.cpu()[~touched])
    # places behind the new tokens keep their codes
    new = cache.data.cpu()[0, :, 0, 0].view(2, 16, dim)
    assert torch.equal(new[:, 2:], data.cpu()[0, :, 0, 0].view(2, 16, dim)[:, 2:])
    assert cache.append(None, k[:0].cuda(), v[:0].cuda(), None, ints(tables[:0]), ints([])) is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,kv_heads", [(128, 8), (32, 32), (256, 6)])
def test_append_of_many_sequences_is_that_of_each(dim, kv_heads, dtype):
    """One call of many tokens against a call for every sequence: the same bytes in the pool.  Among them rows of no sequence in front and behind, more rows than
    tokens, missing pages, tables that are too short, positions outside the table, blocks whose scale grows, values that are not finite."""
    g = rng(dim)
    page, heads, batch, rot = 32, 3, 90, 32
    one, two = (pool(rng(5), 400, page, kv_heads, dim) for _ in range(2))
    fresh = torch.randint(0, 40, (batch,), generator=g).tolist()
    fresh[3], fresh[40], fresh[41] = 0, 150, 1
    while sum(fresh) % 16 != 5:
        fresh[7] += 1
    past = [int(torch.randint(0, 70, (1,), generator=g)) for _ in fresh]
    past[9] = -5                                                       # five rows have no place
    lengths = np.array([p + n for p, n in zip(past, fresh)])
    lengths[20] = -3
    start = np.concatenate([[6], 6 + np.cumsum(fresh)])
    tokens = int(start[-1]) + 9
    assert tokens >= 512 and tokens >= 4 * batch                       # by 16 rows
    tables = np.stack([np.arange(b, 400, batch)[:4] for b in range(batch)])
    tables = np.concatenate([tables, tables[:, :1] + 3000], 1)         # 128 to 159: no page
    tables[12, 0] = -1
    x = [normal(g, tokens, h, dim, dtype=dtype, scale=2.0) for h in (heads, kv_heads, kv_heads)]
    for t in x[1:]:
        t *= torch.exp2(torch.randint(-5, 6, (tokens, 1, 1), generator=g)).to(dtype)
        t[100, 0, 3], t[101, -1, 5], t[150, 1] = float("nan"), float("inf"), 0.0
    at = torch.randint(0, 300, (tokens,), generator=g).numpy()
    at[50], at[200] = 300, -2
    tab, w = M.rope_table(300, rot), normal(g, dim, dtype=dtype).cuda()
    q, k, v = (t.cuda() for t in x)
    more = dict(table=tab, q_weight=w, k_weight=w, eps=1e-6)
    got = one.append(q, k, v, ints(at), ints(tables), ints(lengths), start=ints(start), **more)
    for b in range(batch):
        lo, hi = start[b], start[b + 1]
        if hi > lo:
            want = two.append(q[lo:hi], k[lo:hi], v[lo:hi], ints(at[lo:hi]), ints(tables[b:b + 1]), ints(lengths[b:b + 1]), start=ints([0, hi - lo]), **more)
            # 32 bits in both, in another order in the norm's sum perhaps: a unit in the last place
            a, c = got[lo:hi].float().cpu(), want.float().cpu()
            assert torch.equal(a.isnan(), c.isnan()) and ((a - c).abs() <= c.abs() * torch.finfo(dtype).eps + 1e-6).masked_fill(c.isnan(), True).all()
    assert torch.equal(one.data, two.data) and torch.equal(one.scales, two.scales)
    assert torch.isnan(got[[50, 200]]).all() and not torch.isnan(got[:6]).any()


def test_offsets_beyond_32_bits():
    """Pages on both sides of 2^31 and 2^32 bytes of a pool, through all three calls."""
    page, heads, dim = 64, 8, 128
    piece = heads * page * dim * 2
    pages = (2 ** 32) // piece + 3
    cache = M.KvCache8(pages, page, heads, dim)
    assert cache.data.numel() > 2 ** 32
    g = rng(3)
    use = [0, (2 ** 31) // piece, (2 ** 31) // piece + 1, (2 ** 32) // piece, pages - 1]
    k, v = (normal(g, 300, heads, dim) for _ in range(2))
    cache.append(None, k.cuda(), v.cuda(), None, ints([use]), ints([300]), start=ints([0, 300]))
    slots = np.concatenate([p * page + np.arange(page) for p in use])[:300]
    small, scales = cache.data[use].cpu().numpy(), cache.scales[use].cpu().numpy()
    for x, y in zip(cache.read(ints(slots)), ref.read(small, scales, page, np.arange(300))):
        assert np.array_equal(to_numpy(x), y)
    # half a step of 4 significant bits is 2^-4 of a value at most (one of 4 to 8 in steps of 1/2 is off by up to 1/4)
    assert np.all(np.abs(to_numpy(cache.read(ints(slots))[1]) - to_numpy(v)) <= np.abs(to_numpy(v)) * 2.0 ** -4 + 2.0 ** -10)
    q = normal(g, 1, 8, dim)
    got, sums = cache.attend(q.cuda(), ints([use]), ints([300]), sums=True)
    check_attention(got, sums, *ref.attend_cached(to_numpy(q), small, scales, page, np.arange(5)[None], [300]), torch.float16)


# ---- attention ----------------------------------------------------------------

def check_attention(got, sums, want, total, reach, far, dtype, weight=2.0 ** -15):
    share = reach * 2.0 ** -16 + weight
    close(got, want, dtype, (2 * share * far)[..., None])
    fine = np.isfinite(want)
    norm = np.linalg.norm(want[fine])
    assert norm == 0 or np.linalg.norm(to_numpy(got)[fine] - want[fine]) <= HALF[dtype] * norm
    if sums is not None:
        s = to_numpy(sums)
        assert np.array_equal(np.isnan(s), np.isnan(total)) and np.array_equal(s == -np.inf, total == -np.inf)
        fine = np.isfinite(total)
        assert np.all(np.abs(s[fine] - total[fine]) <= reach[fine] * 2.0 ** -16 + np.abs(total[fine]) * 2.0 ** -21 + 2.0 ** -15)


ATTENTION = [
    # dim, page, heads, kv heads, lengths, queries, window
    (128, 16, 8, 8, [1], None, 0), (128, 16, 4, 2, [2, 15, 16, 17, 31, 32, 33, 0, 47, 48], None, 0), (128, 64, 8, 2, [127, 128, 129, 63, 64, 65], None, 0),
    (64, 32, 40, 8, [300, 0, 5, 1], None, 0), (32, 16, 3, 1, [70, 33], None, 0), (96, 128, 4, 4, [200, 1], None, 0), (160, 16, 5, 1, [50, 129], None, 0),
    (192, 32, 6, 3, [65], None, 0), (224, 16, 2, 2, [40], None, 0), (256, 16, 16, 2, [100, 7], None, 0), (128, 4096, 2, 1, [5000], None, 0),
    (128, 16, 17, 1, [90], None, 0), (64, 16, 64, 1, [90, 33], None, 0),
    (128, 16, 8, 2, [50, 20, 4, 0, 9], [5, 1, 4, 2, 0], 0),                                  # several queries; more of them than tokens; none
    (64, 32, 4, 4, [40, 90], [40, 33], 0), (128, 32, 12, 4, [200], [70], 0), (256, 16, 4, 1, [60], [23], 0), (96, 16, 10, 2, [170, 30], [60, 30], 0),
    (128, 16, 4, 2, [100, 60, 3], None, 7), (64, 16, 8, 8, [100, 60, 3], [4, 9, 3], 20), (128, 32, 2, 1, [150], [40], 1), (96, 16, 3, 3, [300], [3], 33),
    (128, 16, 8, 8, [1500, 700, 3, 0, 1200], None, 0), (64, 64, 8, 1, [2500, 600], [3, 2], 0), (128, 16, 2, 2, [2000, 900], [2, 1], 600),
    (128, 64, 8, 2, [700, 333], [300, 200], 0), (192, 16, 4, 1, [400], [150], 90), (32, 32, 4, 2, [500, 200], [250, 130], 0),
]


def attention_case(case, dtype):
    dim, page, heads, kv_heads, lengths, queries, window = ATTENTION[case]
    g = rng(case)
    cache = pool(g, sum(-(-n // page) for n in lengths) + 2, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths, dtype)
    n = [1] * len(lengths) if queries is None else queries
    start = np.concatenate([[0], np.cumsum(n)])
    q = normal(g, sum(n), heads, dim, dtype=dtype, scale=1.5)
    want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, lengths, start, window=window)
    more = {} if queries is None else dict(start=ints(start), most_queries=max(n))
    return cache, q, tables, lengths, n, window, want, more


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention(case, dtype):
    cache, q, tables, lengths, n, window, want, more = attention_case(case, dtype)
    got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), window=window, sums=True, longest=max(lengths), **more)
    weight = 2.0 ** -15 + (2.0 ** -11 if max(n) * q.shape[1] // cache.kv_heads > 64 else 0)
    check_attention(got, sums, *want, dtype, weight)
    # a bound that is too small or too large changes the launch, not the result's correctness; without the sums
    for longest, most in ((1, 1), (None, max(n) + 100)):
        if more:
            more["most_queries"], weight = most, 2.0 ** -15 + 2.0 ** -11
        check_attention(cache.attend(q.cuda(), ints(tables), ints(lengths), window=window, longest=longest, **more), None, *want, dtype, weight)


@pytest.fixture
def knobs():
    yield M.set_tuning
    M.set_tuning("attention_kernel", 0)
    M.set_tuning("attention_parts", 0)


@pytest.mark.parametrize("parts", [1, 2, 7, 256])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("case", [3, 11, 13, 15, 17, 19, 20, 22, 23, 24, 25, 26])
def test_attention_by_either_kernel_in_parts(case, kernel, parts, knobs):
    """Both kernels over rows that the other one would be taken for, with more parts than a sequence has tokens for among them."""
    for dtype in TYPES:
        cache, q, tables, lengths, n, window, want, more = attention_case(case, dtype)
        knobs("attention_kernel", kernel)
        knobs("attention_parts", parts)
        got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), window=window, sums=True, longest=max(lengths), **more)
        knobs("attention_kernel", 0)
        knobs("attention_parts", 0)
        check_attention(got, sums, *want, dtype, 2.0 ** -15 + (2.0 ** -11 if kernel == 2 else 0))


@pytest.mark.parametrize("parts", [1, 5])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_over_blocks_of_far_apart_scales(dtype, kernel, parts, knobs):
    """Values whose blocks lie far apart, the largest first, last, or seen by few of the rows; the smallest bytes."""
    g = rng(16)
    page, dim, n, heads, queries = 16, 96, 600, 3, 50
    cache = M.KvCache8(38, page, 1, dim)
    tables = sequences(g, cache, [n])
    fill(g, cache, tables, [n])
    q = normal(g, queries, heads, dim, dtype=dtype)
    order = torch.from_numpy(tables[0, :38])
    for first, middle, last in ((110, 110, 110), (123, 110, 83), (83, 110, 123), (110, 125, 110), (50, 83, 50), (103, 116, 104), (0, 1, 3), (90, 90, 1)):
        cache.scales[order[:19], ..., 1], cache.scales[order[19:30], ..., 1], cache.scales[order[30:], ..., 1] = first, middle, last
        knobs("attention_kernel", kernel)
        knobs("attention_parts", parts)
        for window in (0, 100):
            want, total, reach, far = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n], [0, queries], window=window)
            got = cache.attend(q.cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, window=window, longest=n)
            # by the largest value that a row sees: what lies far below it counts for as much as its weight's rounding, no more
            close(got, want, dtype, (2 * (reach * 2.0 ** -16 + 2.0 ** -15 + (2.0 ** -11 if kernel == 2 else 0)) * far)[..., None])


def test_attention_a_long_sequence_and_its_parts():
    """One sequence of 40001 tokens; and the same as two parts joined by their sums."""
    g = rng(77)
    page, dim, heads, kv_heads, n = 64, 128, 8, 2, 40001
    cache = pool(g, -(-n // page), page, kv_heads, dim)
    tables = sequences(g, cache, [n])
    fill(g, cache, tables, [n])
    q = normal(g, 1, heads, dim)
    want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n])
    got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), sums=True, longest=n)
    check_attention(got, sums, *want, torch.float16)
    cut = 250 * page
    parts = [cache.attend(q.cuda(), ints(t), ints([m]), sums=True) for t, m in ((tables[:, :250], cut), (tables[:, 250:], n - cut))]
    w = torch.softmax(torch.stack([s for _, s in parts]).double(), 0)[..., None]
    joined = to_numpy(sum(o.double() * x for (o, _), x in zip(parts, w)))
    assert np.linalg.norm(joined - want[0]) <= 2.0 ** -11 * np.linalg.norm(want[0])


@pytest.mark.parametrize("asked", [3, 20, 150])
@pytest.mark.parametrize("dim", [128, 96])
def test_attention_what_is_masked_has_no_effect(dim, asked):
    """NaN in keys and values of tokens that a query does not see: later ones, those before the window, the rest of pages, table entries that are not needed."""
    g = rng(8)
    page, heads, kv_heads, length, window = 16, 4, 2, 190, 30
    clean, dirty = (pool(rng(i), 16, page, kv_heads, dim) for i in (1, 2))
    tables = sequences(g, clean, [length])
    k, v = fill(rng(9), clean, tables, [length])
    last, early = length - 2, length - asked - 25                     # seen by the last two queries; by those whose window reaches it
    k2, v2 = k.clone(), v.clone()
    for t in (last, early):
        k2[t, 1], v2[t] = float("nan"), float("nan")
        v2[t, 0, 40:] = 1.0
    dirty.append(None, k2.cuda(), v2.cuda(), None, ints(tables), ints([length]), start=ints([0, length]))
    q = normal(g, asked, heads, dim)
    call = dict(start=ints([0, asked]), most_queries=asked, window=window, sums=True)
    first = (length - asked - window + 1) // page
    tables[0, :max(first, 0)] = 2 ** 30                               # in front of every window
    want, total = clean.attend(q.cuda(), ints(tables), ints([length]), **call)
    got, sums = dirty.attend(q.cuda(), ints(tables), ints([length]), **call)
    place = length - asked + np.arange(asked)
    sees = (place >= last) | ((place >= early) & (place - window < early))
    assert sees.any() and (asked < 20 or not sees.all())
    rest = torch.from_numpy(~sees)
    # whether a block is gone through a second time may change the last place; the blocks' scales are the same
    assert (got[rest].double() - want[rest].double()).abs().max() <= 2.0 ** -9 if rest.any() else True
    assert (sums[rest] - total[rest]).abs().max() <= 2.0 ** -12 if rest.any() else True
    reference = ref.attend_cached(to_numpy(q), *content(dirty), page, np.where(tables > 16, 0, tables), [length], [0, asked], window=window)
    assert np.array_equal(np.isnan(to_numpy(got)), np.isnan(reference[0])) and np.isnan(reference[0][sees]).any((1, 2)).all()
    fine = ~np.isnan(reference[0])
    assert np.linalg.norm(to_numpy(got)[fine] - reference[0][fine]) <= 2.0 ** -11 * np.linalg.norm(reference[0][fine])


def test_attention_pages_that_are_needed_and_missing():
    g = rng(12)
    cache = pool(g, 12, 16, 2, 64)
    lengths = [60, 60, 60, 60, 200]
    tables = np.arange(20).reshape(5, 4) % 12
    fill(g, cache, np.arange(12).reshape(1, 12), [192])
    tables[1, 2], tables[2, 0] = 12, -1
    q = normal(g, 5, 4, 64)
    got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), sums=True)
    bad = torch.isnan(got).all(2).all(1).cpu().tolist()
    assert bad == [False, True, True, False, True] and torch.isnan(sums).all(1).cpu().tolist() == bad
    assert not torch.isnan(got[[0, 3]]).any()
    assert torch.isnan(cache.attend(q.cuda(), ints(np.zeros((5, 0))), ints(lengths))).all()
    empty = M.KvCache8(0, 16, 2, 64)
    assert torch.isnan(empty.attend(q.cuda(), ints(tables), ints(lengths))).all()
    none = empty.attend(q.cuda(), ints(tables), ints([0, 0, -3, 0, 0]))
    assert torch.equal(none, torch.zeros_like(none))


@pytest.mark.parametrize("queries", [1, 100])
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_large_and_extreme_scores(dtype, queries):
    """Scores that grow along the sequence, negative and zero scales, blocks whose scales differ by far, a sink far ahead of all others whose value is small."""
    g = rng(14)
    page, dim, n = 16, 64, 400
    cache = pool(g, 25, page, 1, dim)
    tables = sequences(g, cache, [n])
    k, v = normal(g, n, 1, dim, dtype=dtype), normal(g, n, 1, dim, dtype=dtype)
    k += (torch.linspace(-3, 3, n)[:, None, None]).to(dtype)
    v *= torch.exp2(torch.randint(-6, 6, (n // 16, 1, 1), generator=g).float()).repeat_interleave(16, 0).to(dtype)
    cache.append(None, k.cuda(), v.cuda(), None, ints(tables), ints([n]), start=ints([0, n]))
    q = normal(g, queries, 4, dim, dtype=dtype) + 1
    data = content(cache)
    for scale in (1.0, -1.0, 0.0, 0.01, 2.0 ** -130, 7.5):
        want = ref.attend_cached(to_numpy(q), *data, page, tables, [n], [0, queries], scale=scale)
        got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, scale=scale, sums=True)
        check_attention(got, sums, *want, dtype, 2.0 ** -15 + (2.0 ** -11 if queries > 16 else 0))


@pytest.mark.parametrize("queries", [1, 70])
def test_attention_a_token_far_ahead_of_many(queries):
    """A first token 2^20 ahead of 20000 others, with a value of almost nothing: what the others sum up to is kept, in the results and in the sums."""
    g = rng(15)
    page, dim, n = 64, 32, 20000
    cache = M.KvCache8(-(-n // page), page, 1, dim)
    tables = sequences(g, cache, [n])
    k, v = torch.zeros((n, 1, dim)), 1.0 + torch.rand((n, 1, dim), generator=g)
    k[0, 0, 0], v[0] = 14.0, 0.0
    cache.append(None, k.half().cuda(), v.half().cuda(), None, ints(tables), ints([n]), start=ints([0, n]))
    q = torch.zeros((queries, 2, dim))
    q[..., 0] = 1.0
    want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n], [0, queries], scale=1.0)
    got, sums = cache.attend(q.half().cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, scale=1.0, sums=True)
    err = np.abs(to_numpy(got) - want[0]).max(-1) / np.abs(want[0]).max(-1)
    assert err.max() <= 2.0 ** -11 + 2.0 ** -13
    assert np.abs(to_numpy(sums) - want[1]).max() <= 2.0 ** -15


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_streams_outputs_and_rows_of_no_sequence(dtype):
    g = rng(31)
    page, dim, heads, kv_heads = 16, 96, 4, 2
    lengths, start = [40, 25], [2, 7, 10]
    cache = pool(g, 8, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths, dtype)
    q = normal(g, 12, heads, dim, dtype=dtype)
    want = ref.attend_cached(to_numpy(q)[2:10], *content(cache), page, tables, lengths, [0, 5, 8])
    odd = torch.empty(12 * (heads + 1) * (dim + 1) + 1, dtype=dtype, device="cuda")[1:].view(12, heads + 1, dim + 1)[:, :heads, :dim]       # 2 bytes off every boundary
    odd.copy_(q)
    out = torch.full((12, heads, dim + 3), 7.0, dtype=dtype, device="cuda")
    wide = torch.full((2, tables.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:-2] = ints(tables)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = cache.attend(odd, wide[:, 3:-2], ints(lengths), start=ints(start), most_queries=5, out=out[..., :dim], stream=other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    close(got[2:10], want[0], dtype, (2 * (want[2] * 2.0 ** -16 + 2.0 ** -15) * want[3])[..., None])
    assert (out[..., dim:] == 7).all()
    for bad in (dict(q=q.cuda().float()), dict(q=q.cuda()[:, :3]), dict(lengths=ints(lengths).long()), dict(tables=ints(tables)[0]), dict(start=ints([0, 1])), dict(window=2 ** 40)):
        call = dict(dict(q=q.cuda(), tables=ints(tables), lengths=ints(lengths), start=ints(start)), **bad)
        with pytest.raises((TypeError, ValueError, M.MackoError)):
            cache.attend(**call)


@pytest.mark.parametrize("parts", [1, 3, 40])
@pytest.mark.parametrize("kernel", [1, 2])
def test_rows_of_no_sequence_stay_as_they_were(kernel, parts, knobs):
    """In front of the first sequence and behind the last one, with results joined from parts in a workspace of any content."""
    g = rng(32)
    page, dim, heads, kv_heads, lengths, start = 16, 64, 6, 2, [700, 3, 900], [3, 30, 33, 60]
    cache = pool(g, 110, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    q = normal(g, 75, heads, dim)
    want, total, reach, far = ref.attend_cached(to_numpy(q)[3:60], *content(cache), page, tables, lengths, [s - 3 for s in start])
    knobs("attention_kernel", kernel)
    knobs("attention_parts", parts)
    for junk in (1, -1, 2 ** 30):                                      # what the allocator gives the call next
        size = 75 * heads * 256 * (dim + 3) // 4
        del_me = [torch.full((size // n,), junk, dtype=torch.int32, device="cuda") for n in (1, 2, 4, 8, 16)]
        torch.cuda.synchronize()
        del del_me
        out = torch.full((75, heads, dim), 7.0, dtype=torch.float16, device="cuda")
        got = cache.attend(q.cuda(), ints(tables), ints(lengths), start=ints(start), most_queries=27, longest=900, out=out)
        assert (got[:3] == 7).all() and (got[60:] == 7).all()
        close(got[3:60], want, torch.float16, (2 * (reach * 2.0 ** -16 + 2.0 ** -15 + (2.0 ** -11 if kernel == 2 else 0)) * far)[..., None])


def test_a_graph_of_steps():
    """Append and attend in a captured graph, replayed with lengths that grow, with eager work between the replays."""
    g = rng(40)
    page, dim, heads, kv_heads, batch = 16, 128, 8, 2, 3
    one, two = (M.KvCache8(30, page, kv_heads, dim) for _ in range(2))
    tables = ints(np.arange(30).reshape(batch, 10))
    lengths = ints([5, 30, 15])
    tab = M.rope_table(200, dim)
    for cache in (one, two):
        fill(rng(41), cache, np.arange(30).reshape(batch, 10), [5, 30, 15])
    q, k, v = (normal(g, batch, h, dim).cuda() for h in (heads, kv_heads, kv_heads))
    place = lengths.clone()

    def step(cache):
        lengths.add_(1)
        turned = cache.append(q, k, v, place, tables, lengths, table=tab)
        return cache.attend(turned, tables, lengths, longest=160)

    kept = lengths.clone()
    step(one)                                                          # what is made once is made outside
    lengths.copy_(kept)
    fill(rng(41), one, np.arange(30).reshape(batch, 10), [5, 30, 15])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(one)
    for i in range(20):
        for x in (q, k, v):
            x.copy_(normal(g, *x.shape))
        lengths.copy_(kept + i)
        place.copy_(lengths)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        lengths.copy_(kept + i)
        want = step(two)
        assert torch.equal(got, want), i
    held = [torch.cat([x[tables[b].long()].transpose(1, 2).flatten(0, 1)[:-(-(int(n) + 20) // 16)] for b, n in enumerate([5, 30, 15])]) for x in (one.scales, two.scales)]
    assert torch.equal(*held)


def test_the_run_of_a_layer():
    """A prompt, then single tokens: every step's attention against the same over what the cache holds, and against the values before they were rounded."""
    g = rng(50)
    page, dim, heads, kv_heads, n, steps = 16, 64, 8, 2, 45, 25
    cache = M.KvCache8(8, page, kv_heads, dim)
    table = ints([[5, 2, 7, 0, 1]])
    tab = M.rope_table(200, dim)
    q, k, v = (normal(g, n + steps, h, dim) for h in (heads, kv_heads, kv_heads))
    turned = [ref4.rotate(to_numpy(x), np.arange(n + steps), tab.cpu().numpy()) for x in (q, k)]
    done = 0
    for m in [n] + [1] * steps:
        rows = slice(done, done + m)
        done += m
        at, lengths, start = ints(np.arange(done - m, done)), ints([done]), ints([0, m])
        mine = cache.append(q[rows].cuda(), k[rows].cuda(), v[rows].cuda(), at, table, lengths, start=start, table=tab)
        got = cache.attend(mine, table, lengths, start=start, most_queries=m)
        held = ref.attend_cached(to_numpy(mine), *content(cache), page, table.cpu().numpy(), [done], [0, m])
        check_attention(got, None, *held, torch.float16)
        exact = ref.attend(turned[0][rows], turned[1][:done], to_numpy(v)[:done], done - m)[0]
        # E4M3 keeps 4 bits: a key or value is off by 2^-4 of itself at most, 2^-5.4 in the mean; scores here have a spread of 1
        assert np.linalg.norm(to_numpy(got) - exact) <= 2.0 ** -4 * np.linalg.norm(exact)


def test_the_example_runs_the_operators_together(capsys):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # 16-bit results of a computation in 32 bits: half a unit in the last place
    assert example.main(["--tokens", "150", "--steps", "5", "--hidden", "512", "--inner", "1000", "--heads", "8", "--kv-heads", "2", "--bits", "8"]) <= 2.0 ** -11
    assert "8.01 bits a value" in capsys.readouterr().out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [40, 700])
def test_append_strides_streams_and_queries_in_place(tokens, dtype):
    """Tensors off every boundary, queries over themselves, another stream, a captured call that is replayed: all as the plain call, in the pool byte by byte."""
    g = rng(tokens)
    page, dim, heads, kv_heads = 16, 96, 5, 8
    tables, lengths, start = ints(np.arange(50)[None]), ints([tokens + 30]), ints([0, tokens])
    tab, w = M.rope_table(800, 64), normal(g, dim, dtype=dtype).cuda()
    at = torch.randint(0, 800, (tokens,), generator=g).to(torch.int32).cuda()
    x = [normal(g, tokens, h, dim, dtype=dtype).cuda() for h in (heads, kv_heads, kv_heads)]
    more = dict(start=start, table=tab, q_weight=w, k_weight=w, eps=1e-5)
    first = pool(rng(1), 50, page, kv_heads, dim)
    want = first.append(*x, at, tables, lengths, **more)
    same = lambda cache, got: torch.equal(cache.data, first.data) and torch.equal(cache.scales, first.scales) and torch.equal(got.nan_to_num(9.0), want.nan_to_num(9.0))  # noqa: E731

    def odd(t):
        return torch.empty(tokens * (t.shape[1] + 1) * (dim + 1) + 1, dtype=dtype, device="cuda")[1:].view(tokens, t.shape[1] + 1, dim + 1)[:, :t.shape[1], :dim].copy_(t)

    cache = pool(rng(1), 50, page, kv_heads, dim)
    moved = [odd(t) for t in x]
    got = cache.append(*moved, at, tables, lengths, q_out=moved[0], **more)
    assert got.data_ptr() == moved[0].data_ptr() and same(cache, got)
    cache, other = pool(rng(1), 50, page, kv_heads, dim), torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = cache.append(*x, at, tables, lengths, stream=other, **more)
    torch.cuda.current_stream().wait_stream(other)
    assert same(cache, got)
    cache = pool(rng(1), 50, page, kv_heads, dim)
    data, scales = cache.data.clone(), cache.scales.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = cache.append(*x, at, tables, lengths, **more)
    for _ in range(3):
        cache.data.copy_(data)
        cache.scales.copy_(scales)
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(cache, got)
    slots = ints(np.arange(50 * page)[::-1].copy())
    plain = cache.read(slots, dtype)
    side = cache.read(slots, dtype, stream=other)
    torch.cuda.synchronize()
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(plain, side))
    for bad in (dict(k=x[1].float()), dict(v=x[2][:, :3]), dict(lengths=lengths.long()), dict(start=ints([0, 1, 2])), dict(positions=at[:-1]), dict(q=x[0][:-1]), dict(tables=tables[0])):
        call = dict(dict(q=x[0], k=x[1], v=x[2], positions=at, tables=tables, lengths=lengths), **dict(more, **bad))
        with pytest.raises((TypeError, ValueError, M.MackoError)):
            cache.append(**call)


@pytest.mark.parametrize("parts", [1, 4])
@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("dim", [64, 128, 160])
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_many_rows_that_need_missing_pages(dtype, dim, kernel, parts, knobs):
    """Entries that name no page, and a table that is too short, with a page 0 whose values are not numbers: their sequences' rows are NaN, the others' as ever."""
    g = rng(dim + 1)
    page, heads, kv_heads, asked = 16, 4, 2, 40                        # 80 rows on a key/value head
    lengths = [100, 130, 90, 200, 140, 60]
    cache = pool(g, 60, page, kv_heads, dim)
    tables = np.full((6, 13), -1)
    for b, n in enumerate(lengths):
        tables[b, :-(-n // page)] = 1 + np.arange(-(-n // page)) + sum(-(-m // page) for m in lengths[:b])
    fill(g, cache, tables, lengths, dtype)
    cache.data[0, :, :, 1] = 0x7F
    for b, entry in ((0, -1), (1, 60), (2, 2 ** 30), (4, -2 ** 31)):
        tables[b, 2] = entry                                           # tokens that every query sees
    q = normal(g, 6 * asked, heads, dim, dtype=dtype)
    start = np.arange(7) * asked
    for table, missing in ((tables, [0, 1, 2, 4]), (tables[:, :9], [0, 1, 2, 3, 4]), (tables[:, :0], range(6))):
        want = ref.attend_cached(to_numpy(q), *content(cache), page, table, lengths, start)
        assert [b for b in range(6) if np.isnan(want[0][b * asked:(b + 1) * asked]).all()] == list(missing)
        knobs("attention_kernel", kernel)
        knobs("attention_parts", parts)
        got, sums = cache.attend(q.cuda(), ints(table), ints(lengths), start=ints(start), most_queries=asked, longest=200, sums=True)
        check_attention(got, sums, *want, dtype, 2.0 ** -15 + (2.0 ** -11 if kernel != 1 else 0))


@pytest.mark.parametrize("parts", [1, 3, 256])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("dim", [64, 96, 192])
@pytest.mark.parametrize("dtype", TYPES)
def test_sums_are_of_the_weights_before_they_are_rounded(dtype, dim, kernel, parts, knobs):
    """Few tokens that hold nearly all of a row's weight, none of them a power of two in units of the first large one: rounded to 11 bits their sum is off by up to 2^-11."""
    g = rng(61)
    page, heads, queries, n = 32, 2, 40, 2000
    cache = M.KvCache8(-(-n // page), page, 1, dim)
    tables = sequences(g, cache, [n])
    k, v = torch.zeros((n, 1, dim), dtype=dtype), normal(g, n, 1, dim, dtype=dtype)
    k[..., 0] = -8.0
    k[10::200, :, 0], k[150::200, :, 0] = 1.0, 3.0                      # 2^2.9 to 2^4.9 times the weight of the first
    cache.append(None, k.cuda(), v.cuda(), None, ints(tables), ints([n]), start=ints([0, n]))
    q = torch.zeros((queries, heads, dim), dtype=dtype)
    q[..., 0] = 1.0 + torch.arange(queries * heads).view(queries, heads) / 118.0
    want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n], [0, queries], scale=1.0)
    knobs("attention_kernel", kernel)
    knobs("attention_parts", parts)
    call = dict(start=ints([0, queries]), most_queries=queries, scale=1.0, longest=n)
    got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), sums=True, **call)
    for x in (got, cache.attend(q.cuda(), ints(tables), ints([n]), **call)):
        check_attention(x, None, *want, dtype, 2.0 ** -15 + (2.0 ** -11 if kernel == 2 else 0))
    # a weight is off by the rounding of its exponent, 8 bits in front of the point at most, and of its own, its sum by less: 2^-16 of them; the logarithm's result of at most 9 by 2^-21
    assert np.abs(to_numpy(sums) - want[1]).max() <= 2.0 ** -15


@pytest.mark.parametrize("parts", [1, 5])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("dtype", TYPES)
def test_sums_of_a_token_2_to_the_30_ahead_of_131072(dtype, kernel, parts, knobs):
    """Steps of 64 tokens, 2^5 of weight to a lane, that leave a sum in 32 bits above 2^30 as it was: half of the others would be lost, 2^-14 of the sum."""
    page, dim, n, queries = 64, 32, 131072, 70
    cache = M.KvCache8(n // page, page, 1, dim)
    tables = np.arange(n // page)[None]
    k, v = torch.zeros((n, 1, dim)), torch.ones((n, 1, dim))
    k[0, 0, 0], v[0] = 20.0, 0.0                                       # a number of E4M3
    cache.append(None, k.to(dtype).cuda(), v.to(dtype).cuda(), None, ints(tables), ints([n]), start=ints([0, n]))
    q = torch.zeros((queries, 1, dim))
    q[..., 0] = 1.046875                                               # 20.9375, 2^30.2
    knobs("attention_kernel", kernel)
    knobs("attention_parts", parts)
    got, sums = cache.attend(q.to(dtype).cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, scale=1.0, longest=n, sums=True)
    others = n - queries + np.arange(queries)[:, None].astype(np.float64)
    top = np.exp(20.9375)
    assert np.abs(to_numpy(sums) - np.log(top + others)).max() <= 2.0 ** -16
    want = others / (top + others)
    assert np.all(np.abs(to_numpy(got) - want[..., None]) <= want[..., None] * (HALF[dtype] + 2.0 ** -13) + TINY[dtype])


@pytest.mark.parametrize("parts", [1, 3])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("dim", [64, 128, 160])
@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_of_zeros_have_no_scale(dtype, dim, kernel, parts, knobs):
    """Values of whole blocks that are zero: whatever their byte of scale is, results are the same bit by bit."""
    g = rng(62)
    page, heads, queries, n = 64, 3, 40, 2300
    cache = M.KvCache8(36, page, 1, dim)
    tables = sequences(g, cache, [n])
    fill(g, cache, tables, [n], dtype)
    q = normal(g, queries, heads, dim, dtype=dtype)
    order = torch.from_numpy(tables[0, :36]).cuda()
    data = cache.data.clone()
    knobs("attention_kernel", kernel)
    knobs("attention_parts", parts)
    for zeros in ([0], [1, 2], range(5), range(80), [70, 90, 143], [143], range(66, 144)):
        block = torch.zeros(144, dtype=torch.bool, device="cuda")
        block[list(zeros)] = True
        cache.data.copy_(data)
        codes = cache.data[order]                                      # [36 pages, 1, 4 blocks, 2, 16 dim]
        codes[:, 0, :, 1][block.view(36, 4)] = torch.randint(0, 2, (int(block.sum()), 16 * dim), generator=g, dtype=torch.uint8).cuda() * 0x80      # of either sign
        cache.data[order] = codes
        got = []
        for byte in (110, 1, 0, 30, 200):
            scales = cache.scales[order]
            scales[:, 0, :, 1] = torch.where(block.view(36, 4), byte, 110).to(torch.uint8)
            cache.scales[order] = scales
            got.append(cache.attend(q.cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, longest=n, sums=True))
        want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n], [0, queries])
        # element by element: results of some 2^-14, where fp16's numbers are 2^-24 apart, are off by 2^-25, however small they are
        close(got[0][0], want[0], dtype, (2 * (want[2] * 2.0 ** -16 + 2.0 ** -15 + (2.0 ** -11 if kernel == 2 else 0)) * want[3])[..., None])
        assert np.all(np.abs(to_numpy(got[0][1]) - want[1]) <= want[2] * 2.0 ** -16 + np.abs(want[1]) * 2.0 ** -21 + 2.0 ** -15)
        for x, s in got[1:]:
            assert torch.equal(x, got[0][0]) and torch.equal(s, got[0][1]), list(zeros)[:3]


@pytest.mark.parametrize("parts", [1, 3, 40])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("dtype", TYPES)
def test_sums_of_rows_of_no_sequence_stay_too(dtype, bits, kernel, parts, knobs):
    """Results and sums in memory of the caller's, over both caches and packed: rows in front of the first sequence and behind the last one stay as they were."""
    import ctypes

    from paper_2511_13061_amd import kv
    g = rng(33)
    page, dim, heads, kv_heads, tokens, lengths, start = 16, 64, 6, 2, 75, [700, 0, 900], [3, 30, 33, 60]
    q = normal(g, tokens, heads, dim, dtype=dtype).cuda()
    out = torch.full((tokens, heads, dim), 7.0, dtype=dtype, device="cuda")
    sums = torch.full((tokens, heads), 7.0, device="cuda")
    lib, kind, stream = M.load_library(), int(dtype == torch.bfloat16), torch.cuda.current_stream().cuda_stream
    rows = ints(start)
    if bits == 16:
        k, v = (normal(g, tokens, kv_heads, dim, dtype=dtype).cuda() for _ in range(2))
        a = kv._CPrompt(tokens, heads, kv_heads, dim, kind, 3, q.data_ptr(), heads * dim, dim, k.data_ptr(), kv_heads * dim, dim, v.data_ptr(), kv_heads * dim, dim,
                        out.data_ptr(), heads * dim, dim, sums.data_ptr(), rows.data_ptr(), 0, 30, dim ** -0.5)
        assert lib.macko_prompt_attention(ctypes.byref(a), stream) == 0
    else:
        cache = (M.KvCache if bits == 4 else M.KvCache8)(110, page, kv_heads, dim)
        tables = sequences(g, cache, lengths)
        k, v = (normal(g, 110 * page, kv_heads, dim).cuda() for _ in range(2))
        if bits == 4:
            cache.append(None, k, v, None, ints(np.arange(110 * page)))
        else:
            cache.append(None, k, v, None, ints([range(110)]), ints([110 * page]), start=ints([0, 110 * page]))
        table, length = ints(tables), ints(lengths)
        a = kv._CAttention(tokens, heads, kind, 3, q.data_ptr(), heads * dim, dim, out.data_ptr(), heads * dim, dim, sums.data_ptr(), table.data_ptr(), table.stride(0),
                           table.shape[1], length.data_ptr(), rows.data_ptr(), 27, 0, 900, dim ** -0.5)
        name = "macko_kv_attention" if bits == 4 else "macko_kv8_attention"
        knobs("attention_kernel", kernel)
        knobs("attention_parts", parts)
        size = getattr(lib, name + "_workspace")(cache._p, ctypes.byref(a))
        assert (size > 0) == (parts > 1)
        for junk in (1, -1, 2 ** 30):
            work = torch.full((size // 4,), junk, dtype=torch.int32, device="cuda")
            assert getattr(lib, name)(cache._p, ctypes.byref(a), work.data_ptr() if size else None, size, stream) == 0
    torch.cuda.synchronize()
    outside = torch.ones(tokens, dtype=torch.bool)
    outside[3:60] = False
    assert (out[outside] == 7).all() and (sums[outside] == 7).all()
    assert not (sums[~outside] == 7).any() and not (out[~outside] == 7).all(2).any()


@pytest.mark.parametrize("parts", [1, 5])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("byte", [1, 6, 12, 20])
def test_values_of_the_least_scales(byte, kernel, parts, knobs):
    """Values near the end of bf16's range, in the mean of very many: results are far above what 32 bits leave of one over the sum of weights, times the scale."""
    g = rng(63)
    page, dim, n, heads, queries = 64, 64, 20000, 2, 40
    cache = M.KvCache8(-(-n // page), page, 1, dim)
    tables = sequences(g, cache, [n])
    k, v = torch.zeros((n, 1, dim)), 1.0 + torch.rand((n, 1, dim), generator=g)
    cache.append(None, k.bfloat16().cuda(), v.bfloat16().cuda(), None, ints(tables), ints([n]), start=ints([0, n]))
    cache.scales[..., 1] = byte
    q = normal(g, queries, heads, dim, dtype=torch.bfloat16)
    want = ref.attend_cached(to_numpy(q), *content(cache), page, tables, [n], [0, queries])
    knobs("attention_kernel", kernel)
    knobs("attention_parts", parts)
    got = cache.attend(q.cuda(), ints(tables), ints([n]), start=ints([0, queries]), most_queries=queries, longest=n)
    # keys of zero: all weights are alike, and what they are rounded to cancels out; sums of 20000 in 32 bits
    close(got, want[0], torch.bfloat16, np.abs(want[0]) * 2.0 ** -12)
