"""Rotation, the 4-bit key/value cache and attention over it, on the GPU, against tests/kv_reference.py (64 bits).

Tolerances.  A result of 16 bits is off by at most half a unit in the last place, 2^-11 (fp16) or 2^-8 (bf16) of it, from what was
computed.  What was computed: rotation and norm in 32 bits, some ten roundings, 2^-20 of the largest product that enters.  Attention:
a score is off by at most 2^-13 of the sum of its products' magnitudes (the matrix cores line 8-bit products of very different size
up before they add them), so a weight by the same share of it times scale, numerator and denominator alike, and a weight goes in with 16 bits."""
import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
M = pytest.importorskip("paper_2511_13061_amd")

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float16, torch.bfloat16]


def rng(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype=torch.float16, scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)


def ints(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()


def close(got, want, dtype, slack):
    """|got - want| <= half a unit in the last place and slack (an array or a number); NaN and infinities where they belong."""
    got = ref.to_numpy(got)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bound = np.abs(want) * HALF[dtype] * (1 + 2.0 ** -10) + TINY[dtype] + slack
    bad = ~(np.abs(got - want) <= bound) & ~np.isnan(want) & ~(got == want)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the worst by {np.nanmax(np.where(bad, np.abs(got - want) / bound, 0)):.2f} of the bound"


# ---- tables and rotation ------------------------------------------------------

@pytest.mark.parametrize("args", [
    dict(length=300, rot=128), dict(length=1, rot=2), dict(length=57, rot=96, base=500000.0, first=131000), dict(length=64, rot=64, amplitude=1.25),
    dict(length=200, rot=128, factor=4.0), dict(length=200, rot=128, factor=8.0, trained=4096, low=1.0, high=32.0),
    dict(length=90, rot=64, factor=2.5, trained=2048, low=4.0, high=4.0, first=70000), dict(length=0, rot=32)])
def test_rope_table(args):
    got = M.rope_table(**args).cpu().numpy()
    want = ref.table(**args)
    assert got.shape == want.shape and got.dtype == np.float32
    # 64-bit angles are off by 2^-50 of themselves, the result is rounded once
    angle = args["length"] + args.get("first", 0)
    assert np.all(np.abs(got - want) <= np.abs(want) * 2.0 ** -24 + angle * 2.0 ** -49 + 2.0 ** -149)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,rot,norm", [
    (1, 32, 128, 128, False), (7, 3, 128, 64, True), (3, 1, 32, 16, True), (5, 2, 64, 64, False), (65, 5, 96, 96, True), (2, 7, 96, 32, False),
    (4, 9, 160, 80, True), (3, 2, 192, 192, False), (6, 3, 224, 16, True), (9, 4, 256, 256, True), (1000, 33, 64, 48, True), (2, 3, 128, 0, True)])
def test_rotate(tokens, heads, dim, rot, norm, interleaved, dtype):
    g = rng(tokens * 1000 + dim + rot)
    x = normal(g, tokens, heads, dim, dtype=dtype, scale=3.0)
    x[0, 0] = 0                                                  # a head without anything: eps keeps it finite
    w = normal(g, dim, dtype=dtype) if norm else None
    tab = M.rope_table(500, rot, first=3) if rot else None
    at = torch.randint(0, 500, (tokens,), generator=g)
    got = M.rotate(x.cuda(), ints(at) if rot else None, tab, weight=w.cuda() if norm else None, eps=1e-5, interleaved=interleaved)
    want = ref.rotate(ref.to_numpy(x), at.numpy(), tab.cpu().numpy() if rot else None, ref.to_numpy(w) if norm else None, 1e-5, interleaved)
    assert got.dtype == dtype
    size = np.abs(ref.rotate(np.abs(ref.to_numpy(x)), at.numpy(), None, np.abs(ref.to_numpy(w)) if norm else None, 1e-5)).max(-1, keepdims=True)
    close(got, want, dtype, size * 2.0 ** -20)


def test_rotate_strides_place_and_positions_outside_the_table():
    g = rng(5)
    tab = M.rope_table(40, 128)
    at = torch.tensor([0, 39, 40, -1, 7, 2 ** 31 - 1, -2 ** 31, 3])
    fused = normal(g, 8, 6, 128).cuda()
    want = ref.rotate(ref.to_numpy(fused), at.numpy(), tab.cpu().numpy())
    assert np.isnan(want[[2, 3, 5, 6]]).all()
    slack = np.abs(ref.to_numpy(fused)).max() * 2.0 ** -20
    close(M.rotate(fused[:, 1:4], ints(at), tab), want[:, 1:4], torch.float16, slack)                 # a part of a projection's output
    flipped = fused.transpose(0, 1).contiguous().transpose(0, 1)                                      # heads outside, tokens inside
    close(M.rotate(flipped, ints(at), tab), want, torch.float16, slack)
    odd = torch.empty(8 * 6 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(8, 6, 128)        # 2 bytes off every boundary
    odd.copy_(fused)
    out = torch.full((8 * 6 * 131 + 3,), 7.0, dtype=torch.float16, device="cuda")
    view = out[3:3 + 8 * 6 * 131].view(8, 6, 131)[:, :, :128]
    M.rotate(odd, ints(at), tab, out=view)
    close(view, want, torch.float16, slack)
    assert (out[:3] == 7).all() and (out[3:].view(8, 6, 131)[:, :, 128:] == 7).all()                 # nothing beside the heads
    same = fused.clone()
    assert M.rotate(same, ints(at), tab, out=same) is same                                            # in place
    close(same, want, torch.float16, slack)
    one = M.rotate(fused[:1].expand(8, 6, 128), ints(at), tab)                                        # one row for all tokens
    close(one, ref.rotate(np.broadcast_to(ref.to_numpy(fused[:1]), (8, 6, 128)), at.numpy(), tab.cpu().numpy()), torch.float16, slack)
    assert M.rotate(fused[:0], ints([]), tab).shape == (0, 6, 128)
    assert M.rotate(fused[:, :0], ints(at), tab).shape == (8, 0, 128)


def test_rotate_infinities_and_nan_stay_in_their_head():
    g = rng(6)
    x = normal(g, 4, 3, 64)
    x[1, 1, 5], x[2, 0, 7] = float("inf"), float("nan")
    tab = M.rope_table(16, 64)
    got = ref.to_numpy(M.rotate(x.cuda(), ints([1, 2, 3, 4]), tab))
    clean = [(t, h) for t in range(4) for h in range(3) if (t, h) not in ((1, 1), (2, 0))]
    assert all(np.isfinite(got[t, h]).all() for t, h in clean)
    bad = ~np.isfinite(got)
    assert set(np.argwhere(bad[1, 1]).ravel()) == {5, 37} and set(np.argwhere(bad[2, 0]).ravel()) == {7, 39}


# ---- the cache ----------------------------------------------------------------

def pool(g, pages, page, heads, dim):
    """A pool of random bytes: what nobody wrote has to stay as it is and to have no effect."""
    data = torch.randint(0, 256, (pages, heads, ref.piece_bytes(page, dim)), generator=g, dtype=torch.uint8).cuda()
    return M.KvCache(pages, page, heads, dim, data=data)


def slot_bytes(page, dim, slots):
    """Which bytes of a piece belong to these slots of a page."""
    mine = np.zeros(ref.piece_bytes(page, dim), dtype=bool)
    for t in slots:
        (kb, _), (vb, _), kg, vg = ref.addresses(page, dim, t, np.arange(dim))
        for i in (kb, vb, kg, vg):
            mine[i] = True
    return mine


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,page,rot,norm,interleaved", [
    (1, 4, 4, 128, 16, 128, False, False), (37, 10, 2, 64, 32, 32, True, False), (20, 3, 3, 32, 16, 32, False, True), (50, 4, 1, 96, 64, 96, True, True),
    (33, 0, 2, 160, 16, 0, False, False), (19, 6, 3, 192, 128, 64, True, False), (18, 2, 1, 224, 16, 224, False, False), (40, 8, 8, 256, 16, 128, True, True)])
def test_append_and_read(tokens, heads, kv_heads, dim, page, rot, norm, interleaved, dtype):
    g = rng(tokens * 100 + dim)
    pages = -(-tokens // page) + 2
    cache = pool(g, pages, page, kv_heads, dim)
    before = cache.data.cpu().numpy().copy()
    fused = normal(g, tokens, heads + 2 * kv_heads, dim, dtype=dtype, scale=2.0)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    slots = torch.randperm(pages * page, generator=g)[:tokens].numpy()
    if tokens > 4:
        slots[3], slots[4] = -1, pages * page                    # padding, and a slot that does not exist
    wq, wk = (normal(g, dim, dtype=dtype) if norm else None for _ in range(2))
    tab = M.rope_table(100, rot) if rot else None
    at = torch.randint(0, 100, (tokens,), generator=g).numpy()
    if tokens > 6 and rot:
        at[6] = 100                                              # a position that the table does not have: not stored, q is NaN
    dev = fused.cuda()
    got = cache.append(dev[:, :heads] if heads else None, dev[:, heads:heads + kv_heads], dev[:, heads + kv_heads:], ints(at) if rot else None, ints(slots), tab,
                       q_weight=wq.cuda() if norm else None, k_weight=wk.cuda() if norm else None, eps=1e-5, interleaved=interleaved)
    t64 = tab.cpu().numpy() if rot else None
    w64 = [ref.to_numpy(w) if norm else None for w in (wq, wk)]
    if heads:
        want = ref.rotate(ref.to_numpy(q), at, t64, w64[0], 1e-5, interleaved)
        size = np.abs(ref.rotate(np.abs(ref.to_numpy(q)), at, None, None if w64[0] is None else np.abs(w64[0]), 1e-5)).max(-1, keepdims=True)
        close(got, want, dtype, size * 2.0 ** -20)
    else:
        assert got is None
    turned = ref.rotate(ref.to_numpy(k), at, t64, w64[1], 1e-5, interleaved)
    stored = (slots >= 0) & (slots < pages * page) & ~np.isnan(turned).any((1, 2))
    # bytes of other slots are untouched, those of padding rows' too
    after = cache.data.cpu().numpy()
    for p in range(pages):
        mine = slot_bytes(page, dim, [s % page for s in slots[stored] if s // page == p])
        assert np.array_equal(after[p][:, ~mine], before[p][:, ~mine])
    keys, values = ref.read(after, page, dim, slots[stored])
    assert np.array_equal(values, ref.nearest(ref.to_numpy(v)[stored]))
    # keys are rounded to 32 bits on the way: where that moves one over the edge between two codes, it is at the edge within 2^-19
    exact = turned[stored]
    size = np.abs(exact).reshape(*exact.shape[:2], -1, 32).max(-1).repeat(32, -1)
    nudged = [ref.nearest(exact * (1 + s)) for s in (-2.0 ** -19, 0.0, 2.0 ** -19)] + [ref.nearest(exact + s * size) for s in (-2.0 ** -20, 2.0 ** -20)]
    assert np.any([keys == x for x in nudged], axis=0).all()
    assert (keys == nudged[1]).mean() > 0.999
    # and back: what the bytes stand for, rounded to 16 bits, zeros for what is not in the pool; in any order
    for out in TYPES:
        some = np.concatenate([slots, [-1, pages * page, 0, pages * page - 1]])
        back = cache.read(ints(some), out)
        for x, y in zip(back, ref.read(after, page, dim, some)):
            assert x.dtype == out and torch.equal(x.cpu().nan_to_num(-77.0), torch.from_numpy(y).to(out).nan_to_num(-77.0))


@pytest.mark.parametrize("dtype", TYPES)
def test_read_of_every_byte_and_code(dtype):
    """All 255 factors with all 16 codes, results beyond the type's range and below it included."""
    page, dim = 16, 64
    data = np.zeros((16, 1, ref.piece_bytes(page, dim)), dtype=np.uint8)
    codes = data[:, 0, :page * dim]
    codes[:] = (np.arange(page * dim)[None] * 37 + np.arange(16)[:, None]) % 256
    data[:, 0, page * dim:page * dim + page * 2] = np.arange(512).reshape(16, 32) % 256
    data[:, 0, page * dim + page * 2:] = (np.arange(512).reshape(16, 32) * 3 + 1) % 256
    cache = M.KvCache(16, page, 1, dim, data=torch.from_numpy(data).cuda())
    slots = np.arange(256)
    for x, y in zip(cache.read(ints(slots), dtype), ref.read(data, page, dim, slots)):
        want = torch.from_numpy(y).float().to(dtype)             # one rounding: every value is one of 32 bits
        assert torch.equal(x.cpu().nan_to_num(-77.0, posinf=1e30 if dtype == torch.bfloat16 else 6e4), want.nan_to_num(-77.0, posinf=1e30 if dtype == torch.bfloat16 else 6e4))


@pytest.mark.parametrize("dtype", TYPES)
def test_append_edges_of_codes_zeros_and_what_is_not_finite(dtype):
    """Values at the middle between two codes, the largest and the smallest numbers, groups of zeros, groups with an infinity or a NaN."""
    x = torch.zeros((12, 1, 64), dtype=torch.float64)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 0.5, 6.0, 4.0, 0.26, 0.74, 3.49, 5.01, 6.9])
    x[0, 0, :16], x[0, 0, 16:32] = edges, -edges
    x[1] = x[0] * 2.0 ** -6
    x[2, 0, 3], x[2, 0, 40] = 7.03125, -0.0
    x[3] = 0.0
    x[4, 0, 1], x[4, 0, 33] = float("inf"), 1.0
    x[5, 0, 2], x[5, 0, 34] = float("nan"), 1.0
    x[6, 0, 7], x[6, 0, 60] = -float("inf"), 2.0
    big, small = torch.finfo(dtype).max, 2.0 ** (-24 if dtype == torch.float16 else -133)
    x[7, 0, :3] = torch.tensor([big, -big, big / 3])
    x[8, 0, :3] = torch.tensor([small, -small, 3 * small])
    x[9, 0, 5], x[9, 0, 37] = 65504.0, 1.75
    x[10, 0, :32] = torch.linspace(-7, 7, 32)
    x[11, 0, :32] = torch.linspace(-3.5, 3.5, 32)
    x = x.to(dtype)
    cache = pool(rng(1), 1, 16, 1, 64)
    cache.append(None, x.cuda(), x.cuda(), None, ints(np.arange(12)))
    keys, values = ref.read(cache.data.cpu().numpy(), 16, 64, np.arange(12))
    want = ref.nearest(ref.to_numpy(x))
    rows = [i for i in range(12) if i != 7 or dtype == torch.float16]          # 2^128 is an infinity to both
    for got in (keys, values):
        assert np.array_equal(got[rows], want[rows], equal_nan=True)
    assert np.isnan(want[4, 0, :32]).all() and (want[4, 0, 32:] != 0).sum() == 1
    for got in cache.read(ints(np.arange(12)), dtype):
        assert torch.equal(got[rows].cpu().nan_to_num(9e4), torch.from_numpy(want[rows]).to(dtype).nan_to_num(9e4))


def test_offsets_beyond_32_bits():
    """Pages on both sides of 2^31 and 2^32 bytes of a pool, through all three calls."""
    page, heads, dim = 64, 8, 128
    piece = heads * ref.piece_bytes(page, dim)
    pages = (2 ** 32) // piece + 3
    cache = M.KvCache(pages, page, heads, dim)
    assert cache.data.numel() > 2 ** 32
    g = rng(3)
    use = [0, (2 ** 31) // piece, (2 ** 31) // piece + 1, (2 ** 32) // piece, pages - 1]
    slots = np.concatenate([p * page + np.arange(page) for p in use])[:300]
    k, v = (normal(g, 300, heads, dim) for _ in range(2))
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    for x, y in zip(cache.read(ints(slots)), (k, v)):
        assert np.array_equal(ref.to_numpy(x), ref.nearest(ref.to_numpy(y)))
    q = normal(g, 1, 8, dim)
    got, sums = cache.attend(q.cuda(), ints([use]), ints([300]), sums=True)
    small = cache.data[use].cpu().numpy()
    want, total, reach, far = ref.attend(ref.to_numpy(q), small, page, np.arange(5)[None], [300])
    check_attention(got, sums, want, total, reach, far, torch.float16)


# ---- attention ----------------------------------------------------------------

def check_attention(got, sums, want, total, reach, far, dtype):
    share = reach * 2.0 ** -13 + 2.0 ** -15
    close(got, want, dtype, (2 * share * far)[..., None])
    fine = np.isfinite(want)
    norm = np.linalg.norm(want[fine])
    assert norm == 0 or np.linalg.norm(ref.to_numpy(got)[fine] - want[fine]) <= HALF[dtype] * norm
    if sums is not None:
        s = ref.to_numpy(sums)
        assert np.array_equal(np.isnan(s), np.isnan(total)) and np.array_equal(s == -np.inf, total == -np.inf)
        fine = np.isfinite(total)
        assert np.all(np.abs(s - total)[fine] <= (share + np.abs(np.where(fine, total, 0)) * 2.0 ** -21 + 2.0 ** -20)[fine])


def sequences(g, cache, lengths, dirty=True):
    """Tables for these lengths; pages in random order, what is not used of the tables names no page."""
    page = cache.page_size
    order = torch.randperm(cache.pages, generator=g).tolist()
    width = max([-(-n // page) for n in lengths] + [0]) + 2
    tables = np.full((len(lengths), width), -2 ** 31 if dirty else 0, dtype=np.int64)
    for b, n in enumerate(lengths):
        for i in range(-(-max(n, 0) // page)):
            tables[b, i] = order.pop()
    return tables


def fill(g, cache, tables, lengths, scale=1.0):
    """Keys and values of all tokens, through append; returns them as they were given."""
    page = cache.page_size
    slots = np.concatenate([tables[b, np.arange(max(n, 0)) // page] * page + np.arange(max(n, 0)) % page for b, n in enumerate(lengths)] or [np.zeros(0, int)])
    k = normal(g, len(slots), cache.kv_heads, cache.head_dim, scale=scale)
    k[..., ::19] *= 4
    v = normal(g, len(slots), cache.kv_heads, cache.head_dim)
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    return slots


ATTENTION = [
    # dim, page, heads, kv heads, lengths, queries, window
    (128, 16, 8, 8, [1], None, 0), (128, 16, 4, 2, [2, 15, 16, 17, 31, 32, 33, 0, 47, 48], None, 0), (128, 64, 8, 2, [127, 128, 129, 63, 64, 65], None, 0),
    (64, 32, 40, 8, [300, 0, 5, 1], None, 0), (32, 16, 3, 1, [70, 33], None, 0), (96, 128, 4, 4, [200, 1], None, 0), (160, 16, 5, 1, [50, 129], None, 0),
    (192, 32, 6, 3, [65], None, 0), (224, 16, 2, 2, [40], None, 0), (256, 16, 16, 2, [100, 7], None, 0), (128, 4096, 2, 1, [5000], None, 0),
    (128, 16, 17, 1, [90], None, 0), (64, 16, 64, 1, [90, 33], None, 0),                     # more heads to a key head than one or two tiles of rows
    (128, 16, 8, 2, [50, 20, 4, 0, 9], [5, 1, 4, 2, 0], 0),                                  # several queries; more of them than tokens; none
    (64, 32, 4, 4, [40, 90], [40, 33], 0), (128, 32, 12, 4, [200], [70], 0), (256, 16, 4, 1, [60], [23], 0),
    (128, 16, 4, 2, [100, 60, 3], None, 7), (64, 16, 8, 8, [100, 60, 3], [4, 9, 3], 20), (128, 32, 2, 1, [150], [40], 1), (96, 16, 3, 3, [300], [3], 33),
    (128, 16, 8, 8, [1500, 700, 3, 0, 1200], None, 0), (64, 64, 8, 1, [2500, 600], [3, 2], 0), (128, 16, 2, 2, [2000, 900], [2, 1], 600),       # split over workgroups
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention(case, dtype):
    dim, page, heads, kv_heads, lengths, queries, window = ATTENTION[case]
    g = rng(case)
    cache = pool(g, sum(-(-n // page) for n in lengths) + 2, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    n = [1] * len(lengths) if queries is None else queries
    start = np.concatenate([[0], np.cumsum(n)])
    q = normal(g, sum(n), heads, dim, dtype=dtype, scale=1.5)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, lengths, start, window=window)
    more = {} if queries is None else dict(start=ints(start), most_queries=max(n))
    got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), window=window, sums=True, longest=max(lengths), **more)
    check_attention(got, sums, *want, dtype)
    # a bound that is too small or too large changes the launch, not the result's correctness; without the sums
    for longest, most in ((1, 1), (None, max(n) + 100)):
        if queries is not None:
            more["most_queries"] = most
        check_attention(cache.attend(q.cuda(), ints(tables), ints(lengths), window=window, longest=longest, **more), None, *want, dtype)


def test_attention_a_long_sequence_and_its_parts():
    """One sequence of 40001 tokens; and the same as two parts joined by their sums."""
    g = rng(77)
    page, dim, heads, kv_heads, n = 64, 128, 8, 2, 40001
    cache = pool(g, -(-n // page), page, kv_heads, dim)
    tables = sequences(g, cache, [n])
    fill(g, cache, tables, [n])
    q = normal(g, 1, heads, dim)
    data = cache.data.cpu().numpy()
    want = ref.attend(ref.to_numpy(q), data, page, tables, [n])
    got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), sums=True, longest=n)
    check_attention(got, sums, *want, torch.float16)
    cut = 250 * page
    parts = [cache.attend(q.cuda(), ints(t), ints([m]), sums=True) for t, m in ((tables[:, :250], cut), (tables[:, 250:], n - cut))]
    w = torch.softmax(torch.stack([s for _, s in parts]).double(), 0)[..., None]
    joined = ref.to_numpy(sum(o.double() * x for (o, _), x in zip(parts, w)))
    assert np.linalg.norm(joined - want[0]) <= 2.0 ** -11 * np.linalg.norm(want[0])


def test_attention_what_is_masked_has_no_effect():
    """NaN, infinities and wild bytes in tokens that a query does not see: later tokens, those before the window, the rest of pages, pages behind
    the end, table entries that are not needed."""
    g = rng(8)
    page, dim, heads, kv_heads, length, asked, window = 16, 128, 4, 2, 75, 20, 30
    clean, dirty = (pool(rng(i), 8, page, kv_heads, dim) for i in (1, 2))
    tables = sequences(g, clean, [length])
    fill(rng(9), clean, tables, [length])
    fill(rng(9), dirty, tables, [length])
    q = normal(g, asked, heads, dim)
    call = dict(start=ints([0, asked]), most_queries=asked, window=window, sums=True)
    want, total = clean.attend(q.cuda(), ints(tables), ints([length]), **call)
    # token 70 is seen by the last 5 queries alone, token 27 by the first query (place 55, from 26) and the second (from 27): spoil both
    x = torch.full((2, kv_heads, dim), float("nan"), dtype=torch.float16)
    x[1, 0, 40:] = 1.0
    slots = [int(tables[0, t // page] * page + t % page) for t in (70, 27)]
    dirty.append(None, x.cuda(), x.cuda(), None, ints(slots))
    tables[0, 0] = 2 ** 30                                       # tokens 0 to 15: outside every query's window
    got, sums = dirty.attend(q.cuda(), ints(tables), ints([length]), **call)
    sees = [i for i in range(asked) if 55 + i >= 70 or 55 + i - window + 1 <= 27]
    rest = [i for i in range(asked) if i not in sees]
    assert len(sees) == 7 and torch.equal(got[rest], want[rest]) and torch.equal(sums[rest], total[rest])
    reference = ref.attend(ref.to_numpy(q), dirty.data.cpu().numpy(), page, tables, [length], [0, asked], window=window)[0]
    assert np.array_equal(np.isnan(ref.to_numpy(got)), np.isnan(reference)) and np.isnan(reference[sees]).any((1, 2)).all()


def test_attention_values_that_are_not_finite_alone():
    """A token whose values hold a NaN, with keys that are finite: the groups that hold it, of the rows that see it, and nothing else."""
    g = rng(21)
    page, dim, length, asked = 16, 96, 40, 6
    cache = pool(g, 4, page, 1, dim)
    tables = sequences(g, cache, [length])
    slots = fill(g, cache, tables, [length])
    k = normal(g, 1, 1, dim)
    v = normal(g, 1, 1, dim)
    v[0, 0, 50] = float("inf")
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots[37:38]))
    q = normal(g, asked, 3, dim)
    got = ref.to_numpy(cache.attend(q.cuda(), ints(tables), ints([length]), start=ints([0, asked]), most_queries=asked))
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, [length], [0, asked])
    assert np.isnan(want[0][3:, :, 32:64]).all() and not np.isnan(want[0][:3]).any() and not np.isnan(want[0][:, :, :32]).any()
    assert np.array_equal(np.isnan(got), np.isnan(want[0]))
    fine = ~np.isnan(got)
    assert np.linalg.norm(got[fine] - want[0][fine]) <= 2.0 ** -11 * np.linalg.norm(want[0][fine])


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
    # no table at all, no pages at all
    assert torch.isnan(cache.attend(q.cuda(), ints(np.zeros((5, 0))), ints(lengths))).all()
    empty = M.KvCache(0, 16, 2, 64)
    assert torch.isnan(empty.attend(q.cuda(), ints(tables), ints(lengths))).all()
    none = empty.attend(q.cuda(), ints(tables), ints([0, 0, -3, 0, 0]))
    assert torch.equal(none, torch.zeros_like(none))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_large_and_extreme_scores(dtype):
    """Scores that grow along the sequence by far more than the running maximum may lag, negative scales, weights that underflow, huge queries."""
    g = rng(14)
    page, dim, n = 16, 64, 400
    cache = pool(g, 25, page, 1, dim)
    tables = sequences(g, cache, [n])
    slots = tables[0, np.arange(n) // page] * page + np.arange(n) % page
    k = normal(g, n, 1, dim) + (torch.arange(n)[:, None, None] * 0.05).half()
    v = normal(g, n, 1, dim)
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    q = normal(g, 1, 6, dim, dtype=dtype, scale=1.0)
    q[0, 0], q[0, 1], q[0, 2] = 4.0, -4.0, 0.0
    q[0, 3] = q[0, 3] * 100
    q[0, 4] = q[0, 4] * 1e-6
    q[0, 5, ::2] = 0
    data = cache.data.cpu().numpy()
    for scale in (0.125, -0.125, 0.0, 3.0):
        want = ref.attend(ref.to_numpy(q), data, page, tables, [n], scale=scale)
        got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), scale=scale, sums=True)
        check_attention(got, sums, *want, dtype)
    q[0, 0, 3], q[0, 1, 9] = float("nan"), float("inf")
    got = ref.to_numpy(cache.attend(q.cuda(), ints(tables), ints([n])))
    assert np.isnan(got[0, :2]).all() and np.isfinite(got[0, 2:]).all()


def test_attention_strides_streams_and_other_memory():
    g = rng(15)
    page, dim, heads, kv_heads = 16, 128, 6, 3
    lengths = [700, 33, 1200]
    cache = pool(g, 130, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    base = normal(g, 3, heads, dim)
    want = ref.attend(ref.to_numpy(base), cache.data.cpu().numpy(), page, tables, lengths)
    fused = torch.zeros((3, 2 * heads + 1, dim), dtype=torch.float16, device="cuda")
    fused[:, 1:1 + heads] = base.cuda()
    odd = torch.empty(3 * heads * dim + 1, dtype=torch.float16, device="cuda")[1:].view(heads, 3, dim).transpose(0, 1)
    odd.copy_(base)
    wide = torch.full((3, 200), 2 ** 30, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = ints(tables)
    whole = torch.full((3, heads, 2 * dim), 5.0, dtype=torch.float16, device="cuda")
    for q in (fused[:, 1:1 + heads], odd):
        check_attention(cache.attend(q, wide[:, :tables.shape[1]], ints(lengths), out=whole[..., :dim]), None, *want, torch.float16)
        assert (whole[..., dim:] == 5).all()
    # on a stream of its own, by object and by number; the workspace goes back while the call still runs
    side = torch.cuda.Stream()
    args = (base.cuda(), ints(tables), ints(lengths))
    torch.cuda.synchronize()
    first = cache.attend(*args, stream=side)
    again = [cache.attend(*args, stream=side.cuda_stream) for _ in range(5)]
    with torch.cuda.stream(side):
        again.append(cache.attend(*args))
    side.synchronize()
    check_attention(first, None, *want, torch.float16)
    assert all(torch.equal(first, x) for x in again)


def test_a_decoding_step_in_a_graph():
    """append and attend captured once, replayed as the sequences grow: positions, slots and lengths are data."""
    g = rng(16)
    page, dim, heads, kv_heads, batch = 16, 128, 8, 4, 3
    cache = pool(g, 60, page, kv_heads, dim)
    twin = M.KvCache(60, page, kv_heads, dim, data=cache.data.clone())
    lengths = [5, 300, 127]
    tables = sequences(g, cache, [n + 8 for n in lengths])
    for c in (cache, twin):
        fill(rng(4), c, tables, lengths)
    tab = M.rope_table(400, dim)
    w = normal(g, dim).cuda()
    x = torch.zeros((batch, heads + 2 * kv_heads, dim), dtype=torch.float16, device="cuda")
    at, slots, now, tabs = (ints(np.zeros(batch)) for _ in range(3)), None, None, ints(tables)
    at, slots, now = at

    def step(c):
        q = c.append(x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], at, slots, tab, q_weight=w, k_weight=w)
        return c.attend(q, tabs, now, longest=2000, sums=True)

    def feed(i):
        x.copy_(normal(rng(100 + i), batch, heads + 2 * kv_heads, dim))
        n = np.array(lengths) + i
        at.copy_(ints(n))
        slots.copy_(ints(tables[np.arange(batch), n // page] * page + n % page))
        now.copy_(ints(n + 1))

    feed(0)
    step(twin)                                                    # kernels are loaded outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, sums = step(cache)
    for i in range(8):
        feed(i)
        graph.replay()
        torch.cuda.synchronize()
        want, total = step(twin)
        assert torch.equal(out, want) and torch.equal(sums, total) and torch.equal(cache.data, twin.data)
        torch.zeros(1 << 20, device="cuda").sum().item()
    n = np.array(lengths) + 8
    q = M.rotate(x[:, :heads], at, tab, weight=w)
    check_attention(out, sums, *ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, n), torch.float16)


# ---- refusals -----------------------------------------------------------------

@pytest.mark.parametrize("native", [True, False])
def test_refusals_of_the_python_calls(native, monkeypatch):
    if not native:
        monkeypatch.setattr(M.binding, "_native", None)
    cache = M.KvCache(4, 16, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda")
    i3, tab = ints([0, 1, 2]), M.rope_table(8, 64)
    one = ints(np.zeros((3, 1)))
    bad = [
        lambda: M.rotate(x.float(), i3, tab), lambda: M.rotate(x.cpu(), i3, tab), lambda: M.rotate(x[0], i3, tab), lambda: M.rotate(x, i3.long(), tab),
        lambda: M.rotate(x, i3[:2], tab), lambda: M.rotate(x, None, tab), lambda: M.rotate(x, i3, tab.half()), lambda: M.rotate(x, i3, tab[:, :1]),
        lambda: M.rotate(x, i3, M.rope_table(8, 128)), lambda: M.rotate(x, i3, M.rope_table(8, 8)), lambda: M.rotate(x[..., ::2], i3, None),
        lambda: M.rotate(x[..., :40], i3, None), lambda: M.rotate(x, i3, tab, weight=torch.ones(64, device="cuda")), lambda: M.rotate(x, i3, tab, weight=x[0, 0, :32]),
        lambda: M.rotate(x, i3, tab, out=x[:1].expand(3, 2, 64)), lambda: M.rotate(x, i3, tab, out=torch.zeros_like(x, dtype=torch.bfloat16)),
        lambda: M.KvCache(4, 24, 2, 64), lambda: M.KvCache(4, 8, 2, 64), lambda: M.KvCache(4, 8192, 2, 64), lambda: M.KvCache(4, 16, 2, 80), lambda: M.KvCache(4, 16, 2, 288),
        lambda: M.KvCache(-1, 16, 2, 64), lambda: M.KvCache(4, 16, 0, 64), lambda: M.KvCache(2 ** 28, 16, 2, 64), lambda: M.KvCache(4, 16, 2, 64, data=cache.data[:3]),
        lambda: M.KvCache(4, 16, 2, 64, data=cache.data.cpu()), lambda: M.KvCache(4, 16, 2, 64, data=cache.data.char()),
        lambda: cache.append(x, x, x[:2], None, i3), lambda: cache.append(x, x, x, None, i3[:2]), lambda: cache.append(x, x[:, :1], x, None, i3),
        lambda: cache.append(x.bfloat16(), x, x, None, i3), lambda: cache.append(x, x, x, i3, i3.long()), lambda: cache.append(x, x.cpu(), x.cpu(), None, i3),
        lambda: cache.append(x, x, x, None, i3, tab), lambda: cache.append(x, x, x, None, i3, q_out=x[:, :1]),
        lambda: cache.read(i3.long()), lambda: cache.read(i3, torch.float32), lambda: cache.read(i3, k_out=x[:2]), lambda: cache.read(i3.cpu()),
        lambda: cache.attend(x[:2], one, i3), lambda: cache.attend(x, one[0], i3), lambda: cache.attend(x, one, i3.long()), lambda: cache.attend(x[..., :32], one, i3),
        lambda: cache.attend(x[:, :1], one, i3), lambda: cache.attend(x, one, i3, start=i3), lambda: cache.attend(x, one, i3, window=-1),
        lambda: cache.attend(x, one, i3, most_queries=0), lambda: cache.attend(x, one, i3, scale=float("nan")), lambda: cache.attend(x, one, i3, out=x[:, :1].expand(3, 2, 64)),
        lambda: M.rope_table(4, 3), lambda: M.rope_table(4, 64, base=-1.0), lambda: M.rope_table(4, 64, factor=0.0), lambda: M.rope_table(-1, 64, device="cuda"),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, M.MackoError)):
            call()
            pytest.fail(f"call {i} was taken")
    torch.cuda.synchronize()
    # nothing to do is fine
    assert cache.append(x[:0], x[:0], x[:0], i3[:0], i3[:0], tab).shape == (0, 2, 64)
    assert [t.shape[0] for t in cache.read(i3[:0])] == [0, 0]
    assert cache.attend(x[:0], one[:0], i3[:0]).shape == (0, 2, 64)
    assert cache.attend(x[:0], one, i3, start=ints([0, 0, 0, 0])).shape == (0, 2, 64)


def test_native_calls_do_what_the_general_ones_do(monkeypatch):
    M.load_library()
    native = M.binding._native
    assert native is not None
    g = rng(31)
    page, dim, heads, kv_heads, tokens = 16, 64, 4, 2, 9
    tab, at, slots = M.rope_table(50, dim), ints(np.arange(9) * 5), ints(np.arange(9) * 3)
    w = normal(g, dim).cuda()
    x = normal(g, tokens, heads + 2 * kv_heads, dim).cuda()
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    table, lengths, start = ints([[0, 1, -1], [0, 1, 1]]), ints([20, 31]), ints([0, 3, 9])
    kept = torch.zeros((tokens, heads, dim), dtype=torch.float16, device="cuda")
    b = x.bfloat16()
    calls = [
        lambda c: M.rotate(q, at, tab), lambda c: M.rotate(q, at, tab, w, 1e-3, True), lambda c: M.rotate(q, None, None, weight=w), lambda c: M.rotate(q, at, tab, out=kept) is kept,
        lambda c: M.rotate(b, at, tab, weight=w.bfloat16()), lambda c: M.rotate(q.transpose(0, 1), ints([1, 2, 3, 4]), tab),
        lambda c: c.append(q, k, v, at, slots, tab, q_weight=w, k_weight=w, eps=1e-4, interleaved=True), lambda c: c.append(None, k, v, None, slots),
        lambda c: c.append(q, k, v, at, slots, tab, q_out=kept) is kept, lambda c: kept.clone(), lambda c: c.append(b[:, :4], b[:, 4:6], b[:, 6:], at, slots, tab),
        lambda c: c.read(slots), lambda c: c.read(slots, torch.bfloat16), lambda c: c.read(slots, k_out=kept[:, :2])[0].data_ptr() == kept.data_ptr(),
        lambda c: c.attend(q, table, lengths, start=start, most_queries=6, window=11, scale=-0.2, sums=True), lambda c: c.attend(q[:2], table, lengths),
        lambda c: c.attend(q[:2], table, lengths, longest=31, out=kept[:2]) is not None, lambda c: kept.clone(), lambda c: c.attend(b[:2, :4], table, lengths, sums=True),
        lambda c: c.attend(q[:2], table, lengths, scale=0.0), lambda c: c.attend(q[:0], table[:0], lengths[:0]), lambda c: c.data.clone(),
    ]
    results = []
    for part in (native, None):
        monkeypatch.setattr(M.binding, "_native", part)
        cache = M.KvCache(3, page, kv_heads, dim, data=torch.zeros((3, kv_heads, ref.piece_bytes(page, dim)), dtype=torch.uint8, device="cuda"))
        kept.zero_()
        results.append([call(cache) for call in calls])
    for i, (one, two) in enumerate(zip(*results)):
        for a, c in zip(one if isinstance(one, tuple) else (one,), two if isinstance(two, tuple) else (two,)):
            assert type(a) is type(c), i
            assert (torch.equal(a, c) and a.dtype == c.dtype) if isinstance(a, torch.Tensor) else a == c, i


# ---- many rows ----------------------------------------------------------------

PROMPT = [
    # dim, page, heads, kv heads, lengths, queries, window
    (128, 16, 8, 2, [300], [100], 0), (128, 64, 4, 4, [130, 65, 64, 200], [130, 65, 64, 1], 0), (32, 16, 6, 2, [150, 30], [90, 30], 0), (64, 32, 40, 8, [700], [33], 0),
    (96, 16, 3, 1, [90], [90], 0), (160, 16, 2, 1, [140, 77], [70, 40], 0), (192, 64, 3, 3, [300], [129], 0), (224, 16, 1, 1, [99], [80], 0), (256, 32, 8, 2, [260], [40], 0),
    (128, 16, 4, 2, [400, 0, 90], [150, 3, 90], 0), (128, 16, 4, 2, [600], [200], 70), (64, 16, 2, 1, [500, 20], [300, 40], 1), (128, 128, 16, 1, [1000], [6], 333),
    (128, 16, 2, 1, [2500], [90], 0), (256, 16, 2, 2, [1400, 3], [70, 70], 0), (64, 64, 66, 1, [3000, 700], [2, 2], 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_attention_of_many_rows(case, dtype):
    dim, page, heads, kv_heads, lengths, queries, window = PROMPT[case]
    g = rng(1000 + case)
    cache = pool(g, sum(-(-n // page) for n in lengths) + 2, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    start = np.concatenate([[0], np.cumsum(queries)])
    q = normal(g, sum(queries), heads, dim, dtype=dtype, scale=1.5)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, lengths, start, window=window)
    for longest, most in ((max(lengths), max(queries)), (1, max(queries)), (None, 10 * max(queries))):
        got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), start=ints(start), most_queries=most, window=window, longest=longest, sums=True)
        check_attention(got, sums, *want, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("asked", [4, 90])
@pytest.mark.parametrize("sizes", [(1e-4,), (2e-7, 1.0), (1.0, 3e4), (1e-6,), (0.0, 1.0), (0.0,), (1e-6, 1e4, 0.0)])
def test_attention_values_of_any_size(sizes, asked, dtype):
    """Values whose factors lie beyond what fp16 holds, in some tokens or all, groups of zeros among others."""
    g = rng(41)
    page, dim, length = 16, 128, 333
    cache = pool(g, 22, page, 2, dim)
    tables = sequences(g, cache, [length])
    slots = tables[0, np.arange(length) // page] * page + np.arange(length) % page
    k = normal(g, length, 2, dim, dtype=torch.bfloat16)
    size = torch.tensor(sizes, dtype=torch.float64)[torch.arange(length) * 7 // 50 % len(sizes)]
    v = (torch.randn((length, 2, dim), generator=g, dtype=torch.float64) * size[:, None, None]).bfloat16()
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    q = normal(g, asked, 4, dim, dtype=dtype)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, [length], [0, asked])
    got, sums = cache.attend(q.cuda(), ints(tables), ints([length]), start=ints([0, asked]), most_queries=asked, sums=True)
    if dtype == torch.float16 and max(sizes) < 1e-3 and max(sizes) > 0:       # the results themselves are below fp16's normal numbers
        share = want[2] * 2.0 ** -13 + 2.0 ** -15
        close(got, want[0], dtype, (2 * share * want[3])[..., None])
    else:
        check_attention(got, sums, *want, dtype)


@pytest.mark.parametrize("window", [0, 50])
def test_attention_of_many_rows_what_is_masked_has_no_effect(window):
    """As above for the other kernel: NaN and an infinity in tokens that some rows see and others do not, wild bytes elsewhere, pages that are not needed."""
    g = rng(51)
    page, dim, heads, kv_heads, length, asked = 16, 64, 4, 2, 200, 120
    clean, dirty = (pool(rng(i), 16, page, kv_heads, dim) for i in (1, 2))
    tables = sequences(g, clean, [length])
    for c in (clean, dirty):
        fill(rng(9), c, tables, [length])
    q = normal(g, asked, heads, dim)
    call = dict(start=ints([0, asked]), most_queries=asked, window=window, sums=True)
    want, total = clean.attend(q.cuda(), ints(tables), ints([length]), **call)
    k, v = normal(g, 3, kv_heads, dim), normal(g, 3, kv_heads, dim)
    v[0, 0, 40], v[1, 1, 3], k[2, 0, 9] = float("nan"), float("inf"), float("nan")
    spots = (170, 131, 150)
    dirty.append(None, k.cuda(), v.cuda(), None, ints([tables[0, t // page] * page + t % page for t in spots]))
    if window:
        tables[0, 0] = -7                                        # tokens 0 to 15: the first query is at place 80 and sees from 31 on
    got, sums = dirty.attend(q.cuda(), ints(tables), ints([length]), **call)
    place = np.arange(asked) + length - asked
    free = [i for i in range(asked) if not any(t <= place[i] and (not window or t > place[i] - window) for t in spots)]
    assert 40 < len(free) < asked and torch.equal(got[free], want[free]) and torch.equal(sums[free], total[free])
    out, lse, reach, far = ref.attend(ref.to_numpy(q), dirty.data.cpu().numpy(), page, tables, [length], [0, asked], window=window)
    assert np.array_equal(np.isnan(ref.to_numpy(got)), np.isnan(out)) and np.array_equal(np.isnan(ref.to_numpy(sums)), np.isnan(lse))
    fine = ~np.isnan(out)
    assert np.linalg.norm(ref.to_numpy(got)[fine] - out[fine]) <= 2.0 ** -11 * np.linalg.norm(out[fine])
    tables[0, 9] = 99                                            # a page that rows from place 144 on need
    again = ref.to_numpy(dirty.attend(q.cuda(), ints(tables), ints([length]), **call)[0])
    assert np.isnan(again[place >= 144][:window or None]).all()


def test_the_example_runs_the_operators_together(capsys):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # 16-bit results of a computation in 32 bits: half a unit in the last place
    assert example.main(["--tokens", "150", "--steps", "5", "--hidden", "512", "--inner", "1000", "--heads", "8", "--kv-heads", "2"]) <= 2.0 ** -11
    assert "4.25 bits a value" in capsys.readouterr().out


# A call's parts and its kernel follow an estimate of the time, which goes by the rows that there may be: with room for very many it is the kernel for
# many rows, without splits; with the room of the second test, with splits.
def attend_with_room(attend, cache, q, tables, lengths, tokens, **more):
    """As attend(q, ...), with queries of no sequence behind those of q."""
    wide = q.new_zeros((max(tokens, q.shape[0]), *q.shape[1:]))
    wide[:q.shape[0]] = q
    got = attend(cache, wide, tables, lengths, **dict(more, most_queries=wide.shape[0]))
    return tuple(x[:q.shape[0]] for x in got) if isinstance(got, tuple) else got[:q.shape[0]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_attention_of_many_rows_by_the_kernel_for_them(case, dtype):
    dim, page, heads, kv_heads, lengths, queries, window = PROMPT[case]
    g = rng(2000 + case)
    cache = pool(g, sum(-(-n // page) for n in lengths) + 2, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    start = np.concatenate([[0], np.cumsum(queries)])
    q = normal(g, sum(queries), heads, dim, dtype=dtype, scale=1.5)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, lengths, start, window=window)
    got, sums = attend_with_room(M.KvCache.attend, cache, q.cuda(), ints(tables), ints(lengths), 2 ** 18 // heads, start=ints(start), window=window, sums=True)
    check_attention(got, sums, *want, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,room", [(256, 512), (128, 1024), (64, 1024)])
def test_attention_of_many_rows_in_parts(dim, room, dtype):
    g = rng(2100 + dim)
    page, lengths, queries = 64, [8001, 0, 17, 1, 0, 700, 64, 0], [90, 3, 17, 1, 0, 130, 2, 0]
    cache = pool(g, 150, page, 1, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    start = np.concatenate([[0], np.cumsum(queries)])
    q = normal(g, sum(queries), 1, dim, dtype=dtype)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, lengths, start)
    got, sums = attend_with_room(M.KvCache.attend, cache, q.cuda(), ints(tables), ints(lengths), room, start=ints(start), longest=max(lengths), sums=True)
    check_attention(got, sums, *want, dtype)


@pytest.fixture
def very_many(monkeypatch):
    attend = M.KvCache.attend
    monkeypatch.setattr(M.KvCache, "attend", lambda self, q, tables, lengths, **more: attend_with_room(attend, self, q, tables, lengths, 2 ** 18 // q.shape[1], **more))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [(1e-4,), (2e-7, 1.0), (1.0, 3e4), (1e-6,), (0.0, 1.0), (0.0,), (1e-6, 1e4, 0.0)])
def test_attention_of_many_rows_values_of_any_size(very_many, sizes, dtype):
    test_attention_values_of_any_size(sizes, 90, dtype)


@pytest.mark.parametrize("window", [0, 50])
def test_what_is_masked_has_no_effect_in_the_kernel_for_many_rows(very_many, window):
    test_attention_of_many_rows_what_is_masked_has_no_effect(window)
