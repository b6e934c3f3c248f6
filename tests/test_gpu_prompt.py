"""Attention of packed prompts over their own keys and values in 16 bits, on the GPU, against tests/kv8_reference.py (64 bits).

Tolerances.  A result is off by at most half a unit in the last place, 2^-11 (fp16) or 2^-8 (bf16) of it, from what was computed.  What was computed: a score is a sum of
up to 256 exact products in 32 bits, off by 2^-16 of the sum of their magnitudes at most, so a weight by the same share of it times scale; a weight is rounded to
the tensors' type, 2^-11 or 2^-8 of it, numerator and denominator alike.  Sums are of the weights before that: 2^-16 for exponentials and additions."""
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


def packed(q, k, v, start, scale=None, window=0):
    parts = [np.zeros(q.shape), np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2]), np.zeros(q.shape[:2])]
    for lo, hi in zip(start[:-1], start[1:]):
        for whole, part in zip(parts, ref.attend(q[lo:hi], k[lo:hi], v[lo:hi], 0, scale, window)):
            whole[lo:hi] = part
    return parts


def check(got, sums, want, total, reach, far, dtype, weight=None):
    got = to_numpy(got)
    share = reach * 2.0 ** -16 + (HALF[dtype] if weight is None else weight) + 2.0 ** -16
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        bound = np.abs(want) * HALF[dtype] * (1 + 2.0 ** -7) + TINY[dtype] + (2 * share * far)[..., None]
        bad = ~(np.abs(got - want) <= bound) & ~np.isnan(want) & ~(got == want)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, the worst by {np.nanmax(np.where(bad, np.abs(got - want) / bound, 0)):.2f} of the bound"
    fine = np.isfinite(want)
    # weights' errors are independent of each other, those of results too: of the norm both together are less than one bound
    assert np.linalg.norm(got[fine] - want[fine]) <= HALF[dtype] * np.linalg.norm(want[fine])
    if sums is not None:
        s = to_numpy(sums)
        assert np.array_equal(np.isnan(s), np.isnan(total)) and np.array_equal(s == -np.inf, total == -np.inf)
        fine = np.isfinite(total)
        assert np.all(np.abs(s[fine] - total[fine]) <= reach[fine] * 2.0 ** -16 + np.abs(total[fine]) * 2.0 ** -21 + 2.0 ** -16)


PROMPTS = [
    # dim, heads, kv heads, lengths, window
    (128, 4, 4, [1], 0), (128, 4, 1, [33], 0), (64, 5, 1, [1, 2, 3, 0, 0, 63, 64, 65, 1], 0), (128, 2, 2, [127, 128, 129], 0), (32, 3, 3, [200, 70], 0),
    (96, 4, 2, [150, 31], 0), (160, 2, 1, [90, 66], 0), (192, 3, 3, [100], 0), (224, 2, 2, [70, 5], 0), (256, 4, 2, [130, 40], 0), (128, 17, 1, [50, 20], 0),
    (64, 8, 8, [300], 0), (128, 8, 2, [700], 0), (128, 8, 8, [520, 33], 0), (64, 40, 8, [170, 90, 130], 50), (128, 4, 4, [300], 1), (96, 3, 1, [260, 40], 64), (256, 2, 1, [300], 7),
    (64, 16, 16, [1] * 70, 0), (128, 2, 1, list(range(40)), 5), (32, 64, 2, [90, 300], 0), (128, 32, 32, [600], 0),
]


def inputs(case, dtype):
    dim, heads, kv_heads, lengths, window = PROMPTS[case]
    g = rng(case)
    start = np.concatenate([[0], np.cumsum(lengths)])
    q, k, v = (normal(g, int(start[-1]), h, dim, dtype=dtype, scale=s) for h, s in ((heads, 1.5), (kv_heads, 1.0), (kv_heads, 1.0)))
    return q, k, v, start, window


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(case, dtype):
    q, k, v, start, window = inputs(case, dtype)
    want = packed(*(to_numpy(x) for x in (q, k, v)), start, window=window)
    dev = [x.cuda() for x in (q, k, v)]
    got, sums = M.attend_prompt(*dev, ints(start), longest=int(np.diff(start).max()), window=window, sums=True)
    check(got, sums, *want, dtype)
    for longest in (1, None):
        check(M.attend_prompt(*dev, ints(start), longest=longest, window=window), None, *want, dtype)
    if len(start) == 2:
        assert torch.equal(M.attend_prompt(*dev, window=window, longest=int(start[-1])), got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,lengths,window", [(96, [1030], 0), (128, [1, 1100, 40], 0), (128, [1200], 600), (96, [50, 1027, 3], 1000)])
def test_many_rows_that_see_many_tokens(dim, lengths, window, dtype):
    """Calls large enough for blocks of 256 rows, some heads against the reference and all of them against blocks of 128 rows."""
    g = rng(dim + len(lengths))
    heads, kv_heads = 128, 32
    start = np.concatenate([[0], np.cumsum(lengths)])
    q, k, v = (normal(g, int(start[-1]), h, dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    dev = [x.cuda() for x in (q, k, v)]
    got, sums = M.attend_prompt(*dev, ints(start), longest=max(lengths), window=window, sums=True)
    other, other_sums = M.attend_prompt(*dev, ints(start), longest=100, window=window, sums=True)
    for h in (0, 66, 127):
        want = packed(to_numpy(q)[:, h:h + 1], to_numpy(k)[:, h // 4:h // 4 + 1], to_numpy(v)[:, h // 4:h // 4 + 1], start, window=window)
        for out, s in ((got, sums), (other, other_sums)):
            check(out[:, h:h + 1], s[:, h:h + 1], *want, dtype)
    # both are that near to the same; 1.5 * 128 products of a mean magnitude of 0.64 make scores' reach some 11, 20 at most
    a, b = got.double(), other.double()
    assert (a - b).norm() <= 2 * HALF[dtype] * b.norm() and (sums - other_sums).abs().max() <= 2 * (20 * 2.0 ** -16 + 20 * 2.0 ** -21 + 2.0 ** -16)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_streams_outputs_and_rows_of_no_sequence(dtype):
    g = rng(31)
    dim, heads, kv_heads, tokens = 96, 4, 2, 140
    start = [3, 60, 60, 131]
    q, k, v = (normal(g, tokens, h, dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    want = packed(*(to_numpy(x) for x in (q, k, v)), start)
    outside = np.r_[0:3, 131:140]

    def odd(x):                                                      # 2 bytes off every boundary, wider rows
        made = torch.full((tokens * (x.shape[1] + 1) * (dim + 1) + 1,), float("nan"), dtype=dtype, device="cuda")[1:].view(tokens, x.shape[1] + 1, dim + 1)[:, :x.shape[1], :dim]
        return made.copy_(x)

    fused = torch.cat([q, k, v], 1).cuda()
    flipped = [x.cuda().transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    for qkv in ([odd(x) for x in (q, k, v)], fused.split([heads, kv_heads, kv_heads], 1), flipped):
        out = torch.full((tokens, heads, dim + 3), 7.0, dtype=dtype, device="cuda")
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        got, sums = M.attend_prompt(*qkv, ints(start), out=out[..., :dim], stream=other, sums=True)
        torch.cuda.current_stream().wait_stream(other)
        torch.cuda.synchronize()
        assert (out[..., dim:] == 7).all() and (out[outside] == 7).all()
        check(got[3:131], sums[3:131], *(x[3:131] for x in want), dtype)
    dev = [x.cuda() for x in (q, k, v)]
    assert M.attend_prompt(*(x[:0] for x in dev)).shape == (0, heads, dim)
    keep = torch.full((tokens, heads, dim), 5.0, dtype=dtype, device="cuda")
    M.attend_prompt(*dev, ints([0]), out=keep)                       # no sequences
    assert (keep == 5).all()
    for bad in (dict(q=dev[0].float()), dict(q=dev[0][:, :3]), dict(k=dev[1][1:]), dict(v=dev[2][:, :1]), dict(v=dev[2].to(TYPES[dtype == TYPES[0]])), dict(start=ints(start).long()),
                dict(start=ints([start])), dict(window=-1), dict(window=2 ** 40), dict(longest=-1), dict(k=dev[1].cpu()), dict(scale=float("nan")), dict(out=keep[:1].expand(tokens, heads, dim))):
        call = dict(dict(q=dev[0], k=dev[1], v=dev[2], start=ints(start)), **bad)
        with pytest.raises((TypeError, ValueError, M.MackoError)):
            M.attend_prompt(**call)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,heads", [(64, 4), (128, 1), (96, 2), (256, 1)])
def test_what_is_masked_has_no_effect(dim, heads, dtype):
    """NaN and infinities in rows that others do not see: later ones, those before the window, other sequences; in rows that they see, what the formula says."""
    g = rng(dim)
    start, window = [0, 150, 290, 300], 40
    q, k, v = (normal(g, 300, h, dim, dtype=dtype) for h in (heads, 1, 1))
    clean, total = M.attend_prompt(*(x.cuda() for x in (q, k, v)), ints(start), window=window, sums=True)
    k2, v2 = k.clone(), v.clone()
    k2[70], v2[70] = float("nan"), float("nan")
    v2[200, 0, 5], v2[201, 0, 6], v2[230, 0, 7] = float("inf"), -float("inf"), float("nan")
    v2[299, 0, :] = float("inf")
    got, sums = M.attend_prompt(q.cuda(), k2.cuda(), v2.cuda(), ints(start), window=window, sums=True)
    t = np.arange(300)
    sees = lambda s, hi: (t >= s) & (t < min(s + window, hi))  # noqa: E731
    touched = sees(70, 150) | sees(200, 290) | sees(201, 290) | sees(230, 290) | (t == 299)
    g64, c64 = to_numpy(got), to_numpy(clean)
    rest = ~touched
    assert np.isfinite(g64[rest]).all() and np.linalg.norm(g64[rest] - c64[rest]) <= HALF[dtype] * np.linalg.norm(c64[rest])
    assert np.abs(to_numpy(sums)[rest] - to_numpy(total)[rest]).max() <= 2.0 ** -14
    assert np.isnan(g64[sees(70, 150)]).all()
    assert (g64[sees(200, 290)][..., 5] == np.inf).all() and (g64[sees(201, 290)][..., 6] == -np.inf).all() and np.isnan(g64[sees(230, 290)][..., 7]).all()
    assert (g64[299] == np.inf).all()
    others = sees(200, 290) | sees(230, 290)
    channels = np.r_[0:5, 8:dim]
    assert np.linalg.norm(g64[others][..., channels] - c64[others][..., channels]) <= HALF[dtype] * np.linalg.norm(c64[others][..., channels])
    # a NaN in a query is that row's alone
    q2 = q.clone()
    q2[100, 0, 3] = float("nan")
    again = to_numpy(M.attend_prompt(q2.cuda(), k.cuda(), v.cuda(), ints(start), window=window))
    assert np.isnan(again[100, 0]).all()
    again[100, 0] = c64[100, 0]
    assert np.linalg.norm(again - c64) <= HALF[dtype] * np.linalg.norm(c64) and np.isfinite(again).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_large_and_extreme_scores(dtype):
    """Scores that grow along the sequence by far more than the running maximum may lag, negative and zero scales, weights that underflow."""
    g = rng(14)
    dim, n = 64, 400
    q, k, v = (normal(g, n, h, dim, dtype=dtype) for h in (4, 1, 1))
    k = k + torch.linspace(-3, 3, n)[:, None, None].to(dtype)
    q = q + 1
    for scale in (1.0, -1.0, 0.0, 0.01, 2.0 ** -130, 7.5):
        want = packed(*(to_numpy(x) for x in (q, k, v)), [0, n], scale=scale)
        got, sums = M.attend_prompt(q.cuda(), k.cuda(), v.cuda(), scale=scale, sums=True)
        check(got, sums, *want, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ahead", [5.0, 13.0, 16.0, 20.0])
def test_a_token_far_ahead_of_many(ahead, dtype):
    """A first token ahead of 6000 others whose value is zero: what the others sum up to is kept, in the results and in the sums."""
    g = rng(15)
    dim, n = 32, 6000
    k, v = torch.zeros((n, 1, dim)), 1.0 + torch.rand((n, 1, dim), generator=g)
    k[0, 0, 0], v[0] = ahead, 0.0
    q = torch.zeros((n, 1, dim))
    q[..., 0] = 1.0
    q, k, v = (x.to(dtype) for x in (q, k, v))
    got, sums = M.attend_prompt(q.cuda(), k.cuda(), v.cuda(), scale=1.0, sums=True)
    # weights are e^ahead and ones
    top, v64 = np.exp(to_numpy(k)[0, 0, 0]), to_numpy(v)[:, 0]
    count = np.arange(n)[:, None]
    want = np.cumsum(v64, 0) / (top + count)
    # the weight of the first token, those of the others (all the same), the result; below fp16's normal numbers a result is off by 2^-25 alone
    assert np.all(np.abs(to_numpy(got)[:, 0] - want)[1:] <= 2.5 * HALF[dtype] * want[1:] + TINY[dtype])
    assert np.abs(to_numpy(sums)[:, 0] - np.log(top + count[:, 0])).max() <= 2.0 ** -15


def test_sums_join_a_prompt_with_a_cached_prefix():
    """A prefix in the 8-bit cache and a prompt behind it, joined by their sums, against both at once."""
    g = rng(22)
    page, dim, heads, kv_heads, before, n = 16, 64, 4, 2, 100, 50
    cache = M.KvCache8(8, page, kv_heads, dim)
    table = ints([[3, 1, 4, 0, 5, 2, 6]])
    k, v = (normal(g, before + n, kv_heads, dim) for _ in range(2))
    cache.append(None, k[:before].cuda(), v[:before].cuda(), None, table, ints([before]), start=ints([0, before]))
    q = normal(g, n, heads, dim)
    slots = (table[0].long()[:, None] * page + torch.arange(page, device="cuda")).view(-1)[:before].to(torch.int32)
    held = [to_numpy(x) for x in cache.read(slots)]
    new = M.attend_prompt(q.cuda(), k[before:].cuda(), v[before:].cuda(), sums=True)
    # all of the prefix: a window would not do, so each query is a sequence of its own over the same pages
    old = cache.attend(q.cuda(), table.expand(n, -1).contiguous(), ints([before] * n), sums=True)
    w = torch.softmax(torch.stack([old[1], new[1]]).double(), 0)[..., None]
    joined = to_numpy(old[0].double() * w[0] + new[0].double() * w[1])
    want = ref.attend(to_numpy(q), np.concatenate([held[0], to_numpy(k)[before:]]), np.concatenate([held[1], to_numpy(v)[before:]]), before)[0]
    assert np.linalg.norm(joined - want) <= 2.0 ** -11 * np.linalg.norm(want)


def test_a_captured_prompt():
    """In a graph, replayed with other inputs and other sequences, with eager work between the replays."""
    g = rng(40)
    dim, heads, kv_heads, tokens = 128, 8, 2, 300
    q, k, v = (normal(g, tokens, h, dim, dtype=torch.bfloat16).cuda() for h in (heads, kv_heads, kv_heads))
    start = ints([0, 100, 300])
    M.attend_prompt(q, k, v, start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, sums = M.attend_prompt(q, k, v, start, sums=True)
    for i in range(10):
        for x in (q, k, v):
            x.copy_(normal(g, *x.shape, dtype=torch.bfloat16))
        start.copy_(ints([0, 17 * i + 1, 300]))
        graph.replay()
        got = out.clone(), sums.clone()
        torch.cuda.synchronize()
        want = M.attend_prompt(q, k, v, start, sums=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_sums_of_a_token_2_to_the_30_ahead_of_131072(dtype):
    """Steps of 64 tokens, 2^5 of weight to a lane, that leave a sum in 32 bits above 2^30 as it was: half of the others would be lost, 2^-14 of the sum."""
    dim, n = 32, 131072
    q, k, v = torch.zeros((n, 1, dim)), torch.zeros((n, 1, dim)), torch.ones((n, 1, dim))
    q[..., 0], k[0, 0, 0], v[0] = 1.0, 20.875, 0.0
    got, sums = M.attend_prompt(*(x.to(dtype).cuda() for x in (q, k, v)), scale=1.0, sums=True)
    # weights are e^20.875 and ones
    top, others = np.exp(20.875), np.arange(n)[:, None]
    assert np.abs(to_numpy(sums) - np.log(top + others)).max() <= 2.0 ** -16
    want = others / (top + others)
    # the rounding of the first weight, of the others, of the result
    assert np.all(np.abs(to_numpy(got) - want[..., None]) <= 2.5 * HALF[dtype] * want[..., None] + TINY[dtype])
