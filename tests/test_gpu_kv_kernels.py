"""The tests of test_gpu_kv.py by each kernel of the attention by name, with their tokens in one part and in several, and launches of very many workgroups."""
import numpy as np
import pytest

import kv_reference as ref
import test_gpu_kv as base
from test_gpu_kv import TYPES, check_attention, fill, ints, normal, pool, rng, sequences

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
M = pytest.importorskip("paper_2511_13061_amd")

FEW, MANY = 1, 2


def named(kernel, parts):
    M.set_tuning("attention_kernel", kernel)
    M.set_tuning("attention_parts", parts)


@pytest.fixture(autouse=True)
def by_estimate_again():
    yield
    named(0, 0)


# parts up to 16 are joined by one kernel, more of them by another
WAYS = [(FEW, 1), (FEW, 40), (MANY, 1), (MANY, 3)]
way = pytest.mark.parametrize("way", WAYS, ids=lambda w: f"{'few' if w[0] == FEW else 'many'}-{w[1]}")


@way
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(base.ATTENTION)))
def test_attention(case, dtype, way):
    named(*way)
    base.test_attention(case, dtype)


@way
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(base.PROMPT)))
def test_attention_of_many_rows(case, dtype, way):
    named(*way)
    base.test_attention_of_many_rows(case, dtype)


@way
@pytest.mark.parametrize("dtype", TYPES)
def test_large_and_extreme_scores(dtype, way):
    named(*way)
    base.test_attention_large_and_extreme_scores(dtype)


@way
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("asked", [4, 90])
@pytest.mark.parametrize("sizes", [(1e-4,), (2e-7, 1.0), (1.0, 3e4), (0.0, 1.0), (1e-6, 1e4, 0.0)])
def test_values_of_any_size(sizes, asked, dtype, way):
    named(*way)
    base.test_attention_values_of_any_size(sizes, asked, dtype)


@way
def test_what_is_masked_has_no_effect(way):
    named(*way)
    base.test_attention_what_is_masked_has_no_effect()
    for window in (0, 50):
        base.test_attention_of_many_rows_what_is_masked_has_no_effect(window)
    base.test_attention_values_that_are_not_finite_alone()


@way
def test_pages_that_are_needed_and_missing(way):
    named(*way)
    base.test_attention_pages_that_are_needed_and_missing()


@way
def test_strides_streams_and_graphs(way):
    named(*way)
    base.test_attention_strides_streams_and_other_memory()
    base.test_a_decoding_step_in_a_graph()


@pytest.mark.parametrize("parts", [1, 3])
def test_offsets_beyond_32_bits(parts):
    named(MANY, parts)
    base.test_offsets_beyond_32_bits()


@way
@pytest.mark.parametrize("dtype", TYPES)
def test_extreme_scores_of_many_queries(dtype, way):
    """Rows of one call with scores that grow, fall, are far apart or next to nothing, queries that are zero, huge, NaN and infinite among them."""
    named(*way)
    g = rng(61)
    page, dim, n, asked = 16, 64, 500, 70
    cache = pool(g, 32, page, 1, dim)
    tables = sequences(g, cache, [n])
    slots = tables[0, np.arange(n) // page] * page + np.arange(n) % page
    k = normal(g, n, 1, dim) + (torch.arange(n)[:, None, None] * 0.05).half()
    cache.append(None, k.cuda(), normal(g, n, 1, dim).cuda(), None, ints(slots))
    q = normal(g, asked, 2, dim, dtype=dtype)
    size = torch.tensor([1.0, 4.0, -4.0, 0.0, 100.0, 1e-6, 0.1])[torch.arange(asked) % 7]
    q = (q.float() * size[:, None, None] + (size.abs() == 4)[:, None, None] * size[:, None, None]).to(dtype)
    data = cache.data.cpu().numpy()
    call = dict(start=ints([0, asked]), most_queries=asked, sums=True)
    for scale in (0.125, -0.125, 0.0, 2.0):
        want = ref.attend(ref.to_numpy(q), data, page, tables, [n], [0, asked], scale=scale)
        got, sums = cache.attend(q.cuda(), ints(tables), ints([n]), scale=scale, **call)
        check_attention(got, sums, *want, dtype)
        alone = cache.attend(q.cuda(), ints(tables), ints([n]), scale=scale, **dict(call, sums=False))
        check_attention(alone, None, *want, dtype)
    clean = cache.attend(q.cuda(), ints(tables), ints([n]), **call)
    q[3, 0, 3], q[40, 1, 9] = float("nan"), float("inf")
    got = cache.attend(q.cuda(), ints(tables), ints([n]), **call)
    for x, y in zip(got, clean):
        hit = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
        hit[3, 0], hit[40, 1] = True, True
        assert torch.isnan(x[hit]).all() and torch.equal(x[~hit], y[~hit])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel", [FEW, MANY])
@pytest.mark.parametrize("batch,kv_heads,shared,asked", [(30, 32, 1, 1), (64, 16, 2, 3), (65, 16, 1, 2), (90, 12, 1, 1), (300, 4, 1, 1)])
def test_many_sequences(batch, kv_heads, shared, asked, kernel, dtype):
    """More workgroups than are under way at once, sequences of very different lengths (several of the same, some of none) in an order that is not theirs."""
    named(kernel, 1)
    g = rng(batch)
    page, dim = 16, 32
    lengths = torch.randint(0, 120, (batch,), generator=g).tolist()
    lengths[3], lengths[4], lengths[7], lengths[8] = 0, 0, 100, 100
    cache = pool(g, sum(-(-n // page) for n in lengths) + 2, page, kv_heads, dim)
    tables = sequences(g, cache, lengths)
    fill(g, cache, tables, lengths)
    start = np.arange(batch + 1) * asked
    q = normal(g, batch * asked, kv_heads * shared, dim, dtype=dtype)
    want = ref.attend(ref.to_numpy(q), cache.data.cpu().numpy(), page, tables, lengths, start)
    got, sums = cache.attend(q.cuda(), ints(tables), ints(lengths), start=ints(start), most_queries=asked, sums=True)
    check_attention(got, sums, *want, dtype)


@pytest.mark.parametrize("parts", [1, 3])
@pytest.mark.parametrize("page,window", [(16, 0), (256, 0), (64, 2990)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
def test_blocks_that_are_done_again(dim, page, window, parts):
    """bf16 results of rows for which one token without a value is 60 powers of two ahead, beside rows that see all tokens alike; one group of values is not a
    number, and the tokens that the last rows do not see are."""
    named(MANY, parts)
    g = rng(dim + page)
    tokens, asked, gap = 3000, 150, 60.0
    cache = pool(g, -(-tokens // page), page, 1, dim)
    tables = sequences(g, cache, [tokens])
    slots = tables[0, np.arange(tokens) // page] * page + np.arange(tokens) % page
    k, v = normal(g, tokens, 1, dim), normal(g, tokens, 1, dim) + 1
    k[..., :32] = 0
    first = 100                                                  # with the window: the last rows see from 10 on
    k[first, 0, :32], v[first] = 1, 0
    v[1, 0, 5] = float("nan")                                    # a group that the window hides from all rows but the first ones
    cache.append(None, k.cuda(), v.cuda(), None, ints(slots))
    q = torch.zeros((asked, 1, dim), dtype=torch.bfloat16)
    q[::2, :, :32] = 1.0
    scale = gap * np.log(2) / 32
    got = ref.to_numpy(cache.attend(q.cuda(), ints(tables), ints([tokens]), start=ints([0, asked]), most_queries=asked, scale=scale, window=window))
    values = ref.read(cache.data.cpu().numpy(), page, dim, slots)[1][:, 0]
    for i in range(asked):
        p = tokens - asked + i
        lo = max(0, p - window + 1) if window else 0
        w = np.exp(-32 * float(np.float32(scale))) if i % 2 == 0 else 1.0
        weight = np.where(np.arange(lo, p + 1) == first, 1.0, w)
        want = weight @ values[lo:p + 1] / weight.sum()
        fine = ~np.isnan(want)
        assert np.array_equal(np.isnan(got[i, 0]), ~fine) and fine.sum() == dim - 32 * (lo <= 1)
        assert np.linalg.norm((got[i, 0] - want)[fine]) <= (base.HALF[torch.bfloat16] + 2.0 ** -14) * np.linalg.norm(want[fine])
