"""Attention over the 4-bit cache where its statistics, masks and launches are stretched, in both of its kernels, against 64 bits.

Tolerances as in test_gpu_kv.py: half a unit in the last place of a result, 2^-16 for a weight, and for a score a few roundings in 32 bits where its
products are few and exact."""
import math

import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import HALF, TINY, TYPES, attend_with_room, ints, normal, pool, rng, sequences

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
M = pytest.importorskip("paper_2511_13061_amd")

# rows of q (with very many the kernel for many rows is taken), and what is said of the longest sequence (1: it is in one part)
KERNELS = {"few": (0, None), "few, one part": (0, 1), "many": (2 ** 17, None)}


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
