"""Attention in 16 and 8 bits, as timed cases: a prompt over its own keys and values, and a key/value cache in 8 bits, what fills it and what reads it.

  prompt  causal attention of packed sequences over keys and values in 16 bits
  append  queries and keys of the last tokens of sequences normalised (optional) and turned by position; keys and values go to 8 bits and into
          a paged cache; then the whole pool is read back, so that all that the cache now stands for is there to compare
  attend  attention of one or several query tokens a sequence over the paged cache
  read    the values of a list of cache slots

The cache holds blocks of 16 tokens of one head: codes in the 8-bit floating point format E4M3 and one byte b for the keys and one for the
values, a factor 2^(b - 127).  b is the least one from 1 to 246 that brings the largest finite magnitude to 448 at most.  Where new tokens join
others in a block, b is the larger one of what the block has and what the new ones need, and the codes of the tokens before them are rounded again to
the new factor.  Codes are rounded to nearest, ties to even, and stop at 448; what is not finite is stored as NaN.
With D channels a block is   key codes [16][D] | value codes [4][D][4] (byte [t / 4][channel][t % 4])
"""
import math
import random

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 16
MOST_CELLS = 64 * 4096 * 32 * 128          # cached values of the largest attention case
MOST_SCORES = 2 * 32 * 1024 * 8192         # its largest table of scores


def listed():
    def prompt(name, batch, longest, heads, kv_heads, dim, **more):
        return dict(dict(name=name, op="prompt", batch=batch, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, ragged=True, window=0, sums=False,
                         type="fp16"), **more)

    def append(name, batch, fresh, past, heads, kv_heads, dim, rot, page, **more):
        return dict(dict(name=name, op="append", batch=batch, fresh=fresh, past=past, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, page=page, norm=False,
                         interleaved=False, ragged=True, type="fp16"), **more)

    def attend(name, batch, longest, heads, kv_heads, dim, page, **more):
        return dict(dict(name=name, op="attend", batch=batch, longest=longest, heads=heads, kv_heads=kv_heads, dim=dim, page=page, queries=1,
                         ragged=True, empty=0, window=0, sums=False, type="fp16"), **more)

    def read(name, tokens, kv_heads, dim, page, **more):
        return dict(dict(name=name, op="read", tokens=tokens, kv_heads=kv_heads, dim=dim, page=page, scatter=False, skips=False, type="fp16"), **more)

    return [
        # a short question to a 7B-shaped layer: latency
        prompt("prompt_1x33", 1, 33, 32, 32, 128),
        # prompts of many requests side by side, none as long as another, a window; the sums let the results be joined with a cached prefix's
        prompt("prompt_13x1021_window", 13, 1021, 40, 8, 64, window=500, sums=True),
        # long documents
        prompt("prompt_3x8191_bf16", 3, 8191, 32, 8, 128, type="bf16"),
        # one token of a 7B-shaped layer goes into its cache, behind others of its block: latency
        append("append8_1x32x128", 1, 1, 99, 32, 32, 128, 128, 16),
        # the keys and values of long prompts, heads normalised, half of each turned, neighbours paired
        append("append8_5x4096_norm_bf16", 5, 4096, 700, 32, 8, 128, 64, 64, norm=True, interleaved=True, type="bf16"),
        # decoding at the start of a conversation: latency
        attend("attend8_1x50", 1, 50, 32, 32, 128, 16),
        # decoding one sequence at the end of a long context: few heads, all parallelism is along the cache
        attend("attend8_1x131072", 1, 131072, 32, 8, 128, 64),
        # decoding a batch of a 7B-shaped layer (a cache head for every head)
        attend("attend8_64x4096", 64, 4096, 32, 32, 128, 16),
        # several proposed tokens of each sequence checked at once, a window, sequences without tokens; the sums let the result be joined with others
        attend("attend8_37x2999_window", 37, 2999, 40, 8, 64, 32, queries=5, empty=4, window=1000, sums=True),
        # the next part of two long prompts over what is cached of them
        attend("attend8_2x8192_chunk_bf16", 2, 8192, 32, 8, 128, 64, queries=1024, ragged=False, type="bf16"),
        # single tokens back in any order, wide heads
        read("read8_257x256_bf16", 257, 8, 256, 16, scatter=True, skips=True, type="bf16"),
        # a long prefix back for a computation in 16 bits
        read("read8_65536x128", 65536, 8, 128, 64),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 1e15)


def draw(rng):
    """One more case of the same ranges, that costs no more than the largest listed one of its kind."""
    while True:
        case = _drawn(rng)
        if _cost(case) <= max(_cost(c) for c in listed() if c["op"] == case["op"]):
            return case


def _drawn(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    op = rng.choice(["prompt"] * 4 + ["append"] * 3 + ["attend"] * 6 + ["read"] * 2)
    dim = rng.choice([32, 64, 64, 96, 128, 128, 128, 160, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    page = rng.choice([16, 32, 64, 128, 256])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8] if kv_heads <= 8 else [1])
    case = dict(op=op, heads=heads, kv_heads=kv_heads, dim=dim, type=rng.choice(["fp16", "bf16"]))
    ragged = rng.random() < 0.7
    if op == "prompt":
        longest = size(1, 8191)
        batch = size(1, max(1, min(64, 24573 * 48 * 128 // (longest * (heads + 2 * kv_heads) * dim))))
        return dict(case, batch=batch, longest=longest, ragged=ragged, window=rng.choice([0, 0, size(1, 4096)]), sums=rng.random() < 0.3)
    if op == "append":
        batch = size(1, 64)
        fresh = rng.choice([1, 1, rng.randint(2, 8), size(9, 16384)])
        fresh = max(1, min(fresh, 20480 * 48 * 128 // (batch * (heads + 2 * kv_heads) * dim)))
        past = min(rng.choice([0, size(1, 1000), size(1, 8192)]), 20480 * 8 * 128 // (batch * kv_heads * dim))
        return dict(case, batch=batch, fresh=fresh, past=past, page=page, rot=16 * rng.randint(1, dim // 16) if rng.random() < 0.5 else dim,
                    norm=rng.random() < 0.5, interleaved=rng.random() < 0.4, ragged=ragged)
    if op == "read":
        del case["heads"]
        return dict(case, tokens=size(1, min(65536, 65536 * 8 * 128 // (kv_heads * dim))), page=page, scatter=rng.random() < 0.5, skips=rng.random() < 0.3)
    longest = size(1, 131072)
    batch = size(1, max(1, min(64, MOST_CELLS // (longest * kv_heads * dim))))
    queries = min(rng.choice([1, 1, 1, 2, 5, 8, size(9, 1024)]), longest, max(1, MOST_SCORES // (batch * heads * longest)))
    return dict(case, batch=batch, longest=longest, page=page, queries=queries, ragged=ragged,
                empty=rng.choice([0, 0, batch // 8]), window=rng.choice([0, 0, 0, size(1, 8192)]), sums=rng.random() < 0.3)


# ---- inputs -----------------------------------------------------------------

def _shape(case):
    """Lengths of the sequences and numbers of their query tokens, in an order that the seed changes."""
    if case["op"] == "append":
        n, fresh, past = case["batch"], case["fresh"], case["past"]
        r = random.Random("%d %d %d" % (n, fresh, past))
        asked = [r.randint(max(1, fresh // 4), fresh) if case["ragged"] and i else fresh for i in range(n)]
        return [a + (r.randint(0, past) if case["ragged"] and i else past) for i, a in enumerate(asked)], asked
    r = random.Random("%d %d" % (case["batch"], case["longest"]))
    n, longest = case["batch"], case["longest"]
    lengths = [r.randint(max(1, longest // 4), longest) if case["ragged"] and i else longest for i in range(n)]
    if case["op"] == "prompt":
        return lengths, lengths
    queries = case["queries"]
    asked = [min(length, r.randint(1, queries) if case["ragged"] and i else queries) for i, length in enumerate(lengths)]
    for i in range(1, min(n, 1 + case["empty"])):       # a place of the batch that nothing occupies still has its query row
        lengths[i], asked[i] = 0, 1
    return lengths, asked


def _seen(case):
    """Tokens that a sequence's queries reach, and pairs of a query and a token, over all sequences."""
    tokens = pairs = 0
    for length, asked in zip(*_shape(case)):
        window = case["window"] or length
        first = max(0, length - asked + 1)              # what the first query could see
        full = max(0, min(asked, length - max(window, first) + 1)) if length else 0      # queries that see a whole window
        rest = asked - full if length else 0
        tokens += min(length, window + asked - 1)
        pairs += full * window + rest * first + rest * (rest - 1) // 2
    return tokens, pairs


def _pool(case):
    if case["op"] == "read":
        return -(-case["tokens"] // case["page"]) + (3 if case["scatter"] else 1)
    return sum(-(-n // case["page"]) for n in _shape(case)[0]) + 3


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)


def _channels(gen, heads, dim):
    """Keys have a few channels that are larger than the others."""
    wide = torch.rand((heads, dim), generator=gen, device="cuda") < 0.04
    return torch.where(wide, 4.0, 0.9)


def _fill(gen, data, scales, dim):
    """A pool that holds keys and values, some blocks of smaller numbers than others."""
    pages, heads, blocks = scales.shape[:3]
    channels = _channels(gen, heads, dim)[:, None, None]
    step = max(1, (64 << 20) // (heads * blocks * BLOCK * dim))
    for i in range(0, pages, step):
        part = data[i:i + step]
        shape = (len(part), heads, blocks, BLOCK, dim)
        size = torch.exp2(-3.0 * torch.rand(shape[:3] + (1, 1), generator=gen, device="cuda"))
        for j, x in enumerate((_normal(gen, *shape) * channels * size, _normal(gen, *shape) * size)):
            byte = _byte(x.abs().amax((-1, -2)))
            codes = _codes(x, byte[..., None, None])
            if j:
                codes = codes.unflatten(3, (4, 4)).transpose(4, 5)
            part[:, :, :, j] = codes.flatten(3)
            scales[i:i + step, :, :, j] = byte


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, dim, op = TYPES[case["type"]], case["dim"], case["op"]
    s = dict(case, kind=kind)
    kv_heads = case["kv_heads"]
    if op != "read":
        lengths, asked = _shape(case)
        mix = torch.randperm(len(lengths), generator=gen, device="cuda").tolist()
        lengths, asked = [lengths[i] for i in mix], [asked[i] for i in mix]
        start = torch.tensor([0] + asked, device="cuda").cumsum(0)
        s.update(asked=asked, most=max(asked), start=start.to(torch.int32), lengths=torch.tensor(lengths, device="cuda", dtype=torch.int32),
                 scale=dim ** -0.5, single=max(asked) == 1)
    if op in ("prompt", "append"):
        # one projection's output, whose parts are the heads of each kind
        tokens, heads = sum(asked), case["heads"]
        fused = _normal(gen, tokens, heads + 2 * kv_heads, dim)
        fused[:, heads:heads + kv_heads] *= _channels(gen, kv_heads, dim)
        fused = fused.to(kind)
        s["q"], s["k"], s["v"] = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    if op == "prompt":
        return s
    if op == "append":
        rot = case["rot"]
        angle = torch.arange(max(lengths), device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 / rot * torch.arange(rot // 2, device="cuda", dtype=torch.float64))
        s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float()
        s["positions"] = torch.cat([torch.arange(n - a, n, device="cuda", dtype=torch.int32) for n, a in zip(lengths, asked)])
        s["weights"] = [(1.0 + 0.2 * _normal(gen, dim)).to(kind) if case["norm"] else None for _ in range(2)]
    page, pages = case["page"], _pool(case)
    s["data"] = torch.empty((pages, kv_heads, page // BLOCK, 2, BLOCK * dim), dtype=torch.uint8, device="cuda")
    s["scales"] = torch.empty((pages, kv_heads, page // BLOCK, 2), dtype=torch.uint8, device="cuda")
    _fill(gen, s["data"], s["scales"], dim)
    order = torch.randperm(pages, generator=gen, device="cuda")
    if op != "read":
        # entries that no token needs name anything
        tables = torch.randint(-(1 << 30), 1 << 30, (len(lengths), -(-max(lengths) // page) + 2), generator=gen, device="cuda", dtype=torch.int32)
        stale = torch.ones((pages, page), dtype=torch.bool, device="cuda")
        used = 0
        for i, n in enumerate(lengths):
            need = -(-n // page)
            tables[i, :need] = order[used:used + need]
            stale[order[used:used + need]] = torch.arange(need * page, device="cuda").view(need, page) >= n
            used += need
        s["tables"] = tables
    if op == "attend":
        s["q"] = _normal(gen, sum(asked), case["heads"], dim).to(kind)
        # what no sequence holds is left over from others, or was never written
        at, within = stale.nonzero(as_tuple=True)
        keys, values = _parts(s["data"], dim)
        dirt = torch.randint(0, 256, (len(at), kv_heads, 2 * dim), generator=gen, device="cuda", dtype=torch.uint8)
        keys[at, :, within // BLOCK, within % BLOCK] = dirt[..., :dim]
        values[at, :, within // BLOCK, within % BLOCK // 4, :, within % 4] = dirt[..., dim:]
        whole = stale.view(pages, page // BLOCK, BLOCK).all(-1)
        s["scales"].transpose(1, 2)[whole] = torch.randint(0, 256, (int(whole.sum()), kv_heads, 2), generator=gen, device="cuda", dtype=torch.uint8)
    if op == "append":
        s["every"] = torch.arange(pages * page, device="cuda", dtype=torch.int32)
    if op == "read":
        n = case["tokens"]
        slots = torch.randperm(pages * page, generator=gen, device="cuda") if case["scatter"] else (
            order[:, None] * page + torch.arange(page, device="cuda")).view(-1)
        slots = slots[:n].to(torch.int32)
        if case["skips"]:
            slots[::13] = -1
        s["slots"] = slots
    if own:
        import paper_2511_13061_amd as M
        s["cache"] = M.KvCache8(pages, page, kv_heads, dim, data=s["data"], scales=s["scales"])
    return s


# ---- the plain form ----------------------------------------------------------

def _byte(most):
    """The byte of blocks whose largest finite magnitude is `most`, in 32 bits: 448 is 1.75 * 2^8, and a mantissa above 1.75 carries."""
    return (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(1, 246).to(torch.uint8)


def _power(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _codes(x, byte):
    """8-bit codes of x in 32 bits, in units of 2^(byte - 127)."""
    finite = x.isfinite()
    scaled = torch.where(finite, x, 0.0) * _power(254 - byte.to(torch.int32))
    codes = scaled.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(finite, codes, 0x7F)


def _values(codes, byte):
    return codes.view(torch.float8_e4m3fn).float() * _power(byte)


def _parts(data, dim):
    """Key codes [pages, heads, blocks, 16, dim] and value codes [pages, heads, blocks, 4, dim, 4]."""
    return data[:, :, :, 0].unflatten(3, (BLOCK, dim)), data[:, :, :, 1].unflatten(3, (4, dim, 4))


def _turn(x, table, positions, weight, eps, rot, interleaved):
    x = x.float()
    if weight is not None:
        x = x * (1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()) * weight.float()
    c, s = table[positions.long()][:, None].unbind(2)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_read(s, slots):
    keys, values = _parts(s["data"], s["dim"])
    there, slot = (slots >= 0)[:, None, None], slots.long().clamp(min=0)
    page, block, at = slot // s["page"], slot % s["page"] // BLOCK, slot % BLOCK
    byte = s["scales"][page, :, block]
    got = [_values(keys[page, :, block, at], byte[..., :1]), _values(values[page, :, block, at // 4, :, at % 4], byte[..., 1:])]
    return [torch.where(there, x, 0.0).to(s["kind"]) for x in got]


def _plain_append(s):
    how, page, dim = (s["rot"], s["interleaved"]), s["page"], s["dim"]
    q = _turn(s["q"], s["table"], s["positions"], s["weights"][0], 1e-6, *how).to(s["kind"])
    fresh = [_turn(s["k"], s["table"], s["positions"], s["weights"][1], 1e-6, *how), s["v"].float()]
    start, tokens = s["start"].long(), len(q)
    t = torch.arange(tokens, device="cuda")
    of = torch.searchsorted(start, t, right=True) - 1
    place = s["lengths"].long()[of] - start[of + 1] + t
    block = s["tables"].long()[of, place // page] * (page // BLOCK) + place % page // BLOCK      # of the pool
    at = place % BLOCK
    blocks = s["scales"].shape[0] * s["scales"].shape[2]
    first = torch.full((blocks,), BLOCK, device="cuda").scatter_reduce(0, block, at, "amin")
    touched = (first < BLOCK)[:, None]
    codes = [x.transpose(1, 2).flatten(0, 1) for x in _parts(s["data"], dim)]                    # a block of the pool in front
    codes = [codes[0], codes[1].transpose(3, 4).flatten(2, 3)]                                   # [blocks, heads, 16, dim]
    old = s["scales"].transpose(1, 2).flatten(0, 1)
    before = torch.arange(BLOCK, device="cuda") < first[:, None]
    made, bytes_ = [], []
    for j, x in enumerate(fresh):
        finite = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
        most = torch.zeros((blocks, x.shape[1]), device="cuda").scatter_reduce(0, block[:, None].expand_as(finite), finite, "amax")
        need, had = _byte(most), old[..., j]
        byte = torch.where(touched, torch.where((first == 0)[:, None], need, torch.maximum(need, had)), had)
        again = _codes(_values(codes[j], had[..., None, None]), byte[..., None, None])
        c = torch.where((before & touched)[:, None, :, None], again, codes[j])
        c[block, :, at] = _codes(x, byte[block][..., None])
        made.append(c)
        bytes_.append(byte)
    pages, heads = s["scales"].shape[:2]
    back = lambda x: x.unflatten(0, (pages, -1)).transpose(1, 2)  # noqa: E731
    keys, values = _parts(s["data"], dim)
    keys[:] = back(made[0])
    values[:] = back(made[1].unflatten(2, (4, 4)).transpose(3, 4))
    s["scales"][:] = back(torch.stack(bytes_, -1))
    return [q] + _plain_read(s, s["every"])


def _softmax(score, seen, values):
    """Weighted values and logarithms of sums over the last axis of `score`, of what is seen."""
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, (score - top.clamp(min=-3e38)).exp(), 0.0)
    total = p.sum(-1, keepdim=True)
    out = p @ values / torch.where(total > 0, total, 1.0)
    return out, torch.where(total > 0, top + total.log(), -math.inf)


def _plain_attend(s):
    page, dim, kv_heads, shared = s["page"], s["dim"], s["kv_heads"], s["heads"] // s["kv_heads"]
    length, start = s["lengths"].long(), s["start"].long()
    batch, most = len(length), s["most"]
    table = s["tables"].long().clamp(0, len(s["data"]) - 1)
    far = table.shape[1] * page
    codes, byte = _parts(s["data"], dim), s["scales"]
    along = lambda x: x.transpose(1, 2).reshape(batch, kv_heads, far, dim)  # noqa: E731
    keys = along(_values(codes[0][table], byte[table][..., :1, None]).flatten(3, 4))
    values = along(_values(codes[1][table], byte[table][..., 1:, None, None]).transpose(5, 6).flatten(3, 5))
    asked = start[1:] - start[:-1]
    i = torch.arange(most, device="cuda")
    row = (start[:-1, None] + i).clamp(max=len(s["q"]) - 1)
    q = s["q"].float()[row].view(batch, most, kv_heads, shared, dim).permute(0, 2, 1, 3, 4).reshape(batch, kv_heads, most * shared, dim)
    t = torch.arange(far, device="cuda")
    at = (length - asked)[:, None] + i                                                     # a query's own place
    seen = (t <= at[..., None]) & (t < length[:, None, None])
    if s["window"]:
        seen &= t > at[..., None] - s["window"]
    seen = seen[:, None, :, None].expand(-1, kv_heads, -1, shared, -1).reshape(batch, kv_heads, most * shared, far)
    held = (t < length[:, None])[:, None, :, None]
    out, sums = _softmax(q @ keys.transpose(2, 3) * s["scale"], seen, torch.where(held, values, 0.0))
    back = lambda x: x.view(batch, kv_heads, most, shared, -1).permute(0, 2, 1, 3, 4).reshape(batch, most, s["heads"], -1)  # noqa: E731
    token = torch.arange(len(s["q"]), device="cuda")
    of = torch.searchsorted(start, token, right=True) - 1
    out, sums = (back(x)[of, token - start[of]] for x in (out, sums))
    return [out.to(s["kind"]), sums[..., 0]] if s["sums"] else [out.to(s["kind"])]


def _plain_prompt(s):
    dim, kv_heads, shared = s["dim"], s["kv_heads"], s["heads"] // s["kv_heads"]
    outs, totals, first = [], [], 0
    for n in s["asked"]:
        q, k, v = (x[first:first + n].float() for x in (s["q"], s["k"], s["v"]))
        first += n
        q = q.view(n, kv_heads, shared, dim).permute(1, 2, 0, 3).reshape(kv_heads, shared * n, dim)
        i = torch.arange(n, device="cuda")
        seen = i <= i[:, None]
        if s["window"]:
            seen &= i > i[:, None] - s["window"]
        score = (q @ k.permute(1, 2, 0) * s["scale"]).view(kv_heads, shared, n, n)
        out, sums = _softmax(score, seen, v.transpose(0, 1)[:, None])
        outs.append(out.permute(2, 0, 1, 3).reshape(n, s["heads"], dim))
        totals.append(sums[..., 0].permute(2, 0, 1).reshape(n, s["heads"]))
    out = torch.cat(outs).to(s["kind"])
    return [out, torch.cat(totals)] if s["sums"] else [out]


def run(s):
    op = s["op"]
    if op == "prompt":
        if not own:
            return _plain_prompt(s)
        import paper_2511_13061_amd as M
        got = M.attend_prompt(s["q"], s["k"], s["v"], s["start"], longest=s["most"], scale=s["scale"], window=s["window"], sums=s["sums"])
        return list(got) if s["sums"] else [got]
    if op == "append":
        if not own:
            return _plain_append(s)
        cache = s["cache"]
        start = None if s["single"] else s["start"]
        q = cache.append(s["q"], s["k"], s["v"], s["positions"], s["tables"], s["lengths"], start=start, table=s["table"], q_weight=s["weights"][0],
                         k_weight=s["weights"][1], eps=1e-6, interleaved=s["interleaved"])
        return [q, *cache.read(s["every"], s["kind"])]
    if op == "read":
        return list(s["cache"].read(s["slots"], s["kind"])) if own else _plain_read(s, s["slots"])
    if not own:
        return _plain_attend(s)
    more = {} if s["single"] else {"start": s["start"], "most_queries": s["most"]}
    got = s["cache"].attend(s["q"], s["tables"], s["lengths"], longest=s["longest"], scale=s["scale"], window=s["window"], sums=s["sums"], **more)
    return list(got) if s["sums"] else [got]


def work(case):
    dim, op, held = case["dim"], case["op"], 2 * case["kv_heads"] * case["dim"]            # values that a token has in the cache
    if op == "read":
        put = case["tokens"] - (len(range(0, case["tokens"], 13)) if case["skips"] else 0)
        return dict(bytes=put * held + case["tokens"] * (2 * held + 4), flops=put * held)
    if op == "append":
        tokens, pool = sum(_shape(case)[1]), _pool(case) * case["page"]
        turned = tokens * (case["heads"] + case["kv_heads"]) * dim
        return dict(bytes=4 * tokens * case["heads"] * dim + 4 * tokens * (case["rot"] + 1) + 3 * tokens * held + pool * (3 * held + 4),
                    flops=6 * turned + 4 * tokens * held + pool * held)
    tokens, pairs = _seen(case)
    rows = sum(_shape(case)[1]) * case["heads"]
    bytes_ = rows * (4 * dim + 4 * case["sums"]) + (2 * tokens * held if op == "prompt" else tokens * held + 4 * -(-tokens // case["page"]))
    return dict(bytes=bytes_, flops=4 * pairs * case["heads"] * dim)


# ---- the same from the definitions, in 64 bits ---------------------------------

def _exact_turn(x, s, weight):
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / s["dim"] + 1e-6) * weight.double()
    rot = s["rot"]
    near = torch.arange(rot // 2, device="cuda") * (2 if s["interleaved"] else 1)
    far = near + (1 if s["interleaved"] else rot // 2)
    angle = s["table"].double()[s["positions"].long()]
    wave = torch.complex(angle[:, 0], angle[:, 1])[:, None]
    z = torch.complex(x[..., near], x[..., far]) * wave
    y = x.clone()
    y[..., near], y[..., far] = z.real, z.imag
    return y


def _exact_numbers():
    """What the 256 codes stand for."""
    numbers = []
    for code in range(256):
        exponent, fraction = code >> 3 & 15, code & 7
        x = math.ldexp(8 + fraction, exponent - 10) if exponent else math.ldexp(fraction, -9)
        numbers.append((math.nan if code & 127 == 127 else x) * (-1.0 if code & 128 else 1.0))
    return torch.tensor(numbers, dtype=torch.float64, device="cuda")


def _exact_round(x, unit):
    """x as the nearest multiple of the unit that the format has."""
    y = (x / unit).abs().clamp(max=448.0)
    gap = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3.0)                 # torch.round takes ties to even
    return torch.round(y / gap) * gap * unit * x.sign()


def _exact_unit(x):
    """The least power of two that brings x [..., tokens, dim] to 448 at most."""
    most = x.abs().amax((-1, -2), keepdim=True)
    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -140) / 448.0))
    e = torch.where(most > 448.0 * torch.exp2(e), e + 1, torch.where(most <= 448.0 * torch.exp2(e - 1), e - 1, e))
    return torch.exp2(e.clamp(-126.0, 119.0))


def _exact_slots(s, slots):
    """Keys and values of slots >= 0 in 64 bits, taken out of the pool byte by byte."""
    page, dim = s["page"], s["dim"]
    numbers, slots = _exact_numbers(), slots.long()
    flat, bytes_ = s["data"].view(-1), s["scales"].view(-1)
    block = ((slots // page)[:, None] * s["kv_heads"] + torch.arange(s["kv_heads"], device="cuda")) * (page // BLOCK) + (slots % page // BLOCK)[:, None]
    t, d = (slots % BLOCK)[:, None, None], torch.arange(dim, device="cuda")
    got = []
    for j, at in enumerate((t * dim + d, (t // 4 * dim + d) * 4 + t % 4)):
        code = flat[(block * 2 + j)[..., None] * (BLOCK * dim) + at]
        got.append(numbers[code.long()] * torch.exp2(bytes_[block * 2 + j].double() - 127.0)[..., None])
    return got


def _exact_append(s):
    page = s["page"]
    pool = _exact_slots(s, s["every"])
    fresh = [_exact_turn(s["k"], s, s["weights"][1]), s["v"].double()]
    start, tables = s["start"].tolist(), s["tables"].tolist()
    bytes_ = s["scales"]
    for b, length in enumerate(s["lengths"].tolist()):
        place = length - (start[b + 1] - start[b])
        while place < length:
            a, end = place % BLOCK, min(length, place // BLOCK * BLOCK + BLOCK)
            base = tables[b][place // page] * page + place // BLOCK * BLOCK % page          # the block's first slot
            row = start[b + 1] - length + place
            for j in range(2):
                x = fresh[j][row:row + end - place].transpose(0, 1)                         # [heads, tokens, dim]
                had = torch.exp2(bytes_[base // page, :, base % page // BLOCK, j].double() - 127.0)[:, None, None]
                unit = _exact_unit(x)
                if a:
                    unit = torch.maximum(unit, had)
                    pool[j][base:base + a] = _exact_round(pool[j][base:base + a].transpose(0, 1), unit).transpose(0, 1)
                pool[j][base + a:base + a + end - place] = _exact_round(x, unit).transpose(0, 1)
                last = base + a + end - place                                               # what lies behind keeps its codes
                pool[j][last:base + BLOCK] *= (unit / had)[:, 0]
            place = end
    return [_exact_turn(s["q"], s, s["weights"][0]), *pool]


def _exact_rows(q, keys, values, first, s):
    """Rows q [n, heads, dim] at the places first, first + 1, ... over keys and values [tokens, kv heads, dim]: results and sums."""
    out, sums = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    t, at = torch.arange(len(keys), device="cuda"), (first + torch.arange(len(q), device="cuda"))[:, None]
    hidden = (t > at) | ((t <= at - s["window"]) if s["window"] else False)
    for h in range(q.shape[1]):
        g = h // (q.shape[1] // keys.shape[1])
        score = q[:, h].double() @ keys[:, g].T * s["scale"]
        score[hidden] = -math.inf
        sums[:, h] = score.logsumexp(-1)
        out[:, h] = score.softmax(-1) @ values[:, g]
    return out, sums


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "read":
        there = s["slots"] >= 0
        out = []
        for x in _exact_slots(s, s["slots"].clamp(min=0)):
            x[~there] = 0.0
            out.append(x)
        return out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    sums = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    start = s["start"].tolist()
    for b, length in enumerate(s["lengths"].tolist()):
        mine = slice(start[b], start[b + 1])
        if not length:
            continue
        if case["op"] == "prompt":
            keys, values = s["k"][mine].double(), s["v"][mine].double()
        else:
            t = torch.arange(length, device="cuda")
            keys, values = _exact_slots(s, s["tables"][b, t // s["page"]].long() * s["page"] + t % s["page"])
        out[mine], sums[mine] = _exact_rows(s["q"][mine], keys, values, length - (start[b + 1] - start[b]), s)
    return [out, sums] if s["sums"] else [out]
