"""One decoder layer with pruned weights and its keys and values in 4 bits: a prompt in parts of up to 64 tokens, then single tokens.

The seven products are sparse (macko_spmm for a part of the prompt, macko_spmv_group for a token), queries and keys are normalised and turned
and put into the cache in one launch (macko_kv_append), and attention reads the cache (macko_kv_attention).  What is left, the norm of the
residual stream and the gate, is plain PyTorch.  Weights and inputs are random.

    python examples/decoder_layer.py [--tokens 200] [--steps 32] [--hidden 4096 --inner 11008 --heads 32 --kv-heads 32] [--sparsity 0.5]

Prints the time of a part and of a step, and how far the attention's results are from the same in 32 bits over the values that the cache holds.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_13061_amd as M  # noqa: E402


def pruned(rows, cols, sparsity, gen):
    w = torch.randn((rows, cols), generator=gen, device="cuda") * cols ** -0.5
    return M.encode_device((w * (torch.rand((rows, cols), generator=gen, device="cuda") >= sparsity)).half())


class Layer:
    def __init__(self, hidden, inner, heads, kv_heads, sparsity, most_tokens, page=16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, hidden // heads
        shapes = dict(q=(hidden, hidden), k=(kv_heads * self.dim, hidden), v=(kv_heads * self.dim, hidden), o=(hidden, hidden),
                      gate=(inner, hidden), up=(inner, hidden), down=(hidden, inner))
        self.w = {name: pruned(*shape, sparsity, gen) for name, shape in shapes.items()}
        self.norms = [torch.ones(hidden, device="cuda") for _ in range(2)]
        self.q_norm, self.k_norm = (torch.ones(self.dim, dtype=torch.float16, device="cuda") for _ in range(2))
        pages = -(-most_tokens // page)
        self.cache = M.KvCache(pages, page, kv_heads, self.dim)
        self.table = torch.randperm(pages, device="cuda").to(torch.int32)[None]      # the sequence's pages, in no order
        self.rope = M.rope_table(most_tokens, self.dim)
        self.length = 0

    def products(self, names, x):
        """The products of x [tokens, cols] with these weights: a group of matrix-vector products for one token."""
        if x.shape[0] == 1:
            return [y[None] for y in M.spmv_group([self.w[n] for n in names], [x[0]] * len(names))]
        return [self.w[n].spmm(x) for n in names]

    def norm(self, x, weight):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight).half()

    def attention(self, x):
        """The heads' results for the next tokens x [tokens, hidden]; their keys and values stay in the cache."""
        n = x.shape[0]
        q, k, v = (y.view(n, -1, self.dim) for y in self.products(["q", "k", "v"], x))
        at = torch.arange(self.length, self.length + n, device="cuda", dtype=torch.int32)
        slots = self.table[0, (at // self.cache.page_size).long()] * self.cache.page_size + at % self.cache.page_size
        q = self.cache.append(q, k, v, at, slots, self.rope, q_weight=self.q_norm, k_weight=self.k_norm)
        self.length += n
        lengths = torch.tensor([self.length], device="cuda", dtype=torch.int32)
        start = torch.tensor([0, n], device="cuda", dtype=torch.int32)
        return q, self.cache.attend(q, self.table, lengths, start=start, most_queries=n, longest=self.length)

    def __call__(self, x):
        self.q, self.seen = self.attention(self.norm(x, self.norms[0]))
        x = x + self.products(["o"], self.seen.reshape(x.shape[0], -1))[0]
        gate, up = self.products(["gate", "up"], self.norm(x, self.norms[1]))
        return x + self.products(["down"], torch.nn.functional.silu(gate.float()).mul(up).half())[0]

    def plain_attention(self):
        """The last call's attention in 32 bits, from the values that the cache holds."""
        at = torch.arange(self.length, device="cuda", dtype=torch.int32)
        page = self.cache.page_size
        k, v = (y.float().repeat_interleave(self.heads // self.kv_heads, 1).transpose(0, 1).contiguous()
                for y in self.cache.read(self.table[0, (at // page).long()] * page + at % page))
        q = self.q.float().transpose(0, 1)
        score = q @ k.transpose(1, 2).contiguous() * self.dim ** -0.5
        n = q.shape[1]
        score = score.masked_fill(torch.arange(self.length, device="cuda") > torch.arange(self.length - n, self.length, device="cuda")[:, None], -float("inf"))
        return (score.softmax(-1) @ v).transpose(0, 1)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 200), ("steps", 32), ("hidden", 4096), ("inner", 11008), ("heads", 32), ("kv-heads", 32)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--sparsity", type=float, default=0.5)
    a = p.parse_args(argv)
    layer = Layer(a.hidden, a.inner, a.heads, a.kv_heads, a.sparsity, a.tokens + a.steps)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.tokens + a.steps, a.hidden), generator=gen, device="cuda").half()
    far = 0.0
    for name, parts in (("part", [x[i:min(i + 64, a.tokens)] for i in range(0, a.tokens, 64)]), ("step", list(x[a.tokens:].split(1)))):
        times = []
        for part in parts:
            torch.cuda.synchronize()
            t = time.perf_counter()
            y = layer(part)
            torch.cuda.synchronize()
            times.append(time.perf_counter() - t)
            want = layer.plain_attention()
            far = max(far, float((layer.seen.float() - want).norm() / want.norm()))
            assert torch.isfinite(y).all()
        if times:
            print(f"{len(times)} {name}s of {len(parts[0])} tokens: {sorted(times)[len(times) // 2] * 1e6:.0f} us each")
    held = layer.cache.data.numel()
    print(f"{layer.length} tokens in {held / 2 ** 20:.2f} MiB ({held * 8 / (2 * layer.cache.pages * layer.cache.page_size * a.kv_heads * layer.dim):.2f} bits a value); attention against 32 bits: {far:.1e}")
    return far


if __name__ == "__main__":
    main()
