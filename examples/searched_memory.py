"""A memory that is searched: one attention layer whose long context lies in an 8-bit cache and is read through PAG searches.

The context's keys are written into the cache, read back as the numbers that the cache holds, and indexed, one index for each
key/value head.  A decoding step then gives every request a new token: its key and value are appended, its queries are searched, and attention
reads the K tokens found and the last `window` ones.  Attention over all tokens shows what that leaves out.  Every `block` tokens the
indexes take the keys that have left the window.

An index ranks by distance and attention by inner product: keys get one coordinate more, sqrt(R^2 - |k|^2) with R the longest key's length, queries
a zero, and |q' - k'|^2 = |q|^2 + R^2 - 2 <q, k>.

    python examples/searched_memory.py [--tokens 20000] [--steps 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_06660_amd import KvCache, KvTables, PagIndex  # noqa: E402


class SearchedMemory:
    """The cache, block table and indexes of one request in one layer."""

    def __init__(self, capacity, kv_heads=4, heads=16, head_dim=64, page_tokens=64, window=256, block=64, K=64, efS=1024, format="int8"):
        self.kv_heads, self.heads, self.dim, self.window, self.block, self.K, self.efS = kv_heads, heads, head_dim, window, block, K, efS
        pages = -(-capacity // page_tokens)
        self.tables = KvTables(1, pages, pages, page_tokens)
        self.cache = KvCache(pages, kv_heads, head_dim, page_tokens, format)
        self.capacity, self.indexed, self.held = capacity, 0, 0
        self.width = head_dim + 8                       # the coordinate that makes lengths equal, and zeros up to a multiple of 8
        self.indexes = None

    def _new(self, tokens):
        add = torch.full((1,), tokens, dtype=torch.int32, device="cuda")
        step = self.tables.extend(add, tokens, max_new=tokens)
        self.tables.commit(step)
        self.held += tokens
        return step

    def _points(self, slots):
        """Rows [kv_heads, tokens, width] for the indexes: the keys as they are held, on a sphere around the origin."""
        points = torch.zeros(self.kv_heads, slots.shape[0], self.width, device="cuda")
        self.cache.read(slots, out=(points[..., :self.dim].transpose(0, 1), None))
        lengths = points.square().sum(2)
        if self.indexes is None:
            # of later keys too; a longer one gets no coordinate, and is ranked as farther away than its inner product says
            self.radius = 1.2 * lengths.amax(1, keepdim=True)
        points[..., self.dim] = (self.radius - lengths).clamp(min=0.0).sqrt()
        return points

    def fill(self, k, v):
        """The context: written, read back and indexed."""
        step = self._new(k.shape[0])
        self.cache.append(k, v, step.slots)
        self.slots = step.slots
        points = self._points(step.slots)
        self.indexes = [PagIndex.build(points[h].contiguous(), metric="l2", max_degree=32, num_subspaces=self.width // 3, ef_construction=200,
                                       capacity=self.capacity) for h in range(self.kv_heads)]
        self.indexed = k.shape[0]

    def decode(self, q, k, v):
        """One token: q [1, heads, head_dim], k and v [1, kv_heads, head_dim] -> (out, lse) over what was found and the window, and the step."""
        step = self._new(1)
        self.cache.append(k, v, step.slots)
        self.slots = torch.cat([self.slots, step.slots])
        if self.held - self.indexed >= self.window:             # the oldest tokens of the window become searchable before they leave it
            end = self.indexed + self.block
            points = self._points(self.slots[self.indexed:end])
            for h, index in enumerate(self.indexes):
                index.insert(points[h].contiguous())
            self.indexed = end
        queries = torch.zeros(self.heads, self.width, device="cuda")
        queries[:, :self.dim] = q[0]
        group = self.heads // self.kv_heads
        found = [index.search(queries[h * group:(h + 1) * group], self.K, self.efS)[0] for h, index in enumerate(self.indexes)]
        self.ids = torch.cat(found).view(1, self.heads, self.K)
        return self.cache.attend_selected(q, self.ids, step, window=self.window), step


def run(tokens=20_000, steps=64, format="int8", seed=0):
    """-> (mean share of the softmax weight that was read, root mean square difference of the outputs from attention over everything)."""
    torch.manual_seed(seed)
    memory = SearchedMemory(tokens + steps + 64, format=format)
    kv, heads, dim = memory.kv_heads, memory.heads, memory.dim
    # keys spread unevenly over their numbers, as learned ones do: variances i^-0.8, which add up to those of `dim` standard normal numbers
    law = torch.arange(1, dim + 1, device="cuda", dtype=torch.float32) ** -0.4
    law *= (dim / law.square().sum()).sqrt()
    k = (torch.randn(tokens, kv, dim, device="cuda") * law).to(torch.bfloat16)
    v = torch.randn(tokens, kv, dim, device="cuda", dtype=torch.bfloat16)
    memory.fill(k, v)
    shares, errors = [], []
    for _ in range(steps):
        # each head asks for something that a few tokens of the context hold
        at = torch.randint(0, tokens, (heads, 3), device="cuda")
        wanted = k[at, torch.arange(heads, device="cuda")[:, None] // (heads // kv)].float().mean(1)
        q = (5.0 * wanted + 0.3 * torch.randn(heads, dim, device="cuda")).to(torch.bfloat16)[None]
        new = (torch.randn(1, kv, dim, device="cuda") * law).to(torch.bfloat16), torch.randn(1, kv, dim, device="cuda", dtype=torch.bfloat16)
        (out, lse), step = memory.decode(q, *new)
        full, full_lse = memory.cache.attend(q, step)
        shares.append(torch.exp(lse - full_lse))
        errors.append((out.float() - full.float()).square().mean())
    return float(torch.stack(shares).mean()), float(torch.stack(errors).mean().sqrt())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--tokens", type=int, default=20_000)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--format", default="int8", choices=("int8", "fp8"))
    a = p.parse_args()
    share, error = run(a.tokens, a.steps, a.format)
    print("read %.4f of the softmax weight, outputs differ from attention over all %d tokens by %.4f (root mean square)" % (share, a.tokens, error))
