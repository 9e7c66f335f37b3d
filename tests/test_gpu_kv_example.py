"""The example that writes, indexes, searches and attends: what it reads through searches is nearly all of the softmax weight."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("format", ["int8", "fp8"])
def test_searched_memory(format):
    """Each head's query is 4/3 of the sum of three keys of 64 independent standard normal numbers: over sqrt(64) these three score about
    4/3 * 64 / 8 = 10.7 each, the 6,000 others N(0, 4/3 * sqrt(3)), in all some 6,000 e^2.7 = e^11.4.  What is read has to be what was found and the
    window, to the rounding of scores (64 products, 2^-24 each of some 100, and a few roundings after that: below 1e-3 of a logarithm);
    how much of the weight an approximate search finds on data without any structure is a matter of its effort: on average it has to be
    nine tenths of what the best 64 keys of all hold."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("searched_memory", os.path.join(ROOT, "examples", "searched_memory.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    memory = example.SearchedMemory(6000 + 400, format=format)
    torch.manual_seed(1)
    kv, heads, dim = memory.kv_heads, memory.heads, memory.dim
    k, v = (torch.randn(6000, kv, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    memory.fill(k, v)
    shares = []
    for step_number in range(300):
        q = torch.randn(1, heads, dim, device="cuda", dtype=torch.bfloat16)
        at = None
        if step_number % 30 == 0:
            at = torch.randint(0, 6000, (heads, 3), device="cuda")
            q = (4.0 * k[at, torch.arange(heads, device="cuda")[:, None] // (heads // kv)].float().mean(1)).to(torch.bfloat16)[None]
        new = [torch.randn(1, kv, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        (out, lse), step = memory.decode(q, *new)
        if at is None:
            continue
        # against the same weights from scratch, over the numbers that the cache holds
        keys, values = memory.cache.read(memory.slots)
        full, full_lse = memory.cache.attend(q, step)
        for h in range(0, heads, 5):
            scores = (keys[:, h * kv // heads].double() @ q[0, h].double()) / dim ** 0.5
            assert abs(float(torch.logsumexp(scores, 0)) - float(full_lse[0, h])) < 1e-3
            n = scores.numel()
            near = torch.arange(n, device="cuda") >= n - memory.window
            found = near.clone()
            ids = memory.ids[0, h]
            found[ids[(ids >= 0) & (ids < n - memory.window)]] = True
            assert ids.unique().numel() == memory.K
            assert abs(float(torch.logsumexp(scores[found], 0)) - float(lse[0, h])) < 1e-3
            best = near.clone()
            best[torch.topk(scores, memory.K).indices] = True
            shares.append(float(torch.exp(torch.logsumexp(scores[found], 0) - torch.logsumexp(scores[best], 0))))
    assert len(shares) == 40 and sum(shares) / 40 >= 0.9, shares
    assert memory.indexed >= 6000 + 64 and memory.indexes[0].describe()["n"] == memory.indexed
    assert memory.tables.lengths.tolist() == [6300] and memory.held == 6300
