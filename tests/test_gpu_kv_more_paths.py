"""The kernels that other tests of blocks and of the rotated write reach for one width, format or length only: every width and format of prompts' summaries, lists of any length for
any number of heads, long lists that several workgroups read, and queries turned in place whose halves begin anywhere."""
import math

import numpy as np
import pytest

import kv_more_plain as more
import test_gpu_kv_blocks as blocks_of
from test_gpu_kv import DTYPES, ints, kv, wide  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", ["int8", "fp8", "fp4"])
@pytest.mark.parametrize("dim", [8, 64, 128, 136, 192, 256])
@pytest.mark.parametrize("page, block", [(48, 16), (64, 64)])
def test_summaries_of_prompts(kv, fmt, dim, page, block):
    """More tokens than one workgroup each has blocks for; requests that end anywhere, slots that are none between them, numbers of any size, one block of them near the end of 32 bits.
    Blocks of no request stay as they were."""
    kv_heads, tokens, pages = 3, 2500, 2500 // 8
    rng = np.random.default_rng(dim + block)
    order, slots, first = rng.permutation(pages), [], 0
    while len(slots) < tokens:
        at = np.arange(int(rng.integers(1, 200)))
        slots += (order[first + at // page] * page + at % page).tolist() + [-1] * int(rng.integers(0, 2))
        first += -(-len(at) // page)
    slots = slots[:tokens]
    assert tokens * kv_heads > 4096
    gen = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randn(tokens, kv_heads, dim, device="cuda", generator=gen) * 2.0 ** torch.randint(-6, 7, (tokens, kv_heads, 1), device="cuda", generator=gen)
    x[100:130] *= 2.0 ** 117
    x[500:600, 0] = 0.0
    where = torch.tensor(slots).cuda()
    cache = kv.KvCache(pages, kv_heads, dim, page, fmt)
    cache.append(x, x, where)
    codes = torch.randint(-127, 128, (pages, kv_heads, page // block, 2, -(-dim // 64) * 64), dtype=torch.int8, device="cuda")
    exponents = torch.randint(-60, 60, (pages, kv_heads, page // block), dtype=torch.int8, device="cuda")
    before = codes.cpu().numpy().copy(), exponents.cpu().numpy().copy()
    blocks = kv.KvBlocks.from_tensors(cache, codes, exponents)
    blocks.update(where)
    keys = wide(cache.read(torch.arange(pages * page, device="cuda"))[0]).reshape(pages, page // block, block, kv_heads, dim)
    got, e_got = codes.cpu().numpy(), exponents.cpu().numpy()
    held = {}
    for s in slots:
        if s >= 0:
            held[s // block] = max(held.get(s // block, 0), s % block + 1)
    touched = np.zeros(e_got.shape, bool)
    for b, count in held.items():
        at = b // (page // block), b % (page // block)
        for h in range(kv_heads):
            want, e = more.summary(keys[at][:count, h])
            touched[at[0], h, at[1]] = True
            assert e_got[at[0], h, at[1]] == e and (got[at[0], h, at[1], :, :dim] == want).all(), (b, h)
            assert (got[at[0], h, at[1], :, dim:] == 0).all()
    assert (got[~touched] == before[0][~touched]).all() and (e_got[~touched] == before[1][~touched]).all() and not touched.all()


def lists_case(kv, n, width, heads, kv_heads, id_heads, dim, ks, few_codes=False):
    """Two tokens that may choose among all n blocks, and about half of them, of any summaries; a table with room for `width` blocks."""
    block = page = 16
    rng = np.random.default_rng(n + heads)
    cache = kv.KvCache(n + 1, kv_heads, dim, page)
    most = 2 if few_codes else 128
    codes = rng.integers(1 - most, most, (n + 1, kv_heads, 1, 2, -(-dim // 64) * 64)).astype(np.int8)
    codes[..., dim:] = 0
    exponents = rng.integers(0, 1 if few_codes else 3, (n + 1, kv_heads, 1)).astype(np.int8)
    blocks = kv.KvBlocks.from_tensors(cache, torch.tensor(codes).cuda(), torch.tensor(exponents).cuda())
    table = np.full((1, width), -1)
    table[0, :n] = rng.permutation(n + 1)[:n]
    if n > 3:
        table[0, [1, n // 2]] = n + 1, -7                    # pages that are none
    positions = [n * block - 1, max(n // 2 * block - 5, 0)]
    q = torch.randn(2, heads, dim, generator=torch.Generator().manual_seed(n)).half()
    if few_codes:
        q = q.sign()
    step = kv.KvStep(ints(table), requests=ints([0, 0]), positions=ints(positions))
    there = (table[0, :n] >= 0) & (table[0, :n] <= n)
    own = codes[np.where(there, table[0, :n], 0), :, 0].astype(np.float64)[..., :dim]               # [blocks, kv_heads, 2, dim]
    powers = 2.0 ** exponents[np.where(there, table[0, :n], 0), :, 0].astype(np.float64)
    scores = np.full((2, id_heads, n), -math.inf)
    for t in range(2):
        for h in range(heads):
            c, e = more.query_codes(wide(q[t, h]))
            g, i = h * kv_heads // heads, h * id_heads // heads
            s = (own[:, g, 0] @ np.maximum(c, 0) + own[:, g, 1] @ np.minimum(c, 0)) * powers[:, g] * 2.0 ** e
            scores[t, i] = np.maximum(scores[t, i], s)
    for k in ks:
        got = blocks.select(q.cuda(), step, k, id_heads=id_heads).cpu().numpy()
        for t in range(2):
            may = np.flatnonzero(there[:positions[t] // block + 1])
            for i in range(id_heads):
                best = np.sort(may[np.lexsort((may, -scores[t, i, may]))[:k]])
                want = np.concatenate([best, np.full(k - len(best), -1)])
                assert (got[t, i] == want).all(), (k, t, i)


@pytest.mark.parametrize("n, width", [(1, 1), (63, 64), (65, 65), (256, 256), (257, 300), (512, 1024), (1024, 1024), (1025, 1025), (900, 1100), (4096, 4096), (4097, 4097), (8192, 8192),
                                      (8193, 8193), (9000, 16_384), (16_384, 16_384), (16_385, 16_385), (40_000, 50_000)])
@pytest.mark.parametrize("heads, kv_heads, id_heads", [(4, 2, 4), (40, 1, 1), (8, 1, 8)])
@pytest.mark.parametrize("few_codes", [False, True])
def test_lists_of_any_length(kv, n, width, heads, kv_heads, id_heads, few_codes):
    lists_case(kv, n, width, heads, kv_heads, id_heads, 64, sorted({1, min(n, 7), 64, max(n // 2, 1), n + 3}), few_codes)


@pytest.mark.parametrize("dim", [8, 64, 128, 192, 256])
@pytest.mark.parametrize("heads, kv_heads, id_heads", [(40, 2, 2), (34, 1, 1), (36, 1, 2), (48, 1, 48), (64, 2, 8), (51, 1, 17), (16, 1, 1), (10, 1, 5)])
@pytest.mark.parametrize("n, width", [(300, 300), (300, 1500), (1500, 1500), (2500, 9000)])
def test_lists_of_any_number_of_heads(kv, dim, heads, kv_heads, id_heads, n, width):
    """One tile of columns and several, of whole lists and of a list's heads, for every width of a row; in one workgroup and in parts."""
    lists_case(kv, n, width, heads, kv_heads, id_heads, dim, [5, 100])


class Written:
    """Memory of test_gpu_kv, filled by the cache's own write (which has tests of its own) so that long contexts are quick."""

    def __init__(self, kv, contexts, kv_heads, dim, page, fmt, seed):
        rng = np.random.default_rng(seed)
        counts = [-(-c // page) for c in contexts]
        self.pages = sum(counts) + 2
        order = rng.permutation(self.pages)
        self.table = np.full((len(contexts), max(counts + [1]) + 1), -1)
        self.page, self.fmt, self.dim, self.kv_heads, self.contexts = page, fmt, dim, kv_heads, contexts
        data_shape, exponent_shape = more.shapes(self.pages, kv_heads, page, dim, fmt)
        data = torch.full(data_shape, 0x7F, dtype=torch.uint8, device="cuda")
        data[..., dim // 2 if fmt == "fp4" else dim:] = 0
        self.cache = kv.KvCache.from_tensors(data, torch.full(exponent_shape, 127, dtype=torch.int8, device="cuda"), dim, fmt)
        slots, first = [], 0
        for b, (c, n) in enumerate(zip(contexts, counts)):
            self.table[b, :n] = order[first:first + n]
            first += n
            at = np.arange(c)
            slots.append(self.table[b, at // page] * page + at % page)
        slots = torch.tensor(np.concatenate(slots)).cuda()
        x = torch.randn(2, len(slots), kv_heads, dim, generator=torch.Generator().manual_seed(seed)) * 2.0 ** torch.tensor(rng.integers(-1, 2, (2, len(slots), kv_heads, 1)))
        x[0, ..., ::16] *= 3
        self.cache.append(x[0].float().cuda(), x[1].float().cuda(), slots)
        if fmt != "fp4":
            for b, (c, n) in enumerate(zip(contexts, counts)):
                if c % 16:
                    data[self.table[b, n - 1], :, c % page:, :, :dim] = 0x7F
        k, v = (wide(y).reshape(self.pages, page, kv_heads, dim) for y in self.cache.read(torch.arange(self.pages * page, device="cuda")))
        self.numbers = np.stack([k, v], 3).transpose(0, 2, 1, 3, 4)

    def rows(self, b, at, head):
        p, t = self.table[b, at // self.page], at % self.page
        return self.numbers[p, head, t, 0], self.numbers[p, head, t, 1]


@pytest.mark.parametrize("fmt", ["int8", "fp8", "fp4"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("tokens, heads, id_heads, k, window, softcap, slopes", [
    (3, 4, 4, 40, 300, 0.0, False), (2, 6, 2, 70, 0, 30.0, False), (3, 20, 1, 60, 100, 300.0, True), (1, 1, 1, 100, 4000, 0.0, True), (70, 4, 4, 40, 64, 100.0, False)])
def test_blocks_of_long_lists(kv, monkeypatch, fmt, dim, tokens, heads, id_heads, k, window, softcap, slopes):
    """Lists that several workgroups share, and lists that one reads, of every width and format, without a cap, with a small one and with a large one."""
    monkeypatch.setattr(blocks_of, "Memory", Written)
    blocks_of.blocks_case(kv, [5000 - 7 * i for i in range(min(tokens, 3))], heads, 1, id_heads, dim, 64, 64, k, window, fmt, "fp16" if dim % 128 else "bf16", softcap=softcap,
                          slopes=slopes, news=[-(-tokens // min(tokens, 3))] * min(tokens, 3))


def turned_within_its_roundings(got, q, positions, f, pairs, dtype):
    """x cos a - y sin a in 32 bits.  The cosine and the sine are rounded, and one of the products: |x cos a| + 2 |y sin a| times 2^-24, which is at most sqrt(5) * 2^-24 of the
    pair's length (sqrt(1 + 4) by Cauchy and Schwarz, since cos^2 + sin^2 = 1); they were off by 2^-50 before.  Then the sum is rounded to 32 bits, half a step, 2^-24 of it, and from there to a
    16-bit type: 2^-8 of it for bf16 (8 bits), 2^-11 for fp16 (11 bits) and half its least step, 2^-25."""
    want = more.turn(q, positions, f, pairs)
    n = 2 * len(f)
    size = np.zeros_like(q)
    first, second = (slice(0, n // 2), slice(n // 2, n)) if pairs == "halves" else (slice(0, n, 2), slice(1, n, 2))
    size[..., first] = size[..., second] = np.hypot(q[..., first], q[..., second])
    tol = (math.sqrt(5) * 2.0 ** -24 * (1 + 2.0 ** -20) + 2.0 ** -48) * size
    tol = tol + 2.0 ** -24 * (np.abs(want) + tol)
    if dtype != "fp32":
        tol = tol + {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype] * (np.abs(want) + tol) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    got = wide(got)
    assert (np.abs(got - want)[..., :n] <= tol[..., :n]).all() and (got[..., n:] == q[..., n:]).all()


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("dim, turned, dtype, pairs", [(72, 72, "fp16", "halves"), (96, 24, "bf16", "halves"), (80, 40, "fp32", "halves"), (128, 128, "fp32", "halves"), (8, 8, "bf16", "halves"),
                                                       (256, 248, "fp16", "halves"), (64, 64, "bf16", "neighbours"), (200, 72, "fp32", "neighbours"), (128, 128, "fp16", "halves")])
@pytest.mark.parametrize("tokens, heads", [(1, 1), (5, 7), (1500, 3)])
def test_queries_turned_in_place(kv, fmt, dim, turned, dtype, pairs, tokens, heads):
    """The same numbers as in a tensor of their own, in dense rows and in rows among others, which stay as they were."""
    rng = np.random.default_rng(dim + tokens)
    f = (10000.0 ** (-np.arange(turned // 2) / (turned // 2))).astype(np.float32)
    rotation = kv.KvRotation(torch.tensor(f).cuda(), pairs)
    cache = kv.KvCache(tokens // 16 + 1, 1, dim, 16, fmt)
    k, slots = torch.zeros(tokens, 1, dim, device="cuda", dtype=DTYPES[dtype]), torch.arange(tokens, device="cuda")
    positions = rng.integers(-1000, 1_000_000, tokens)
    at = torch.tensor(positions, dtype=torch.int32).cuda()
    q = torch.tensor(rng.standard_normal((tokens, heads, dim)) * 2.0 ** rng.integers(-8, 9, (tokens, heads, 1))).to(DTYPES[dtype]).cuda()
    apart = cache.append_rotated(k, k, slots, at, rotation, q=q)
    turned_within_its_roundings(apart, wide(q), positions, f, pairs, dtype)
    among = torch.full((tokens, 2 * heads + 1, dim + 8), 3.0, device="cuda", dtype=DTYPES[dtype])
    rows = among[:, 1::2, :dim]
    for own in (q.clone(), rows):
        own.copy_(q)
        assert cache.append_rotated(k, k, slots, at, rotation, q=own, out=own) is own and torch.equal(own, apart)
    rows.fill_(3.0)
    assert bool((among == 3.0).all())


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("dim, heads, kv_heads, contexts, news", [
    (128, 8, 2, [700], [1]), (128, 32, 8, [3000, 40, 9000], [1, 1, 1]), (128, 8, 2, [40_000], [1]), (128, 8, 2, [1500, 700], [1500, 700]), (192, 4, 1, [5000, 300], [10, 4]),
    (64, 40, 2, [5000, 900], [1, 1]), (256, 4, 1, [2500], [100]), (64, 4, 1, [900, 2000], [70, 900])])
def test_the_same_bits_every_time(kv, fmt, dim, heads, kv_heads, contexts, news):
    """Attention over everything, over listed tokens and over blocks, in shares and in one workgroup, by the kernels for few rows and for many: runs of one call are equal bit for bit, also
    beside each other on several streams."""
    m = Written(kv, contexts, kv_heads, dim, 64, fmt, 5)
    positions = [p for c, a in zip(contexts, news) for p in range(c - a, c)]
    requests = [b for b, a in enumerate(news) for _ in range(a)]
    n = len(positions)
    gen = torch.Generator(device="cuda").manual_seed(dim)
    q = torch.randn(n, heads, dim, device="cuda", generator=gen).half()
    step = kv.KvStep(ints(m.table), ints(np.concatenate([[0], np.cumsum(news)])), ints(contexts), ints(requests), ints(positions), max_new=max(news))
    few = kv.KvStep(ints(m.table), requests=ints(requests[-4:]), positions=ints(positions[-4:]))
    ids = torch.randint(0, min(contexts), (min(n, 4), kv_heads, 2200), device="cuda", generator=gen)
    chosen = torch.randint(0, min(contexts) // 64 + 1, (min(n, 4), kv_heads, 50), device="cuda", generator=gen).int()
    blocks = kv.KvBlocks(m.cache, 64)

    def one():
        return (*m.cache.attend(q, step, softcap=30.0), *m.cache.attend(q, step), *m.cache.attend_selected(q[-4:], ids, few, window=64), *blocks.attend(q[-4:], chosen, few, window=64))

    first, results = one(), []
    torch.cuda.synchronize()
    for s in [torch.cuda.Stream() for _ in range(3)] * 3:
        with torch.cuda.stream(s):
            results.append(one())
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(r, first))
