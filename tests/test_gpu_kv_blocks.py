"""Summaries of blocks, the choice among them and attention over the chosen ones, against a plain implementation in 64 bits: summaries and choices
are equal, since they are integers times powers of two; attention to the tolerances of attention over listed tokens."""
import math

import numpy as np
import pytest

import kv_more_plain as more
from test_gpu_kv import DTYPES, check_attention, ints, kv, wide  # noqa: F401
from test_gpu_kv_fp4 import Memory

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def summaries(m, block):
    """Of every block of every request: {(request, block, head): (codes, exponent)}."""
    out = {}
    for b, c in enumerate(m.contexts):
        for j in range(-(-c // block)):
            for h in range(m.kv_heads):
                out[b, j, h] = more.summary(m.rows(b, np.arange(j * block, min(c, (j + 1) * block)), h)[0])
    return out


def filled(kv, m, block):
    """KvBlocks over memory that held anything, with all blocks of the requests summarised."""
    per = m.page // block
    codes = torch.randint(-127, 128, (m.pages, m.kv_heads, per, 2, -(-m.dim // 64) * 64), dtype=torch.int8)
    codes[..., m.dim:] = 0
    blocks = kv.KvBlocks.from_tensors(m.cache, codes.cuda(), torch.randint(-3, 3, (m.pages, m.kv_heads, per), dtype=torch.int8).cuda())
    slots = [int(m.table[b, p // m.page]) * m.page + p % m.page for b, c in enumerate(m.contexts) for p in range(c)]
    blocks.update(torch.tensor(slots, dtype=torch.int64).cuda())
    return blocks, codes


@pytest.mark.parametrize("fmt", ["int8", "fp8", "fp4"])
@pytest.mark.parametrize("dim, kv_heads, page, block", [(64, 1, 16, 16), (128, 3, 64, 32), (80, 2, 96, 96), (192, 2, 32, 16), (256, 1, 128, 128), (8, 5, 64, 64)])
def test_update(kv, fmt, dim, kv_heads, page, block):
    """Blocks that end anywhere; the ones of no request stay as they were."""
    m = Memory(kv, [1, 15, 16, 17, 40, 130, 257], kv_heads, dim, page, fmt, dim)
    blocks, before = filled(kv, m, block)
    codes, exponents = blocks.codes.cpu().numpy(), blocks.exponents.cpu().numpy()
    assert blocks.block_tokens == block
    touched = np.zeros(codes.shape[:3], bool)
    for (b, j, h), (want, e) in summaries(m, block).items():
        page_of, place = m.table[b, j * block // page], j * block % page // block
        touched[page_of, h, place] = True
        assert exponents[page_of, h, place] == e and (codes[page_of, h, place, :, :dim] == want).all(), (b, j, h)
        assert (codes[page_of, h, place, :, dim:] == 0).all()
    assert (codes[~touched] == before.numpy()[~touched]).all() and not touched.all()


def test_update_token_by_token(kv):
    """Steps of one token and of some, with slots that are none: after each the blocks' summaries are those of what they hold."""
    kv_heads, dim, page, block = 2, 64, 64, 32
    m = Memory(kv, [0, 0], kv_heads, dim, page, "int8", 1)
    cache, one, all_ = kv.KvCache(4, kv_heads, dim, page), None, None
    one, all_ = kv.KvBlocks(cache, block), kv.KvBlocks(cache, block)
    order, length = [2, 0, 3], 0
    for n in (1, 1, 30, 1, 31, 1, 40, 3):
        at = np.arange(length, length + n)
        slots = torch.tensor([order[p // page] * page + p % page for p in at] + [-1, 1 << 40]).cuda()
        x = torch.randn(n + 2, kv_heads, dim, device="cuda")
        cache.append(x, x, slots)
        one.update(slots)
        length += n
        all_.codes.zero_()
        all_.exponents.zero_()
        all_.update(torch.tensor([order[p // page] * page + p % page for p in range(length)]).cuda())
        assert torch.equal(one.codes, all_.codes) and torch.equal(one.exponents, all_.exponents)
    assert m.pages == 2 and int((one.codes != 0).any(-1).any(-1).sum()) == kv_heads * -(-length // block)


def test_update_of_prompts(kv):
    """Waves that look at many tokens."""
    kv_heads, dim, page, block, tokens = 8, 16, 32, 16, 3000
    cache = kv.KvCache(tokens // 8, kv_heads, dim, page, "fp8")
    rng = np.random.default_rng(4)
    order, slots, first = rng.permutation(tokens // 8), [], 0
    while len(slots) < tokens:
        n = int(rng.integers(1, 100))
        at = np.arange(n)
        slots += (order[first + at // page] * page + at % page).tolist() + [-1] * int(rng.integers(0, 2))
        first += -(-n // page)
    slots = slots[:tokens]
    x = torch.randn(tokens, kv_heads, dim, device="cuda")
    where = torch.tensor(slots).cuda()
    cache.append(x, x, where)
    blocks = kv.KvBlocks(cache, block)
    blocks.update(where)
    keys = wide(cache.read(torch.arange(cache.num_pages * page, device="cuda"))[0]).reshape(cache.num_pages, page // block, block, kv_heads, dim)
    codes, exponents = blocks.codes.cpu().numpy(), blocks.exponents.cpu().numpy()
    held = {}
    for s in slots:
        if s >= 0:
            held[s // block] = max(held.get(s // block, 0), s % block + 1)
    for b, count in held.items():
        for h in range(kv_heads):
            want, e = more.summary(keys[b // 2, b % 2, :count, h])
            assert exponents[b // 2, h, b % 2] == e and (codes[b // 2, h, b % 2, :, :dim] == want).all()


def choice(m, table, block, q, requests, positions, window, k, id_heads):
    """The lists of every token in 64 bits."""
    held = summaries(m, block)
    q = wide(q)
    tokens, heads = q.shape[:2]
    out = np.full((tokens, id_heads, k), -1)
    for t in range(tokens):
        b, p = requests[t], positions[t]
        if b < 0 or b >= len(m.contexts) or p < window:
            continue
        each = {}
        for h in range(heads):
            codes, e = more.query_codes(q[t, h])
            g = h * m.kv_heads // heads
            for j in range((p - window) // block + 1):
                if 0 <= table[b, j * block // m.page] < m.pages:
                    s, es = held[b, j, g]
                    score = float((s[0] * np.maximum(codes, 0) + s[1] * np.minimum(codes, 0)).sum()) * 2.0 ** (e + es)
                    i = h * id_heads // heads
                    each[i, j] = max(each.get((i, j), -math.inf), score)
        for i in range(id_heads):
            out[t, i] = more.select([(j, s) for (x, j), s in each.items() if x == i], k)
    return out


def select_case(kv, contexts, heads, kv_heads, id_heads, dim, page, block, k, window, fmt, dtype, seed=3, pad=1, news=None, edges=False, wide_table=0):
    m = Memory(kv, contexts, kv_heads, dim, page, fmt, seed)
    blocks, _ = filled(kv, m, block)
    news = [min(1, c) for c in contexts] if news is None else news
    requests = [b for b, a in enumerate(news) for _ in range(a)] + [-1] * pad
    positions = [p for c, a in zip(contexts, news) for p in range(c - a, c)] + [-1] * pad
    tokens = len(positions)
    q = torch.randn(tokens, heads, dim, generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype])
    table = m.table
    if wide_table:
        table = np.concatenate([table, np.full((len(contexts), wide_table), -1)], 1)
    if edges:
        q[0, 0] = 0.0                                       # all blocks are equal: the first ones
        q[1, heads - 1, 3], q[1, 0, 0], q[2, 0, 5] = math.nan, math.inf, -math.inf
        table = table.copy()
        table[3, 1] = m.pages
    step = kv.KvStep(ints(table), requests=ints(requests), positions=ints(positions))
    out = torch.full((tokens, id_heads, k + 3), 77, dtype=torch.int32, device="cuda")
    got = blocks.select(q.cuda(), step, k, window=window, id_heads=id_heads, out=out[..., :k])
    want = choice(m, table, block, q, requests, positions, window, k, id_heads)
    assert (got.cpu().numpy() == want).all()
    assert (out[..., k:] == 77).all()
    if kv_heads == id_heads:
        assert torch.equal(blocks.select(q.cuda(), step, k, window=window), got)
    return m, blocks, step, q, got


@pytest.mark.parametrize("fmt, dtype", [("int8", "bf16"), ("fp4", "fp16")])
@pytest.mark.parametrize("dim, page, block", [(64, 32, 16), (128, 64, 64), (80, 96, 48), (192, 16, 16), (256, 64, 32)])
@pytest.mark.parametrize("k, window", [(1, 0), (3, 1), (7, 40), (40, 16)])
def test_select(kv, fmt, dtype, dim, page, block, k, window):
    select_case(kv, [300, 1, 40, 650, 64, 17, 0], 4, 2, 2, dim, page, block, k, window, fmt, dtype)


@pytest.mark.parametrize("heads, kv_heads, id_heads", [(1, 1, 1), (8, 2, 8), (8, 2, 4), (6, 2, 2), (12, 1, 4), (40, 2, 2), (36, 1, 2), (48, 1, 48), (5, 5, 5), (34, 1, 1)])
def test_select_heads(kv, heads, kv_heads, id_heads):
    select_case(kv, [500, 90, 813, 333, 250], heads, kv_heads, id_heads, 64, 32, 16, 9, 20, "int8", "fp16", pad=2, edges=True)


@pytest.mark.parametrize("wide_table", [0, 700, 9000])
@pytest.mark.parametrize("k", [5, 64, 600])
def test_select_by_every_path(kv, wide_table, k):
    """Tables for more blocks than one workgroup's, than LDS has keys for; the same choice."""
    select_case(kv, [9000, 3000, 33, 1600], 4, 2, 4, 64, 32, 16, k, 100, "int8", "bf16", wide_table=wide_table, edges=True)


@pytest.mark.parametrize("contexts", [[900, 20, 33], [1500, 700, 33], [2500, 1000, 16], [3900, 2000, 17]])
@pytest.mark.parametrize("heads, id_heads, k", [(4, 2, 20), (8, 8, 70)])
def test_select_by_any_number_of_waves(kv, contexts, heads, id_heads, k):
    select_case(kv, contexts, heads, 2, id_heads, 64, 32, 16, k, 30, "int8", "bf16", news=[3, 2, 1], edges=False)


@pytest.mark.parametrize("context, heads, id_heads, k", [(3300, 4, 2, 30), (3300, 8, 8, 3), (12_000, 4, 2, 200), (12_000, 4, 4, 900)])
def test_select_for_many_tokens(kv, context, heads, id_heads, k):
    """More workgroups than run at once: the lists of the same tokens a few at a time."""
    m = Memory(kv, [context, 700], 2, 64, 64, "int8", 9)
    blocks, _ = filled(kv, m, 16)
    n = 640
    rng = np.random.default_rng(k)
    requests = rng.integers(0, 2, n)
    positions = np.where(requests == 0, rng.integers(-1, context, n), rng.integers(-1, 700, n))
    q = torch.randn(n, heads, 64, device="cuda", dtype=torch.bfloat16)

    def lists(a, b):
        return blocks.select(q[a:b], kv.KvStep(ints(m.table), requests=ints(requests[a:b]), positions=ints(positions[a:b])), k, window=20, id_heads=id_heads)

    assert torch.equal(lists(0, n), torch.cat([lists(a, a + 20) for a in range(0, n, 20)]))


@pytest.mark.parametrize("dim, heads, wide_table", [(256, 15, 900), (256, 14, 900), (64, 16, 800), (192, 14, 990)])
def test_select_of_as_many_lists_as_fit(kv, dim, heads, wide_table):
    """Keys of all lists of a head that just fit LDS, or just do not."""
    select_case(kv, [1500, 333], heads, 1, heads, dim, 16, 16, 7, 5, "fp4", "fp16", wide_table=wide_table)


def test_pages_that_do_not_exist(kv):
    """Page numbers out of range count as absent, in lists and in the window; requests and positions out of range read nothing."""
    m = Memory(kv, [128, 40, 40], 1, 64, 32, "int8", 4)
    table = m.table.copy()
    table[0, 1], table[0, 3] = m.pages, -5
    step = kv.KvStep(ints(table), requests=ints([0, 7, 2, -3]), positions=ints([127, 39, 2_000_000_000, 5]))
    q = torch.randn(4, 2, 64).to(torch.bfloat16)
    blocks = kv.KvBlocks(m.cache, 32)
    out, lse = blocks.attend(q.cuda(), ints(np.tile(np.arange(-1, 5), (4, 1, 1))), step, window=10)
    keys = lambda t, h: np.concatenate([np.arange(32), np.arange(64, 96)])
    check_attention(m, q, out, lse, "bf16", [0, 0, 0, 0], [127, -1, -1, -1], keys, 64 ** -0.5)
    assert (blocks.select(q.cuda(), step, 4)[1:] == -1).all() and blocks.select(q.cuda(), step, 4)[0, 0].tolist() == [0, 2, -1, -1]


def test_select_of_many_equal_scores(kv):
    """Keys that repeat from block to block: the first blocks of those that are equal."""
    dim, page = 64, 64
    cache = kv.KvCache(40, 1, dim, page)
    blocks = kv.KvBlocks(cache, 16)
    x = torch.randn(16 * 3, 1, dim, generator=torch.Generator().manual_seed(2)).repeat(53, 1, 1)[:2500].cuda()
    slots = torch.arange(2500, device="cuda")
    cache.append(x, x, slots)
    blocks.update(slots)
    q = torch.randn(3, 2, dim, generator=torch.Generator().manual_seed(5)).half()
    keys = wide(cache.read(slots)[0])[:, 0]
    for width in (40, 2000):
        table = np.concatenate([np.arange(40), np.full(width - 40, -1)])[None]
        step = kv.KvStep(ints(table), requests=ints([0] * 3), positions=ints([2499, 2400, 100]))
        for k in (1, 20, 53, 80, 160):
            got = blocks.select(q.cuda(), step, k, id_heads=1).cpu().numpy()
            for t, p in enumerate((2499, 2400, 100)):
                scores = []
                for j in range(p // 16 + 1):
                    s, es = more.summary(keys[j * 16:j * 16 + 16])
                    each = []
                    for h in range(2):
                        codes, e = more.query_codes(wide(q[t, h]))
                        each.append(float((s[0] * np.maximum(codes, 0) + s[1] * np.minimum(codes, 0)).sum()) * 2.0 ** (e + es))
                    scores.append((j, max(each)))
                assert got[t, 0].tolist() == more.select(scores, k), (width, k, t)


def blocks_case(kv, contexts, heads, kv_heads, id_heads, dim, page, block, k, window, fmt, dtype, softcap=0.0, slopes=False, seed=2, pad=1, news=None):
    m = Memory(kv, contexts, kv_heads, dim, page, fmt, seed)
    rng = np.random.default_rng(seed)
    news = [min(1, c) for c in contexts] if news is None else news
    requests = [b for b, a in enumerate(news) for _ in range(a)] + [-1] * pad
    positions = [p for c, a in zip(contexts, news) for p in range(c - a, c)] + [-1] * pad
    tokens = len(positions)
    q = torch.tensor(rng.standard_normal((tokens, heads, dim))).to(DTYPES[dtype])
    slope = np.exp2(-8.0 * (1 + np.arange(heads)) / heads).astype(np.float32) if slopes else None
    # blocks of the request in any order and of none: -1, beyond the token, far beyond, listed twice, in the window
    ids = np.full((tokens, id_heads, k), -1, np.int32)
    for t in range(tokens):
        for i in range(id_heads):
            row = rng.integers(-1, max(positions[t], 0) // block + 3, k)
            row[rng.random(k) < 0.1] = -1
            row[rng.random(k) < 0.03] = 2 ** 31 - 1
            row[rng.random(k) < 0.03] = 2 ** 28 + 1
            if t % 5 == 4:
                row[:] = -1
            ids[t, i] = row
    step = kv.KvStep(ints(m.table), requests=ints(requests), positions=ints(positions))
    blocks = kv.KvBlocks(m.cache, block)
    out, lse = blocks.attend(q.cuda(), torch.tensor(ids).cuda(), step, window=window, softcap=softcap, slopes=None if slope is None else torch.tensor(slope).cuda())

    def keys_of(t, h):
        p, row = positions[t], ids[t, h * id_heads // heads].astype(np.int64)
        at = (row[row >= 0][:, None] * block + np.arange(block)).ravel()
        return np.concatenate([at[at <= p - window], np.arange(max(0, p - window + 1), p + 1)]).astype(int)

    check_attention(m, q, out, lse, dtype, requests, positions, keys_of, dim ** -0.5, softcap, slope)


@pytest.mark.parametrize("fmt, dtype", [("int8", "bf16"), ("fp8", "fp16"), ("fp4", "bf16")])
@pytest.mark.parametrize("dim, page, block", [(64, 32, 16), (128, 64, 64), (80, 96, 48), (192, 16, 16), (256, 64, 32)])
@pytest.mark.parametrize("k, window", [(1, 0), (2, 1), (5, 40), (12, 16)])
def test_attend_blocks(kv, fmt, dtype, dim, page, block, k, window):
    blocks_case(kv, [300, 1, 40, 650, 64, 17, 0], 4, 2, 2, dim, page, block, k, window, fmt, dtype)


@pytest.mark.parametrize("heads, kv_heads, id_heads", [(1, 1, 1), (8, 2, 8), (8, 2, 4), (40, 2, 2), (48, 1, 2), (12, 4, 12)])
@pytest.mark.parametrize("fmt, softcap, slopes", [("int8", 30.0, False), ("fp4", 0.0, True), ("fp8", 300.0, True)])
def test_attend_blocks_heads_cap_and_distance(kv, heads, kv_heads, id_heads, fmt, softcap, slopes):
    blocks_case(kv, [200, 90, 513, 33, 50], heads, kv_heads, id_heads, 64, 64, 32, 6, 20, fmt, "fp16", softcap=softcap, slopes=slopes, pad=2, news=[1, 3, 2, 1, 4])


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("tokens, k, window, slopes", [(1, 40, 0, False), (3, 40, 300, True), (5, 64, 100, False), (30, 48, 64, False)])
def test_attend_blocks_of_long_lists(kv, fmt, tokens, k, window, slopes):
    """Lists that one workgroup reads, and lists that several share."""
    blocks_case(kv, [5000 - 7 * i for i in range(tokens)], 16, 1, 16, 64, 64, 64, k, window, fmt, "fp16", slopes=slopes)


def test_attend_blocks_nothing_at_all(kv):
    blocks_case(kv, [200, 90], 4, 2, 2, 64, 32, 32, 0, 0, "int8", "fp16")
    blocks_case(kv, [200, 90], 4, 2, 4, 64, 32, 32, 0, 7, "fp4", "fp16")


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_attend_blocks_far_away_with_slopes(kv, fmt):
    """Blocks that are all 300,000 tokens away, slope 1: their weights are those of the distances from each other."""
    dim, page, position = 64, 64, 300_000
    m = Memory(kv, [256], 1, dim, page, fmt, 7)
    table = np.full((1, position // page + 1), -1)
    table[0, :4] = m.table[0, :4]
    q = torch.randn(1, 2, dim, generator=torch.Generator().manual_seed(7)).half()
    step = kv.KvStep(ints(table), requests=ints([0]), positions=ints([position]))
    ids = ints([[[3, 0, 1]]])
    out, lse = kv.KvBlocks(m.cache, 64).attend(q.cuda(), ids, step, slopes=torch.ones(2, device="cuda"))
    at = np.concatenate([np.arange(192, 256), np.arange(128)])
    for h in range(2):
        k, v = m.rows(0, at, 0)
        o, l, spread, products = plain_row(wide(q[0, h]), k, v, dim, position - at)
        from kv_plain import tolerance
        tol_o, _ = tolerance(dim, 11, o, spread, products, 0.0, 256.0)
        # lse holds a number of 300,000 to half a step
        assert abs(float(lse[0, h]) - l) <= 2.0 ** -6 * 1.5 and (np.abs(wide(out[0, h]) - o) <= tol_o).all()


def plain_row(q, k, v, dim, distance):
    import kv_plain as plain
    return plain.attend_row(q, k, v, dim ** -0.5, slope=1.0, distance=distance)


@pytest.mark.parametrize("fmt", ["int8", "fp8", "fp4"])
def test_choosing_every_block_is_attention(kv, fmt):
    """With room for all blocks what is chosen and read is everything."""
    m, blocks, step, q, ids = select_case(kv, [700, 50, 333], 8, 2, 2, 128, 64, 32, 30, 0, fmt, "fp16")
    out, lse = blocks.attend(q.cuda(), ids, step)
    positions = [699, 49, 332, -1]
    check_attention(m, q, out, lse, "fp16", [0, 1, 2, -1], positions, lambda t, h: np.arange(positions[t] + 1), 128 ** -0.5)


def test_the_best_blocks_hold_what_a_query_looks_for(kv):
    """Keys of a block are one vector of 64 signs, to a twentieth, which 4 bits hold as +-1: a query along a key scores 2 * 64 * 0.95 or more with its own block and, with a block of
    which a signs are alike, 2 * 1.05 a - 2 * 0.95 (64 - a) at most, which is less for a < 61; 61 of 64 random signs are alike once in 10^14.
    Its own 64 keys score 15 and more over sqrt(64), the 20,000 others 2 (2 a - 64) / 8, N(0, 2): 64 e^15 against 20,000 e^2."""
    torch.manual_seed(1)
    n, heads, dim, page = 20_000, 4, 64, 64
    tables, cache = kv.KvTables(1, 400, 400, page), kv.KvCache(400, heads, dim, page, "fp4")
    blocks = kv.KvBlocks(cache)
    step = tables.extend(ints([n]), n)
    signs = torch.randint(0, 2, (n // page + 1, heads, dim), device="cuda").float() * 2 - 1
    k = (signs.repeat_interleave(page, 0)[:n] * (0.95 + 0.1 * torch.rand(n, heads, dim, device="cuda"))).to(torch.bfloat16)
    v = torch.randn(n, heads, dim, device="cuda", dtype=torch.bfloat16)
    cache.append(k, v, step.slots)
    blocks.update(step.slots)
    q = 2.0 * k[7777:7778]
    last = kv.KvStep(step.table, ints([0, 1]), step.context, ints([0]), ints([n - 1]))
    ids = blocks.select(q, last, 8, window=64)
    assert (ids == 7777 // 64).any(-1).all()
    out, lse = blocks.attend(q, ids, last, window=64)
    full, full_lse = cache.attend(q, last)
    assert (torch.exp(lse - full_lse) > 0.99).all()


# ---- a decoding loop ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("max_pages", [6, 400])
def test_captured_step(kv, fmt, max_pages):
    """extend, the rotated write, summaries, the choice and attention in a graph: every replay against the same step without one."""
    heads, kv_heads, dim, page = 8, 2, 64, 32
    torch.manual_seed(3)
    state = []
    for _ in range(2):
        tables, cache = kv.KvTables(5, max_pages, 40, page), kv.KvCache(40, kv_heads, dim, page, fmt)
        state.append((tables, cache, kv.KvBlocks(cache, 16), kv.KvStep.empty(5, 8)))
    rotation = kv.KvRotation(torch.rand(16, device="cuda"))
    add = torch.zeros(5, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(8, kv_heads, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q = torch.zeros(8, heads, dim, device="cuda", dtype=torch.bfloat16)

    def one(tables, cache, blocks, step):
        tables.extend(add, 8, max_new=8, out=step, commit=True)
        turned = cache.append_rotated(k, v, step.slots, step.positions, rotation, q=q)
        blocks.update(step.slots)
        ids = blocks.select(turned, step, 2, window=10)
        return (turned, ids, *blocks.attend(turned, ids, step, window=10), *cache.attend(turned, step))

    one(*state[0])                       # loads the kernels; nothing was added
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = one(*state[0])
    for i in range(12):
        add.copy_(torch.tensor([[1, 1, 1, 1, 1], [3, 0, 1, 4, 0], [0, 0, 8, 0, 0], [1, 2, 0, 0, 5]][i % 4], dtype=torch.int32))
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = one(*state[1])
        torch.cuda.synchronize()
        for got, w in zip(captured, want):
            assert torch.equal(got, w), i
        for a, b in zip(state[0][:3], state[1][:3]):
            for name in ("table", "lengths", "free_count", "data", "exponents", "codes"):
                if hasattr(a, name):
                    assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)


def test_the_same_every_time_and_on_any_stream(kv):
    m = Memory(kv, [3000, 100, 2222], 4, 128, 64, "fp4", 6)
    blocks, _ = filled(kv, m, 32)
    q = torch.randn(3, 16, 128, device="cuda").half()
    for width in (0, 2000):
        table = np.concatenate([m.table, np.full((3, width), -1)], 1)
        step = kv.KvStep(ints(table), ints([0, 1, 2, 3]), ints([3000, 100, 2222]), ints([0, 1, 2]), ints([2999, 99, 2221]))

        def one():
            ids = blocks.select(q, step, 40, window=100, id_heads=16)
            return (ids, *blocks.attend(q, ids, step, window=100), *m.cache.attend(q, step))

        first = one()
        torch.cuda.synchronize()
        side, results = [torch.cuda.Stream() for _ in range(3)], []
        for s in side * 4:
            with torch.cuda.stream(s):
                results.append(one())
        torch.cuda.synchronize()
        for r in results:
            assert all(torch.equal(a, b) for a, b in zip(r, first))


def test_wrong_calls_are_refused(kv):
    cache = kv.KvCache(4, 2, 64, 64)
    blocks = kv.KvBlocks(cache, 32)
    table = ints([[0, 1], [2, 3]])
    step = kv.KvStep(table, ints([0, 1, 3]), ints([1, 2]), ints([0, 1, 1]), ints([0, 0, 1]))
    q, ids = torch.zeros(3, 4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(3, 2, 5, device="cuda", dtype=torch.int32)
    codes, exponents = blocks.codes, blocks.exponents
    bad = [lambda: kv.KvBlocks(cache, 24), lambda: kv.KvBlocks(cache, 128), lambda: kv.KvBlocks(cache, 0), lambda: kv.KvBlocks(None, 32),
           lambda: kv.KvBlocks.from_tensors(cache, codes[:3], exponents), lambda: kv.KvBlocks.from_tensors(cache, codes, exponents[..., :1]),
           lambda: kv.KvBlocks.from_tensors(cache, codes.float(), exponents), lambda: kv.KvBlocks.from_tensors(cache, codes.cpu(), exponents),
           lambda: kv.KvBlocks.from_tensors(cache, codes[..., :32].contiguous(), exponents), lambda: blocks.update(torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: blocks.update(torch.zeros(3, dtype=torch.int64)), lambda: blocks.select(q.float(), step, 2), lambda: blocks.select(q[:2], step, 2),
           lambda: blocks.select(q, step, -1), lambda: blocks.select(q, step, 2, window=-1), lambda: blocks.select(q, step, 2, id_heads=1),
           lambda: blocks.select(q, step, 2, id_heads=3), lambda: blocks.select(q, step, 2, id_heads=0), lambda: blocks.select(q, step, 1 << 26),
           lambda: blocks.select(q, kv.KvStep(table, ints([0, 1, 3]), ints([1, 2])), 2), lambda: blocks.select(q, step, 5, out=ids[..., :4]),
           lambda: blocks.select(q, step, 5, out=ids.long()), lambda: blocks.select(q, step, 5, out=ids.transpose(1, 2).contiguous().transpose(1, 2)),
           lambda: blocks.attend(q, ids.long(), step), lambda: blocks.attend(q, ids[:2], step), lambda: blocks.attend(q, ids[:, :1], step),
           lambda: blocks.attend(q[..., :32], ids, step), lambda: blocks.attend(q, ids, step, softcap=-1.0),
           lambda: blocks.attend(q, ids, kv.KvStep(table, ints([0, 1, 3]), ints([1, 2]))), lambda: blocks.attend(q.float().requires_grad_().half(), ids, step)]
    for i, call in enumerate(bad):
        with pytest.raises(kv.PagError):
            call()
            pytest.fail("call %d was not refused" % i)
    assert blocks.select(q, step, 0).shape == (3, 2, 0) and blocks.select(q[:0], kv.KvStep(table, requests=ints([]), positions=ints([])), 4).shape == (0, 2, 4)
