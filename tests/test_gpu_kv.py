"""The 8-bit key/value cache on the GPU against a plain implementation in 64 bits: block tables, writing, reading, attention over all
tokens and over listed ones."""
import math

import numpy as np
import pytest

import kv_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def kv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2603_06660_amd import kv, load_library
    load_library()
    return kv


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def wide(x):
    return x.double().cpu().numpy()


# ---- block tables -----------------------------------------------------------------------------------------------------------


def check_step(step, tables, want, table):
    torch.cuda.synchronize()
    for name in ("offsets", "context", "granted", "lengths", "free_count", "slots", "positions", "requests"):
        assert getattr(step, name).tolist() == list(want[name]), name
    assert (tables.table.cpu().numpy() == table).all()


@pytest.mark.parametrize("requests, page, max_pages, pages, most, pad", [
    (1, 16, 4, 4, 70, 0), (1, 32, 1, 1, 33, 3), (7, 16, 5, 20, 60, 2), (64, 64, 6, 400, 3, 0), (64, 16, 40, 700, 300, 100),
    (1100, 16, 3, 2000, 9, 0), (2500, 16, 2, 3000, 2, 5), (3, 128, 40, 100, 4000, 0)])
def test_extend(kv, requests, page, max_pages, pages, most, pad):
    """Several steps, some of whose requests find no room, in a row or no pages, some with nothing or less than nothing to add."""
    rng = np.random.default_rng(requests * 1000 + page)
    tables = kv.KvTables(requests, max_pages, pages, page)
    tables.free_pages.copy_(ints(rng.permutation(pages)))
    table = np.full((requests, max_pages), -1)
    lengths, free, count = np.zeros(requests, int), tables.free_pages.cpu().numpy(), pages
    for round_ in range(4):
        add = rng.integers(-1, most + 1, requests)
        total = int(np.maximum(add, 0).sum()) + pad
        want = plain.extend(lengths, table, free, count, add, page, total)
        step = tables.extend(ints(add), total, max_new=most)
        check_step(step, tables, want, table)
        tables.commit(step)
        lengths, count = np.array(want["lengths"]), want["free_count"][0]
    assert (lengths > 0).any()


def test_extend_a_step_that_is_dropped_takes_nothing_and_a_refused_request_keeps_what_it_has(kv):
    tables = kv.KvTables(3, 4, 5, 16)
    tables.commit(tables.extend(ints([20, 5, 0]), 25))
    before = tables.lengths.clone(), tables.free_count.clone()
    step = tables.extend(ints([40, 3, 1]), 44)                     # request 0 takes the two pages that are left, request 2 wants one
    assert step.granted.tolist() == [1, 1, 0] and step.context.tolist() == [60, 8, 0] and step.lengths.tolist() == [60, 8, 0]
    assert torch.equal(tables.lengths, before[0]) and torch.equal(tables.free_count, before[1])
    again = tables.extend(ints([12, 3, 1]), 16, out=kv.KvStep.empty(3, 16))
    assert again.granted.tolist() == [1, 1, 1] and again.context.tolist() == [32, 8, 1] and again.free_count.tolist() == [1]


def test_extend_in_place_and_release(kv):
    """Pages go round: what is released is handed out again, last page first."""
    rng = np.random.default_rng(5)
    tables = kv.KvTables(40, 8, 150, 16)
    table, lengths, free = np.full((40, 8), -1), np.zeros(40, int), list(range(149, -1, -1))
    step = None
    for round_ in range(8):
        add = rng.integers(0, 40, 40)
        total = int(add.sum())
        want = plain.extend(lengths, table, free, len(free), add, 16, total)
        step = tables.extend(ints(add), total, commit=True)
        check_step(step, tables, want, table)
        lengths, free = np.array(want["lengths"]), free[:want["free_count"][0]]
        assert tables.lengths.tolist() == lengths.tolist() and tables.free_count.tolist() == [len(free)]
        done = (rng.random(40) < 0.4).astype(int)
        tables.release(ints(done))
        for r in np.flatnonzero(done):
            free += table[r, :-(-lengths[r] // 16)].tolist()
            lengths[r] = 0
        assert tables.lengths.tolist() == lengths.tolist() and tables.free_count.tolist() == [len(free)]
        assert tables.free_pages[:len(free)].tolist() == free
    assert len(free) < 150


def test_extend_with_a_stack_of_the_free_pages_alone(kv):
    """The stack need not have room for pages that are held: their numbers may lie beyond its size."""
    rng = np.random.default_rng(8)
    pages, order = 60, np.random.default_rng(9).permutation(60)
    lengths = np.array([100, 3, 0, 64, 250])
    table, first = np.full((5, 20), -1), 0
    for r, n in enumerate(-(-lengths // 16)):
        table[r, :n] = order[first:first + n]
        first += n
    free = order[first:]
    for add in ([1, 1, 1, 1, 1], [40, 0, 60, 16, 3], rng.integers(0, 30, 5).tolist()):
        mine = table.copy()
        tables = kv.KvTables.from_tensors(ints(lengths), ints(table), ints(free), ints([len(free)]), 16)
        want = plain.extend(lengths, mine, free, len(free), add, 16, sum(add))
        check_step(tables.extend(ints(add), sum(add)), tables, want, mine)


def test_extend_of_no_tokens_at_all(kv):
    tables = kv.KvTables(2, 2, 2, 16)
    step = tables.extend(ints([0, -3]), 0)
    assert step.offsets.tolist() == [0, 0, 0] and step.granted.tolist() == [1, 1] and step.context.tolist() == [0, 0]


# ---- writing and reading ------------------------------------------------------------------------------------------------------


def garbage(shape, seed):
    return torch.randint(0, 256, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.uint8)


def new_cache(kv, pages, heads, dim, page, fmt, seed):
    """A cache over memory that was used for something else before (zeros behind head_dim, which the format asks for)."""
    width = -(-dim // 64) * 64
    data = garbage((pages, heads, page, 2, width), seed)
    data[..., dim:] = 0
    exponents = garbage((pages, heads, page // 16, 2), seed + 1).view(torch.int8)
    return kv.KvCache.from_tensors(data.cuda(), exponents.cuda(), dim, fmt), data.numpy().copy(), exponents.numpy().copy()


def same_cache(cache, data, exponents):
    assert (cache.exponents.cpu().numpy() == exponents).all()
    got = cache.data.cpu().numpy()
    if cache.format == "fp8":        # -0 and 0 are one number
        got, data = np.where(got == 128, 0, got), np.where(data == 128, 0, data)
    assert (got == data).all()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim, heads, page, dtype", [(64, 1, 16, "bf16"), (128, 2, 32, "fp16"), (80, 3, 48, "fp32"), (192, 2, 16, "fp32"),
                                                     (256, 1, 64, "bf16"), (8, 2, 16, "fp16")])
def test_append_bit_for_bit(kv, fmt, dim, heads, page, dtype):
    """Steps of one and of many tokens; blocks that begin, go on, outgrow their exponents; nothing beside them is touched."""
    rng = np.random.default_rng(dim + page)
    pages = 9
    cache, data, exponents = new_cache(kv, pages, heads, dim, page, fmt, dim)
    order = rng.permutation(pages)
    length = 0
    for n in (1, 1, 3, 12, 1, 37, 1, 2, 20):
        n = min(n, pages * page - length)
        at = np.arange(length, length + n)
        slots = order[at // page] * page + at % page
        x = [torch.tensor(rng.standard_normal((n, heads, dim)) * 2.0 ** rng.integers(-6, 7, (n, heads, 1))).to(DTYPES[dtype]) for _ in range(2)]
        if n == 3:
            x[0][1, 0] = 0.0
            x[1][:] = 0.0
        cache.append(x[0].cuda(), x[1].cuda(), torch.tensor(slots).cuda())
        plain.append(data, exponents, dim, fmt, wide(x[0]), wide(x[1]), slots)
        same_cache(cache, data, exponents)
        length += n
    slots = torch.tensor(order[np.arange(length) // page] * page + np.arange(length) % page)
    want = plain.numbers(data, exponents, dim, fmt)[slots.numpy() // page, :, slots.numpy() % page]      # [tokens, heads, 2, dim]
    for name in ("fp32", "bf16", "fp16"):
        got = cache.read(slots.cuda(), dtype=DTYPES[name])
        for kind in range(2):
            # the first two hold every number; the third rounds some
            exact = torch.tensor(want[:, :, kind]).to(DTYPES[name])
            assert got[kind].dtype == DTYPES[name] and (got[kind].cpu() == exact).all()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_append_of_values_at_the_edges(kv, fmt):
    """Zeros, infinities, NaN, the smallest and largest numbers, numbers whose magnitude is exactly a largest code's."""
    most = plain.LARGEST[fmt]
    rows = [[0.0] * 8, [math.nan] * 8, [math.inf, -math.inf, 1.0, -2.0, math.nan, 0.0, 3.0, most], [1e-38, -1e-40, 0, 0, 0, 0, 0, 2.0 ** -126],
            [3.0e38, -3.4e38, 1.0, 0, 0, 0, 0, 0], [most, -most, most / 2, 1.0, 0.5, 0.25, 0, 0], [most * 1.0001, 0, 0, 0, 0, 0, 0, 1.0],
            [most * 2.0 ** -64, 2.0 ** -66, -(2.0 ** -65), 0, 0, 0, 0, 0], [-0.0, 1.5, 2.5, -2.5, 3.5, 1.0625, 1.1875, 17.0]]
    for together in (False, True):
        pages = len(rows) + 2
        cache, data, exponents = new_cache(kv, pages, 1, 8, 16, fmt, 3)
        x = torch.tensor(rows, dtype=torch.float32)[:, None]
        # each row in a block of its own, after a row of small numbers; or all in one block, one after the other
        for i in range(len(rows)):
            if not together:
                small = torch.full((1, 1, 8), 2.0 ** -70)
                cache.append(small.cuda(), small.cuda(), torch.tensor([i * 16]).cuda())
                plain.append(data, exponents, 8, fmt, wide(small), wide(small), [i * 16])
            slot = i if together else i * 16 + 1
            cache.append(x[i:i + 1].cuda(), -x[i:i + 1].cuda(), torch.tensor([slot]).cuda())
            plain.append(data, exponents, 8, fmt, wide(x[i:i + 1]), -wide(x[i:i + 1]), [slot])
            same_cache(cache, data, exponents)


@pytest.mark.parametrize("tokens, heads", [(300, 12), (700, 8), (5000, 8)])
def test_append_of_prompts(kv, tokens, heads):
    """Waves with one new token, with 4 and with 16; runs that begin and end anywhere in a block, with slots that are none between them."""
    rng = np.random.default_rng(tokens)
    dim, page, pages = 16, 32, tokens // 8 + 40
    cache, data, exponents = new_cache(kv, pages, heads, dim, page, "fp8", tokens)
    order, slots, first = rng.permutation(pages), [], 0
    while len(slots) < tokens:                       # a request: some tokens from some place on, in pages of its own
        n, start = int(rng.integers(1, 70)), int(rng.integers(0, page))
        at = np.arange(start, start + n)
        need = int(at[-1]) // page + 1
        if first + need > pages:
            break
        slots += (order[first + at // page] * page + at % page).tolist() + [-1] * int(rng.integers(0, 3) == 0)
        first += need
    slots = (slots + [-1] * tokens)[:tokens]
    x = [torch.tensor(rng.standard_normal((tokens, heads, dim)) * 2.0 ** rng.integers(-6, 7, (tokens, heads, 1))).to(torch.bfloat16) for _ in range(2)]
    cache.append(x[0].cuda(), x[1].cuda(), torch.tensor(slots).cuda())
    plain.append(data, exponents, dim, "fp8", wide(x[0]), wide(x[1]), slots)
    same_cache(cache, data, exponents)
    numbers = plain.numbers(data, exponents, dim, "fp8")
    at = np.maximum(slots, 0)
    want = torch.tensor(np.where(np.asarray(slots)[:, None, None, None] < 0, 0.0, numbers[at // page, :, at % page]))
    got = cache.read(torch.tensor(slots).cuda(), dtype=torch.bfloat16)
    for kind in range(2):
        assert torch.equal(got[kind].cpu(), want[:, :, kind].to(torch.bfloat16))


def test_append_leaves_out_slots_that_are_none(kv):
    cache, data, exponents = new_cache(kv, 3, 2, 64, 16, "int8", 9)
    slots = np.array([-1, 5, 6, -7, 48, 1 << 40, 17, 32, -(1 << 62)])
    x = torch.randn(len(slots), 2, 64)
    cache.append(x.cuda(), x.cuda(), torch.tensor(slots).cuda())
    plain.append(data, exponents, 64, "int8", wide(x), wide(x), slots.tolist())
    same_cache(cache, data, exponents)
    out = cache.read(torch.tensor([-1, 32, 48, 1 << 40]).cuda())
    assert (out[0][[0, 2, 3]] == 0).all() and (out[1][[0, 2, 3]] == 0).all()
    assert (wide(out[0][1]) == plain.numbers(data, exponents, 64, "int8")[2, :, 0, 0]).all()


def test_strides_of_inputs_and_outputs(kv):
    """Slices of a fused projection go in, rows come out head by head."""
    tokens, heads, dim = 37, 3, 64
    fused = torch.randn(tokens, 5 * heads, dim + 8, device="cuda", dtype=torch.bfloat16)
    k, v = fused[:, heads:2 * heads, :dim], fused[:, 3 * heads:4 * heads, 8:]
    slots = torch.arange(tokens, device="cuda")
    one, two = kv.KvCache(3, heads, dim, 16), kv.KvCache(3, heads, dim, 16)
    one.append(k, v, slots)
    two.append(k.contiguous(), v.contiguous(), slots)
    assert torch.equal(one.data, two.data) and torch.equal(one.exponents, two.exponents)
    by_head = torch.full((heads, tokens, dim), 7.0, device="cuda")
    one.read(slots, out=(by_head.transpose(0, 1), None))
    assert torch.equal(by_head, two.read(slots)[0].transpose(0, 1))
    values = torch.empty(tokens, heads, 2 * dim, device="cuda", dtype=torch.float16)
    one.read(slots, out=(None, values[..., dim:]))
    assert torch.equal(values[..., dim:], two.read(slots, dtype=torch.float16)[1])


# ---- attention ------------------------------------------------------------------------------------------------------------------


class Memory:
    """Requests with random keys and values in scattered pages of memory that holds anything elsewhere."""

    def __init__(self, kv, contexts, kv_heads, dim, page, fmt, seed, spread=1.0):
        rng = np.random.default_rng(seed)
        counts = [-(-c // page) for c in contexts]
        self.pages = sum(counts) + 2
        order = rng.permutation(self.pages)
        self.table = np.full((len(contexts), max(counts + [1]) + 1), -1)
        self.page, self.fmt, self.dim, self.kv_heads, self.contexts = page, fmt, dim, kv_heads, contexts
        data = np.full((self.pages, kv_heads, page, 2, -(-dim // 64) * 64), 0x7F, np.uint8)      # NaN, in one format
        exponents = np.full((self.pages, kv_heads, page // 16, 2), 127, np.int8)
        data[..., dim:] = 0
        first = 0
        for b, (c, n) in enumerate(zip(contexts, counts)):
            self.table[b, :n] = order[first:first + n]
            first += n
            at = np.arange(c)
            slots = self.table[b, at // page] * page + at % page
            x = rng.standard_normal((2, c, kv_heads, dim)) * spread * 2.0 ** rng.integers(-1, 2, (2, 1, kv_heads, 1))
            x[0, ..., :: 16] *= 3
            plain.append(data, exponents, dim, fmt, x[0], x[1], slots)
            # only what is behind the end of the request stays as it was
            if c % 16:
                data[self.table[b, n - 1], :, c % page:, :, :dim] = 0x7F
        # numbers of unused memory are never looked at
        self.numbers = plain.numbers(data, np.minimum(exponents, 100), dim, fmt)
        self.cache = kv.KvCache.from_tensors(torch.tensor(data).cuda(), torch.tensor(exponents).cuda(), dim, fmt)

    def rows(self, b, at, head):
        p, t = self.table[b, at // self.page], at % self.page
        return self.numbers[p, head, t, 0], self.numbers[p, head, t, 1]


def check_attention(memory, q, out, lse, dtype, requests, positions, keys_of, scale, softcap=0.0, slopes=None):
    """keys_of(token, head) -> positions that the row reads."""
    q, out, lse = wide(q), wide(out), wide(lse)
    assert not np.isnan(out).any() and not np.isnan(lse).any()
    heads = q.shape[1]
    worst = 0.0
    for t in range(q.shape[0]):
        for h in range(heads):
            at = keys_of(t, h) if positions[t] >= 0 else np.zeros(0, int)
            if len(at) == 0:
                assert (out[t, h] == 0).all() and lse[t, h] == -math.inf, (t, h)
                continue
            k, v = memory.rows(requests[t], at, h * memory.kv_heads // heads)
            slope = slopes[h] if slopes is not None else 0.0
            o, l, spread, products = plain.attend_row(q[t, h], k, v, scale, softcap, slope, positions[t] - at)
            tol_o, tol_l = plain.tolerance(memory.dim, 8 if dtype == "bf16" else 11, o, spread, products, softcap,
                                           abs(slope) * (positions[t] - at.min()))
            assert abs(lse[t, h] - l) <= tol_l, (t, h, lse[t, h], l, tol_l)
            worst = max(worst, float((np.abs(out[t, h] - o) / tol_o).max()))
            assert worst <= 1.0, (t, h, worst)
    return worst


def attend_case(kv, contexts, news, heads, kv_heads, dim, page, fmt, dtype, window=0, softcap=0.0, slopes=False, pad=0, seed=1, scale=None, max_new=None):
    m = Memory(kv, contexts, kv_heads, dim, page, fmt, seed)
    tokens = sum(news) + pad
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(tokens, heads, dim, generator=gen).to(DTYPES[dtype])
    slope = np.exp2(-8.0 * (1 + np.arange(heads)) / heads).astype(np.float32) if slopes else None
    requests = [b for b, a in enumerate(news) for _ in range(a)] + [-1] * pad
    positions = [p for c, a in zip(contexts, news) for p in range(c - a, c)] + [-1] * pad
    step = kv.KvStep(ints(m.table), offsets=ints(np.concatenate([[0], np.cumsum(news)])), context=ints(contexts), max_new=max(news) if max_new is None else max_new)
    out = (torch.full((tokens, heads, dim), 7.0, dtype=DTYPES[dtype], device="cuda"), torch.full((tokens, heads), 7.0, device="cuda"))
    got = m.cache.attend(q.cuda(), step, window=window, softcap=softcap, slopes=None if slope is None else torch.tensor(slope).cuda(), out=out, scale=scale)
    assert got[0] is out[0] and got[1] is out[1]

    def keys_of(t, h):
        p = positions[t]
        return np.arange(max(0, p - window + 1) if window else 0, p + 1)

    check_attention(m, q, out[0], out[1], dtype, requests, positions, keys_of, dim ** -0.5 if scale is None else scale, softcap, slope)
    return m


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
def test_attend_one_token_each(kv, fmt, dim):
    """Lengths around the edges of blocks, tiles and units, one without a token, one longer than many units."""
    contexts = [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 300, 1000]
    attend_case(kv, contexts, [1] * len(contexts), 8, 2, dim, 32, fmt, "bf16" if dim % 128 else "fp16")


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 1), (16, 1), (17, 1), (40, 1), (12, 4), (64, 2)])
@pytest.mark.parametrize("page", [16, 48, 128])
def test_attend_groups_and_pages(kv, heads, kv_heads, page):
    attend_case(kv, [5, 70, 333], [1, 1, 1], heads, kv_heads, 64, page, "int8", "fp16")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim, heads, kv_heads, dtype", [(64, 4, 4, "bf16"), (128, 8, 2, "fp16"), (96, 6, 2, "bf16"), (192, 2, 1, "fp16"), (256, 16, 2, "bf16")])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_attend_chunks(kv, fmt, dim, heads, kv_heads, dtype, window):
    """Several new tokens, some requests with nothing but them, one with none, padding behind."""
    attend_case(kv, [1, 40, 70, 37, 200, 130], [1, 40, 3, 0, 17, 33], heads, kv_heads, dim, 16, fmt, dtype, window=window, pad=3)


@pytest.mark.parametrize("softcap, slopes, window", [(30.0, False, 0), (0.0, True, 0), (2.0, True, 50), (0.5, False, 7)])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [20, 1, 60, 90]])
def test_attend_cap_and_distance(kv, softcap, slopes, window, news):
    attend_case(kv, [33, 1, 200, 90], news, 6, 2, 128, 32, "fp8", "bf16", window=window, softcap=softcap, slopes=slopes)


def test_attend_many_requests(kv):
    """More requests than threads of a workgroup, more units than workgroups; empty ones between."""
    rng = np.random.default_rng(3)
    contexts = rng.integers(0, 60, 300)
    contexts[::7] = 0
    news = np.minimum(1, contexts)
    attend_case(kv, contexts.tolist(), news.tolist(), 2, 1, 64, 16, "int8", "bf16")


def test_attend_pieces_of_several_units(kv):
    attend_case(kv, [20_000, 9000, 30_011], [1, 2, 1], 8, 8, 64, 64, "int8", "fp16")
    attend_case(kv, [5000, 2000, 3011], [40, 70, 100], 8, 8, 64, 64, "fp8", "fp16")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
def test_attend_two_tiles_of_rows_in_pieces(kv, fmt, dim):
    """17 to 64 rows to a key over more keys than one workgroup reads."""
    attend_case(kv, [4100, 2300, 900], [1, 2, 0], 20, 1, dim, 64, fmt, "bf16")
    attend_case(kv, [3000, 40], [8, 8], 8, 1, dim, 64, fmt, "fp16", window=2500, softcap=20.0)


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [40, 128])
@pytest.mark.parametrize("softcap, slopes, window", [(0.0, False, 0), (30.0, False, 0), (0.0, True, 90), (5.0, True, 0)])
def test_attend_long_chunks(kv, fmt, dim, softcap, slopes, window):
    """More than 128 rows to a key, in one request of several."""
    attend_case(kv, [400, 33, 0, 150], [300, 33, 0, 1], 2, 1, dim, 32, fmt, "fp16", softcap=softcap, slopes=slopes, window=window, pad=2)


@pytest.mark.parametrize("max_new", [0, 1, 4, 16, 20, 37, 300])
def test_attend_with_any_hint(kv, max_new):
    """max_new decides which kernels run, and not what they compute, also where it is wrong."""
    attend_case(kv, [2900, 40, 700], [37, 5, 1], 4, 1, 64, 64, "int8", "fp16", max_new=max_new)


def test_attend_of_a_long_chunk(kv):
    """Pieces of many thousand keys, by each of the kernels: rows here and there against the plain form, all rows against each other."""
    context, new, heads, kv_heads, dim = 20_003, 448, 32, 8, 64
    m = Memory(kv, [context], kv_heads, dim, 64, "fp8", 4)
    q = torch.randn(new, heads, dim, generator=torch.Generator().manual_seed(4)).half()
    some = [0, 1, 200, 447]
    first = None
    for max_new in (1, 16, 20, 448):
        step = kv.KvStep(ints(m.table), offsets=ints([0, new]), context=ints([context]), max_new=max_new)
        out, lse = m.cache.attend(q.cuda(), step)
        check_attention(m, q[some], out[some], lse[some], "fp16", [0] * len(some), [context - new + t for t in some],
                        lambda t, h: np.arange(context - new + some[t] + 1), dim ** -0.5)
        if first is None:
            first = out, lse
        # weights of 11 bits and an output of 11 bits on each side, of numbers that are below 8 in magnitude
        assert (out.float() - first[0].float()).abs().max() <= 4 * 2.0 ** -11 * 8 and (lse - first[1]).abs().max() <= 2.0 ** -10


def test_attend_of_more_rows_than_a_launch_has_threads_for(kv):
    """2^19 requests of 16 heads: the results are those of the requests a thousand at a time, to 11 bits of weights and 11 of output on both sides."""
    requests, heads, dim = 1 << 19, 16, 8
    m = Memory(kv, [48] * 8, 1, dim, 16, "int8", 12)
    order = torch.randint(0, 8, (requests,), generator=torch.Generator().manual_seed(12))
    table = torch.tensor(m.table, dtype=torch.int32)[order].cuda()
    context = (torch.arange(requests, dtype=torch.int32, device="cuda") * 7) % 49
    offsets = torch.arange(requests + 1, dtype=torch.int32, device="cuda")
    q = torch.randn(requests, heads, dim, device="cuda").half()
    out, lse = m.cache.attend(q, kv.KvStep(table, offsets=offsets, context=context, max_new=1))
    for first in (0, 262_000, requests - 1000):
        step = kv.KvStep(table[first:first + 1000], offsets=offsets[:1001].clone(), context=context[first:first + 1000].clone(), max_new=1)
        some, some_lse = m.cache.attend(q[first:first + 1000], step)
        there = context[first:first + 1000] > 0
        most = some.float().abs().max()
        assert (out[first:first + 1000].float() - some.float()).abs().max() <= 4 * 2.0 ** -11 * max(float(most), 1.0)
        assert (lse[first:first + 1000] - some_lse)[there].abs().max() <= 2.0 ** -10 and (lse[first:first + 1000][~there] == -math.inf).all()


def test_attend_scores_far_apart(kv):
    """A running maximum that rises by a lot, late; scores that leave one key only; scale 0, where all weights are equal."""
    for scale in (20.0, -3.0, 0.0):
        attend_case(kv, [400, 90], [3, 1], 4, 2, 64, 16, "int8", "fp16", scale=scale)


def test_attend_values_of_very_different_blocks(kv):
    """Blocks whose exponents are far apart: a weight times a block's scale does not leave the range of a 16-bit float."""
    dim, page = 64, 16
    cache = kv.KvCache(8, 1, dim, page)
    data, exponents = np.zeros((8, 1, 16, 2, 64), np.uint8), np.zeros((8, 1, 1, 2), np.int8)
    gen = torch.Generator().manual_seed(5)
    k = torch.randn(128, 1, dim, generator=gen)
    v = torch.randn(128, 1, dim, generator=gen)
    for i, e in enumerate((0, -40, 12, 0, -90, 30, 5, 0)):
        v[16 * i:16 * i + 16] *= 2.0 ** e
    v[48:64] = 0
    for order in ((0, 1, 2, 3, 4, 5, 6, 7), (5, 2, 0, 1, 3, 4, 6, 7), (1, 3, 4, 1, 1, 1, 1, 1)):
        slots = torch.arange(128)
        cache.append(k.cuda(), v.cuda(), slots.cuda())
        plain.append(data, exponents, dim, "int8", wide(k), wide(v), slots.tolist())
        numbers = plain.numbers(data, exponents, dim, "int8")
        for n in (16, 40, 128):
            step = kv.KvStep(ints([order]), offsets=ints([0, 1]), context=ints([n]))
            q = torch.randn(1, 2, dim, generator=gen).half()
            out, lse = cache.attend(q.cuda(), step)
            at = np.arange(n)
            rows = numbers[np.array(order)[at // 16], 0, at % 16]
            for h in range(2):
                o, l, spread, products = plain.attend_row(wide(q[0, h]), rows[:, 0], rows[:, 1], dim ** -0.5)
                tol_o, tol_l = plain.tolerance(dim, 11, o, spread, products)
                if np.abs(o).max() < 60000:
                    assert (np.abs(wide(out[0, h]) - o) <= tol_o).all()
                assert abs(float(lse[0, h]) - l) <= tol_l


def test_attend_rows_with_infinities_and_nan_spoil_only_themselves(kv):
    m = Memory(kv, [50, 90], 2, 64, 16, "int8", 4)
    q = torch.randn(4, 4, 64).half()
    step = kv.KvStep(ints(m.table), offsets=ints([0, 2, 4]), context=ints([50, 90]))
    clean = m.cache.attend(q.cuda(), step)
    q[0, 1, 5], q[3, 2, 0], q[2, 0, 7] = math.nan, math.inf, -math.inf
    out, lse = m.cache.attend(q.cuda(), step)
    spoilt = torch.zeros(4, 4, dtype=torch.bool)
    spoilt[0, 1] = spoilt[3, 2] = spoilt[2, 0] = True
    assert torch.isnan(out.cpu()[spoilt]).all()
    assert torch.equal(out.cpu()[~spoilt], clean[0].cpu()[~spoilt]) and torch.equal(lse.cpu()[~spoilt], clean[1].cpu()[~spoilt])


def test_attend_pages_that_do_not_exist(kv):
    """Page numbers out of range and contexts beyond the table count as absent."""
    m = Memory(kv, [64, 40], 1, 64, 16, "fp8", 4)
    q = torch.randn(2, 2, 64).to(torch.bfloat16)
    table = m.table.copy()
    table[0, 1], table[0, 2] = m.pages, -5
    step = kv.KvStep(ints(table), offsets=ints([0, 1, 2]), context=ints([64, 40]))
    out, lse = m.cache.attend(q.cuda(), step)
    keys = lambda t, h: np.concatenate([np.arange(16), np.arange(48, 64)]) if t == 0 else np.arange(40)
    check_attention(m, q, out, lse, "bf16", [0, 1], [63, 39], keys, 64 ** -0.5)
    ids = torch.arange(64, device="cuda").expand(2, 1, 64).contiguous()
    step = kv.KvStep(ints(table), requests=ints([0, 7]), positions=ints([63, 39]))
    out, lse = m.cache.attend_selected(q.cuda(), ids, step)
    check_attention(m, q, out, lse, "bf16", [0, 1], [63, -1], keys, 64 ** -0.5)
    step = kv.KvStep(ints(m.table), offsets=ints([0, 1, 2]), context=ints([2_000_000_000, -4]))
    out, lse = m.cache.attend(q.cuda(), step)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()


def test_attend_is_the_same_every_time_and_on_any_stream(kv):
    m = Memory(kv, [3000, 100, 2222], 4, 128, 64, "int8", 6)
    q = torch.randn(3, 16, 128, device="cuda").half()
    step = kv.KvStep(ints(m.table), offsets=ints([0, 1, 2, 3]), context=ints([3000, 100, 2222]), requests=ints([0, 1, 2]), positions=ints([2999, 99, 2221]))
    ids = torch.randint(0, 2000, (3, 16, 200), device="cuda")
    first, listed = m.cache.attend(q, step), m.cache.attend_selected(q, ids, step, window=100)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    results = []
    for s in side * 4:
        with torch.cuda.stream(s):
            results.append((m.cache.attend(q, step), m.cache.attend_selected(q, ids, step, window=100)))
    torch.cuda.synchronize()
    for a, b in results:
        assert torch.equal(a[0], first[0]) and torch.equal(a[1], first[1])
        assert torch.equal(b[0], listed[0]) and torch.equal(b[1], listed[1])


def test_rows_beyond_32_bits_of_offset(kv):
    """A cache of 5 GB: pages whose bytes lie behind the first 4 GB."""
    pages, heads, page, dim = 5 * (1 << 30) // (2 * 64 * 256), 2, 64, 128
    cache = kv.KvCache.from_tensors(torch.empty((pages, heads, page, 2, dim), dtype=torch.uint8, device="cuda"),
                                    torch.empty((pages, heads, page // 16, 2), dtype=torch.int8, device="cuda"), dim, "int8")
    order = np.array([pages - 1, 3, pages - 70, pages // 2])
    at = np.arange(250)
    slots = torch.tensor(order[at // page] * page + at % page).cuda()
    k, v = torch.randn(250, heads, dim, device="cuda"), torch.randn(250, heads, dim, device="cuda")
    cache.append(k, v, slots)
    small = kv.KvCache(4, heads, dim, page)
    small.append(k, v, torch.tensor(at).cuda())
    for x, y in zip(cache.read(slots), small.read(torch.tensor(at).cuda())):
        assert torch.equal(x, y)
    q = torch.randn(1, 4, dim, device="cuda").half()
    ids = torch.tensor([249, 0, 100, 64, 63, 128, -1]).cuda().view(1, 1, -1).expand(1, 2, 7)
    for a, b in ((kv.KvStep(ints([order]), ints([0, 1]), ints([250]), ints([0]), ints([249])),
                  kv.KvStep(ints([[0, 1, 2, 3]]), ints([0, 1]), ints([250]), ints([0]), ints([249]))),):
        assert all(torch.equal(x, y) for x, y in zip(cache.attend(q, a), small.attend(q, b)))
        assert all(torch.equal(x, y) for x, y in zip(cache.attend_selected(q, ids, a), small.attend_selected(q, ids, b)))


# ---- attention over listed tokens -------------------------------------------------------------------------------------------------


def selected_case(kv, contexts, heads, kv_heads, id_heads, dim, k, window, fmt, dtype, page=32, softcap=0.0, slopes=False, seed=2, pad=0):
    m = Memory(kv, contexts, kv_heads, dim, page, fmt, seed)
    rng = np.random.default_rng(seed)
    tokens = len(contexts) + pad
    q = torch.tensor(rng.standard_normal((tokens, heads, dim))).to(DTYPES[dtype])
    slope = np.exp2(-8.0 * (1 + np.arange(heads)) / heads).astype(np.float32) if slopes else None
    # positions of the request and of none: -1, beyond the token, far beyond, listed twice, in the window
    ids = np.full((tokens, id_heads, k), -1, np.int64)
    for t, c in enumerate(contexts):
        for i in range(id_heads):
            row = rng.integers(-1, c + 3, k)
            row[rng.random(k) < 0.1] = -1
            row[rng.random(k) < 0.02] = (1 << 40) + 3
            if t % 5 == 4:
                row[:] = -1
            ids[t, i] = row
    requests, positions = list(range(len(contexts))) + [-1] * pad, [c - 1 for c in contexts] + [-1] * pad
    step = kv.KvStep(ints(m.table), requests=ints(requests), positions=ints(positions))
    out, lse = m.cache.attend_selected(q.cuda(), torch.tensor(ids).cuda(), step, window=window, softcap=softcap,
                                       slopes=None if slope is None else torch.tensor(slope).cuda())

    def keys_of(t, h):
        p, row = positions[t], ids[t, h * id_heads // heads]
        return np.concatenate([row[(row >= 0) & (row <= p - window)], np.arange(max(0, p - window + 1), p + 1)]).astype(int)

    check_attention(m, q, out, lse, dtype, requests, positions, keys_of, dim ** -0.5, softcap, slope)


@pytest.mark.parametrize("fmt, dtype", [("int8", "bf16"), ("fp8", "fp16")])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("k, window", [(1, 0), (10, 1), (33, 16), (100, 64), (300, 0)])
def test_selected(kv, fmt, dtype, dim, k, window):
    selected_case(kv, [300, 1, 40, 130, 64, 17], 4, 2, 2, dim, k, window, fmt, dtype)


@pytest.mark.parametrize("heads, kv_heads, id_heads", [(1, 1, 1), (8, 2, 8), (8, 2, 4), (40, 2, 2), (48, 1, 2), (12, 4, 12)])
def test_selected_heads(kv, heads, kv_heads, id_heads):
    selected_case(kv, [200, 90, 513, 33, 50], heads, kv_heads, id_heads, 64, 70, 20, "int8", "fp16", pad=2)


@pytest.mark.parametrize("softcap, slopes", [(30.0, False), (0.0, True), (1.0, True)])
def test_selected_cap_and_distance(kv, softcap, slopes):
    selected_case(kv, [200, 90, 513, 33, 50], 6, 2, 2, 128, 70, 20, "fp8", "bf16", softcap=softcap, slopes=slopes)


def test_selected_nothing_at_all(kv):
    """No ids and no window: zeros."""
    selected_case(kv, [200, 90], 4, 2, 2, 64, 0, 0, "int8", "fp16")
    selected_case(kv, [200, 90], 4, 2, 4, 64, 0, 7, "int8", "fp16")


def test_selected_long_lists(kv):
    selected_case(kv, [5000, 3000, 1500], 4, 2, 2, 64, 1024, 600, "int8", "fp16")


@pytest.mark.parametrize("fmt, dim", [("int8", 128), ("fp8", 64), ("fp8", 256)])
def test_selected_of_many_tokens(kv, fmt, dim):
    """More lists than workgroups run at once."""
    rng = np.random.default_rng(6)
    selected_case(kv, rng.integers(1, 400, 45).tolist(), 16, 8, 8, dim, 90, 20, fmt, "bf16")


@pytest.mark.parametrize("tokens, k, window", [(1, 2500, 0), (3, 1200, 300), (5, 1900, 100), (5, 2600, 64), (17, 2600, 64)])
def test_selected_longer_lists(kv, tokens, k, window):
    """Lists that one workgroup reads, and lists that several share."""
    selected_case(kv, [3000 - 7 * i for i in range(tokens)], 16, 1, 16, 64, k, window, "int8", "fp16", page=64)


def test_selected_everything_is_attention(kv):
    """Listing every position, or a window over all of them, is attention over all tokens, to the order of its sums."""
    m = Memory(kv, [700, 50], 2, 128, 64, "fp8", 8)
    q = torch.randn(2, 8, 128).half()
    positions = ints([699, 49])
    step = kv.KvStep(ints(m.table), offsets=ints([0, 1, 2]), context=ints([700, 50]), requests=ints([0, 1]), positions=positions)
    everything = lambda t, h: np.arange(700 if t == 0 else 50)
    ids = torch.randperm(700, device="cuda").expand(2, 2, 700).contiguous()
    for got in (m.cache.attend_selected(q.cuda(), ids, step), m.cache.attend_selected(q.cuda(), ids[..., :0], step, window=1000),
                m.cache.attend_selected(q.cuda(), ids, step, window=1000), m.cache.attend(q.cuda(), step), m.cache.attend(q.cuda(), step, window=701)):
        check_attention(m, q, got[0], got[1], "fp16", [0, 1], [699, 49], everything, 128 ** -0.5)


# ---- a decoding loop ----------------------------------------------------------------------------------------------------------------


def test_captured_step(kv):
    """extend, append and both attentions in a graph: every replay against the same step without one."""
    heads, kv_heads, dim, page = 8, 2, 64, 16
    torch.manual_seed(3)
    state = []
    for _ in range(2):
        tables, cache = kv.KvTables(5, 6, 40, page), kv.KvCache(40, kv_heads, dim, page)
        state.append((tables, cache, kv.KvStep.empty(5, 8)))
    add = torch.zeros(5, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(8, kv_heads, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q = torch.zeros(8, heads, dim, device="cuda", dtype=torch.bfloat16)
    ids = torch.zeros(8, kv_heads, 20, dtype=torch.int64, device="cuda")

    def one(tables, cache, step):
        tables.extend(add, 8, max_new=8, out=step, commit=True)
        cache.append(k, v, step.slots)
        return (*cache.attend(q, step, window=30), *cache.attend_selected(q, ids, step, window=4))

    one(*state[0])                       # loads the kernels; nothing was added
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = one(*state[0])
    for i in range(12):
        add.copy_(torch.tensor([[1, 1, 1, 1, 1], [3, 0, 1, 4, 0], [0, 0, 8, 0, 0], [1, 2, 0, 0, 5]][i % 4], dtype=torch.int32))
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape))
        ids.copy_(torch.randint(-1, 30, ids.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = one(*state[1])
        torch.cuda.synchronize()
        for got, w in zip(captured, want):
            assert torch.equal(got, w), i
        for a, b in zip(state[0][:2], state[1][:2]):
            for name in ("table", "lengths", "free_count", "data", "exponents"):
                if hasattr(a, name):
                    assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)


def test_wrong_tensors_are_refused(kv):
    cache, tables = kv.KvCache(4, 2, 64, 16), kv.KvTables(2, 4, 4, 16)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    x = torch.zeros(3, 2, 64, device="cuda", dtype=torch.bfloat16)
    step = kv.KvStep(tables.table, ints([0, 1, 3]), ints([1, 2]), ints([0, 1, 1]), ints([0, 0, 1]))
    q, ids = torch.zeros(3, 4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(3, 2, 5, device="cuda", dtype=torch.int64)
    bad = [lambda: cache.append(x[:2], x, slots), lambda: cache.append(x, x.float(), slots), lambda: cache.append(x, x, slots.int()),
           lambda: cache.append(x.cpu(), x, slots), lambda: cache.append(x.transpose(1, 2).contiguous().transpose(1, 2), x, slots),
           lambda: cache.append(x.double(), x.double(), slots), lambda: cache.read(slots, dtype=torch.float64), lambda: cache.read(slots, out=(None, None)),
           lambda: cache.read(slots, out=(torch.zeros(3, 2, 66, device="cuda")[..., 1:65], None)),
           lambda: cache.attend(q.float(), step), lambda: cache.attend(q[:2], step), lambda: cache.attend(q[:, :3], step), lambda: cache.attend(q[..., :32], step),
           lambda: cache.attend(q, step, softcap=-1.0), lambda: cache.attend(q, step, window=-1), lambda: cache.attend(q, step, slopes=torch.zeros(3, device="cuda")),
           lambda: cache.attend(q, step, scale=math.nan), lambda: cache.attend(q, kv.KvStep(tables.table, requests=ints([0] * 3), positions=ints([0] * 3))),
           lambda: cache.attend(torch.zeros(3, 4, 68, device="cuda", dtype=torch.bfloat16)[..., 2:66], step),
           lambda: cache.attend(q, kv.KvStep.empty(2, 3)),
           lambda: cache.attend_selected(q, ids.int(), step), lambda: cache.attend_selected(q, ids[:2], step),
           lambda: cache.attend_selected(q, ids[:, :1], step), lambda: cache.attend_selected(q, ids.expand(3, 2, 5).repeat(1, 2, 1)[:, :3], step),
           lambda: cache.attend_selected(q, ids, kv.KvStep(tables.table, ints([0, 1, 3]), ints([1, 2]))),
           lambda: tables.extend(ints([1]), 1), lambda: tables.extend(ints([1, 1]).long(), 2), lambda: tables.extend(ints([1, 1]), 2, out=kv.KvStep.empty(2, 3)),
           lambda: tables.extend(ints([1, 1, 1])[:2], 2, out=step), lambda: tables.commit(step), lambda: tables.release(ints([1])),
           lambda: kv.KvCache(4, 2, 68, 16), lambda: kv.KvCache(4, 2, 264, 16), lambda: kv.KvCache(4, 2, 64, 24).read(slots),
           lambda: kv.KvStep(tables.table, ints([0, 1]))]
    for i, call in enumerate(bad):
        with pytest.raises(kv.PagError):
            call()
            pytest.fail("call %d was not refused" % i)
