"""The 8-bit key/value cache on the GPU where arguments leave their usual range: what does not fit, what lies far apart, rows that nothing covers."""
import math

import numpy as np
import pytest

import kv_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


def plain_rows(lengths, table, free, count, add, page, total):
    """plain.extend for a step of `total` rows that may be fewer than the new tokens: who has not all of its rows gets nothing."""
    wanted = np.maximum(np.asarray(add, np.int64), 0)
    ends = np.cumsum(wanted)
    short = (wanted > 0) & (ends > total)
    kept = np.where(short, 0, wanted)
    want = plain.extend(lengths, table, free, count, kept, page, max(total, int(kept.sum())))
    for r in np.flatnonzero(short):
        want["granted"][r] = want["context"][r] = 0
    want["offsets"] = [0] + ends.tolist()
    row = np.searchsorted(ends, np.arange(total), side="right")
    want["requests"] = np.where(row < len(ends), row, -1).tolist()
    return want


def check_step(step, tables, want, table):
    torch.cuda.synchronize()
    for name in ("offsets", "context", "granted", "lengths", "free_count", "slots", "positions", "requests"):
        assert getattr(step, name).tolist() == list(want[name]), name
    assert (tables.table.cpu().numpy() == table).all()


@pytest.mark.parametrize("requests, page, max_pages, pages, most, short", [
    (1, 16, 4, 4, 60, 1), (1, 16, 4, 4, 60, 50), (3, 16, 8, 20, 40, 30), (64, 16, 40, 900, 90, 200), (64, 64, 100, 4000, 600, 9000),
    (1500, 16, 3, 4000, 9, 2000)])
def test_extend_with_fewer_rows_than_tokens(kv, requests, page, max_pages, pages, most, short):
    """Tables whose rows hold the page numbers of requests that ended; what has no rows takes nothing and leaves nothing, and is served when the next
    step has rows for it.  In place and beside the tables, in one launch and in two."""
    rng = np.random.default_rng(requests + short)
    tables = kv.KvTables(requests, max_pages, pages, page)
    table, lengths, free = np.full((requests, max_pages), -1), np.zeros(requests, int), list(range(pages - 1, -1, -1))
    for round_ in range(6):
        add = rng.integers(-1, most + 1, requests)
        if round_ == 0:
            add[-1] = most
        total = int(np.maximum(add, 0).sum())
        total = total if round_ == 4 else max(total - short, 0)
        want = plain_rows(lengths, table, free, len(free), add, page, total)
        commit = round_ % 2 == 1
        step = tables.extend(ints(add), total, commit=commit)
        check_step(step, tables, want, table)
        if not commit:
            tables.commit(step)
        lengths, free = np.array(want["lengths"]), free[:want["free_count"][0]]
        # every page is held by one request or free
        held = [p for r in range(requests) for p in table[r, :-(-lengths[r] // page)].tolist()]
        assert sorted(held + free) == list(range(pages))
        done = (rng.random(requests) < 0.5).astype(int)
        tables.release(ints(done))
        for r in np.flatnonzero(done):
            free += table[r, :-(-lengths[r] // page)].tolist()
            lengths[r] = 0
        assert tables.lengths.tolist() == lengths.tolist() and tables.free_pages[:len(free)].tolist() == free


def test_extend_by_more_tokens_than_32_bits_count(kv):
    tables = kv.KvTables(4, 4, 8, 16)
    step = tables.extend(ints([5, (1 << 31) - 1, (1 << 31) - 1, 0]), 20)
    assert step.granted.tolist() == [1, 0, 0, 1] and step.context.tolist() == [5, 0, 0, 0] and step.lengths.tolist() == [5, 0, 0, 0]
    assert step.requests.tolist() == [0] * 5 + [1] * 15 and step.positions.tolist() == list(range(5)) + [-1] * 15
    assert step.slots.tolist() == list(range(5)) + [-1] * 15
    assert step.free_count.tolist() == [7]


def test_a_step_of_fewer_requests_than_the_tables_is_refused_every_time(kv):
    two, three, step = kv.KvTables(2, 4, 8, 16), kv.KvTables(3, 4, 8, 16), kv.KvStep.empty(2, 6)
    for _ in range(2):
        for _ in range(2):
            with pytest.raises(kv.PagError):
                three.extend(ints([1, 1, 1]), 6, out=step)
        assert two.extend(ints([2, 3]), 6, out=step).context.tolist() == [2, 3]
    assert three.table.eq(-1).all() and three.lengths.tolist() == [0, 0, 0]


# ---- attention ----------------------------------------------------------------------------------------------------------------


class Memory:
    """One cache whose tokens are given, in pages in some order; numpy copies of what it holds."""

    def __init__(self, kv, k, v, page, fmt, seed=1):
        n, self.kv_heads, self.dim = k.shape
        self.page, self.fmt = page, fmt
        pages = -(-n // page)
        self.order = np.random.default_rng(seed).permutation(pages)
        data = np.zeros((pages, self.kv_heads, page, 2, -(-self.dim // 64) * 64), np.uint8)
        exponents = np.zeros((pages, self.kv_heads, page // 16, 2), np.int8)
        at = np.arange(n)
        plain.append(data, exponents, self.dim, fmt, np.asarray(k, np.float64), np.asarray(v, np.float64), self.order[at // page] * page + at % page)
        self.numbers = plain.numbers(data, exponents, self.dim, fmt)
        self.cache = kv.KvCache.from_tensors(torch.tensor(data).cuda(), torch.tensor(exponents).cuda(), self.dim, fmt)

    def rows(self, at, head):
        p, t = self.order[at // self.page], at % self.page
        return self.numbers[p, head, t, 0], self.numbers[p, head, t, 1]


def check_rows(memory, q, out, lse, bits, positions, keys_of, scale, softcap=0.0, slopes=None, slack=0.0):
    """Each row against 64 bits.  The cap counts in a score's error up to 64, where another form of it begins, whose error is the score's;
    a slope counts with the distance between the keys that a row reads, not with their distance from the row: only lse, a number of 32
    bits, is off by its own size.  slack: added to out's tolerance, times the largest |value|."""
    q, out, lse = wide(q), wide(out), wide(lse)
    heads = q.shape[1]
    for t in range(q.shape[0]):
        for h in range(heads):
            at = keys_of(t, h)
            if len(at) == 0:
                assert (out[t, h] == 0).all() and lse[t, h] == -math.inf, (t, h)
                continue
            k, v = memory.rows(at, h * memory.kv_heads // heads)
            slope = 0.0 if slopes is None else float(slopes[h])
            o, l, spread, products = plain.attend_row(q[t, h], k, v, scale, softcap, slope, positions[t] - at)
            tol_o, tol_l = plain.tolerance(memory.dim, bits, o, spread, products, min(softcap, 64.0), abs(slope) * float(at.max() - at.min()))
            assert abs(lse[t, h] - l) <= tol_l + 2.0 ** -22 * abs(l), (t, h, lse[t, h], l, tol_l)
            assert (np.abs(out[t, h] - o) <= tol_o + slack * np.abs(v).max()).all(), (t, h, np.abs(out[t, h] - o).max(), tol_o.min())


def normal(shape, seed, scale=1.0):
    return np.random.default_rng(seed).standard_normal(shape) * scale


@pytest.mark.parametrize("window", [0, 1, 4, 7, (1 << 31) - 17, (1 << 31) - 1])
@pytest.mark.parametrize("max_new", [1, 20, 300])
def test_requests_that_hold_fewer_tokens_than_they_have_rows(kv, max_new, window):
    """Rows in front of a request's first token read nothing, whatever the window; the others read what there is."""
    for n, rows in ((5, 10), (1, 70), (40, 41), (1200, 1290)):
        m = Memory(kv, normal((n, 2, 64), 1), normal((n, 2, 64), 2), 16, "int8")
        q = torch.tensor(normal((rows + 2, 4, 64), 3)).half()
        positions = list(range(n - rows, n)) + [n - 2, n - 1]
        step = kv.KvStep(ints([m.order] * 2), offsets=ints([0, rows, rows + 2]), context=ints([n, n]), max_new=max_new)
        out, lse = m.cache.attend(q.cuda(), step, window=window)
        some = [t for t in range(rows + 2) if rows < 100 or t % 41 == 0 or t >= rows - 2]
        check_rows(m, q[some], out[some], lse[some], 11, [positions[t] for t in some],
                   lambda t, h: np.arange(max(0, positions[some[t]] - window + 1) if window else 0, positions[some[t]] + 1), 0.125)


@pytest.mark.parametrize("max_new", [1, 16, 20, 37, 300])
def test_a_step_with_fewer_rows_than_its_requests_have_tokens(kv, max_new):
    """The rows that there are stand where they stood."""
    n = 900
    m = Memory(kv, normal((n, 1, 64), 1), normal((n, 1, 64), 2), 16, "int8")
    q = torch.tensor(normal((37, 4, 64), 3)).half()
    step = kv.KvStep(ints([m.order] * 3), offsets=ints([0, 5, 70, 90]), context=ints([n, 500, 40]), max_new=max_new)
    out, lse = m.cache.attend(q.cuda(), step)
    positions = list(range(n - 5, n)) + list(range(500 - 65, 500 - 65 + 32))
    check_rows(m, q, out, lse, 11, positions, lambda t, h: np.arange(positions[t] + 1), 0.125)


@pytest.mark.parametrize("dim, new, heads", [(64, 100, 1), (128, 20, 5), (128, 1, 24), (128, 70, 4), (192, 25, 4), (192, 1, 3), (256, 100, 1), (256, 1, 30), (80, 40, 2)])
@pytest.mark.parametrize("softcap, slopes, window", [(0.0, False, 0), (20.0, True, 0), (500.0, False, 90)])
def test_values_far_apart_in_every_kernel(kv, dim, new, heads, softcap, slopes, window):
    """Rows of every width, in one tile, in two, by four waves and by eight: a few blocks of values of 2^40 to 2^120 among zeros and usual ones, with a cap, with slopes, with a window."""
    n = 1500
    rng = np.random.default_rng(dim + new)
    v = rng.standard_normal((n, 1, dim))
    for block in range(0, n, 16):
        v[block:block + 16] *= rng.choice([0.0, 1.0, 1.0, 1.0, 2.0 ** 40, 2.0 ** 120])
    for fmt in ("int8", "fp8"):
        m = Memory(kv, rng.standard_normal((n, 1, dim)), v, 48, fmt)
        slope = np.exp2(-8.0 * (1 + np.arange(heads)) / heads).astype(np.float32) if slopes else None
        q = torch.tensor(normal((new, heads, dim), 3)).to(torch.bfloat16)
        some = sorted({0, new // 2, new - 1})
        positions = np.arange(n - new, n)[some]
        step = kv.KvStep(ints([m.order]), offsets=ints([0, new]), context=ints([n]), max_new=new)
        out, lse = m.cache.attend(q.cuda(), step, softcap=softcap, window=window, slopes=None if slope is None else torch.tensor(slope).cuda())
        check_rows(m, q[some], out[some], lse[some], 8, positions, lambda t, h: np.arange(max(0, positions[t] - window + 1) if window else 0, positions[t] + 1),
                   dim ** -0.5, softcap, slope, slack=2.0 ** -18)


@pytest.mark.parametrize("max_new, n", [(1, 200), (1, 3000), (20, 200), (20, 3000), (300, 200), (300, 3000)])
def test_rows_before_the_first_request_are_zeros(kv, max_new, n):
    """offsets that begin behind row 0; in one workgroup and in shares, with few and with many rows."""
    m = Memory(kv, normal((n, 2, 64), 1), normal((n, 2, 64), 2), 16, "fp8")
    q = torch.tensor(normal((9, 4, 64), 3)).half()
    step = kv.KvStep(ints([m.order] * 2), offsets=ints([4, 5, 7]), context=ints([n, n - 3]), max_new=max_new)
    positions = [-1] * 4 + [n - 1, n - 5, n - 4] + [-1] * 2
    for _ in range(2):
        room = torch.full((1 << 22,), 1, dtype=torch.int32, device="cuda")      # what the workspace holds afterwards
        del room
        out, lse = m.cache.attend(q.cuda(), step, out=(torch.full((9, 4, 64), 7.0).half().cuda(), torch.full((9, 4), 7.0).cuda()))
        check_rows(m, q, out, lse, 11, positions, lambda t, h: np.arange(positions[t] + 1), 0.125)


CAPS = [65.0, 1e3, 1e4, 1e6, 1e30, 3e38]


@pytest.mark.parametrize("softcap", CAPS + [1e-3, 1e-30])
@pytest.mark.parametrize("dim, new", [(64, 1), (128, 40), (192, 3), (256, 33)])
def test_attend_with_any_cap(kv, softcap, dim, new):
    """A cap far above the scores leaves them as they are, to the rounding of a score; one far below makes all weights equal.  One row a
    key, two tiles of rows, the wide kernel; in one workgroup and in shares."""
    for n, fmt in ((300, "int8"), (2600, "fp8")):
        m = Memory(kv, normal((n, 1, dim), 1, 2.0), normal((n, 1, dim), 2), 64, fmt)
        q = torch.tensor(normal((new, 5, dim), 3)).half()
        step = kv.KvStep(ints([m.order]), offsets=ints([0, new]), context=ints([n]), max_new=new)
        out, lse = m.cache.attend(q.cuda(), step, softcap=softcap)
        some = sorted({0, new // 2, new - 1})
        positions = [n - new + t for t in some]
        check_rows(m, q[some], out[some], lse[some], 11, positions, lambda t, h: np.arange(positions[t] + 1), dim ** -0.5, softcap)


@pytest.mark.parametrize("softcap", CAPS + [1e-3, 1e-30])
def test_selected_with_any_cap(kv, softcap):
    m = Memory(kv, normal((400, 2, 96), 1, 2.0), normal((400, 2, 96), 2), 32, "int8")
    q = torch.tensor(normal((2, 6, 96), 3)).half()
    for k in (50, 2900):
        ids = np.random.default_rng(k).integers(0, 400, (2, 2, k))
        step = kv.KvStep(ints([m.order]), requests=ints([0, 0]), positions=ints([398, 399]))
        out, lse = m.cache.attend_selected(q.cuda(), torch.tensor(ids).cuda(), step, window=7, softcap=softcap)

        def keys_of(t, h):
            p, row = 398 + t, ids[t, h // 3]
            return np.concatenate([row[row <= p - 7], np.arange(p - 6, p + 1)])

        check_rows(m, q, out, lse, 11, [398, 399], keys_of, 96 ** -0.5, softcap)


def test_a_cap_of_nearly_nothing_and_keys_of_zeros(kv):
    """Scores of zero under a cap that 32 bits hardly hold."""
    m = Memory(kv, np.zeros((40, 1, 64)), normal((40, 1, 64), 2), 16, "int8")
    q = torch.tensor(normal((33, 4, 64), 3)).half()
    for new in (1, 33):
        step = kv.KvStep(ints([m.order]), offsets=ints([0, new]), context=ints([40]), requests=ints([0] * new), positions=ints(np.arange(40 - new, 40)))
        out, lse = m.cache.attend(q[:new].cuda(), step, softcap=1e-44)
        check_rows(m, q[:new], out, lse, 11, list(range(40 - new, 40)), lambda t, h: np.arange(40 - new + t + 1), 64 ** -0.5)
        ids = torch.arange(40).expand(new, 1, 40).contiguous().cuda()
        out, lse = m.cache.attend_selected(q[:new].cuda(), ids, step, softcap=1e-44)
        check_rows(m, q[:new], out, lse, 11, list(range(40 - new, 40)), lambda t, h: np.arange(40 - new + t + 1), 64 ** -0.5)


@pytest.mark.parametrize("page, position", [(16, 5000), (64, 300_000), (1 << 20, 5_000_000), (1 << 20, 1_000_000_000)])
@pytest.mark.parametrize("softcap", [0.0, 30.0])
def test_selected_far_away_with_slopes(kv, page, position, softcap):
    """A list of tokens that all lie far from the one that reads them, without a window: their distances' differences decide, and these are small
    numbers.  Slopes up to where slope * distance is some 10^8."""
    n, dim, heads = 300, 64, 4
    m = Memory(kv, normal((n, 1, dim), 1), normal((n, 1, dim), 2), page, "int8")
    table = np.full((1, position // page + 1), -1)
    table[0, :len(m.order)] = m.order
    slopes = np.array([1.0, 0.25, 0.1, 0.003], np.float32) * min(1.0, 1e8 / position)
    q = torch.tensor(normal((1, heads, dim), 3)).half()
    for k in (1, 33, 300, 3000):
        ids = np.random.default_rng(k).integers(0, n, (1, 1, k))
        step = kv.KvStep(ints(table), requests=ints([0]), positions=ints([position]))
        out, lse = m.cache.attend_selected(q.cuda(), torch.tensor(ids).cuda(), step, slopes=torch.tensor(slopes).cuda(), softcap=softcap)
        check_rows(m, q, out, lse, 11, [position], lambda t, h: ids[0, 0], dim ** -0.5, softcap, slopes)


FINITE = 255.0 * 2.0 ** 120      # the largest finite bf16


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_the_largest_numbers_stay_finite(kv, fmt):
    """A block whose largest magnitude lies near the end of 32 bits is rounded up to 2^128: what is read back, and attention's mean of it, ends at
    the largest number that 16 bits of bf16 hold."""
    top = float(torch.finfo(torch.float32).max)
    for big, new in ((top, 1), (FINITE, 1), (math.inf, 1), (top, 40), (FINITE, 300)):
        n = max(3000 if new == 1 else 40, new)
        v = normal((n, 1, 64), 2)
        v[::3] = np.where(np.arange(64) % 2, big, -big)
        v[1::3] = np.where(np.arange(64) % 4 < 2, top, -top)
        k = torch.tensor(normal((n, 1, 64), 1))
        cache = kv.KvCache(-(-n // 16), 1, 64, 16, fmt)
        slots = torch.arange(n).cuda()
        cache.append(k.float().cuda(), torch.tensor(v).float().cuda(), slots)
        numbers = plain.numbers(cache.data.cpu().numpy(), cache.exponents.cpu().numpy(), 64, fmt).reshape(-1, 16, 2, 64).reshape(-1, 2, 64)[:n]
        assert np.abs(numbers[:, 1]).max() >= 2.0 ** 128
        held = np.clip(numbers, -FINITE, FINITE)
        for dtype in (torch.float32, torch.bfloat16):
            got = cache.read(slots, dtype=dtype)
            assert (wide(got[0][:, 0]) == numbers[:, 0]).all() and (wide(got[1][:, 0]) == held[:, 1]).all()
        q = torch.tensor(normal((new, 2, 64), 3)).to(torch.bfloat16)
        positions = np.arange(n - new, n)
        step = kv.KvStep(ints([np.arange(-(-n // 16))]), offsets=ints([0, new]), context=ints([n]), requests=ints([0] * new), positions=ints(positions), max_new=new)
        one = torch.full((new, 1, 1), 3, dtype=torch.int64).cuda()
        for (out, lse), keys in ((cache.attend(q.cuda(), step), None), (cache.attend(q.cuda(), step, window=1), 1), (cache.attend_selected(q.cuda(), one, step), 3)):
            for t in range(0, new, 13):
                p = positions[t]
                at = np.arange(p + 1) if keys is None else np.array([p]) if keys == 1 else np.array([3] if p >= 3 else [], int)
                for h in range(2):
                    o, l, spread, products = plain.attend_row(wide(q[t, h]), numbers[at, 0], numbers[at, 1], 0.125)
                    tol_o, tol_l = plain.tolerance(64, 8, o, spread, products)
                    assert (np.abs(wide(out[t, h]) - np.clip(o, -FINITE, FINITE)) <= tol_o).all() and (l == lse[t, h] or abs(float(lse[t, h]) - l) <= tol_l)


@pytest.mark.parametrize("new, heads", [(1, 2), (1, 20), (40, 4), (300, 2)])
@pytest.mark.parametrize("n", [160, 3200])
def test_values_whose_exponents_are_as_far_apart_as_they_can_be(kv, new, heads, n):
    """The sum of the weights is that of all keys, whatever their values' sizes: zeros beside numbers near the end of 32 bits, in any order, in one wave's
    tiles, in several waves' and in several workgroups'.  A weight that is less than 2^-31 of the row's largest times its block's scale is lost from
    the values' sum, as a 16-bit float cannot hold it."""
    dim, n = 64, max(n, new + 20)
    for seed in range(3):
        rng = np.random.default_rng(seed)
        v = rng.standard_normal((n, 1, dim))
        for block in range(0, n, 16):
            v[block:block + 16] *= [0.0, 2.0 ** -80, 1.0, 2.0 ** 40, 2.0 ** 90, 2.0 ** 120][rng.integers(0, 6) if seed else min(5, block * 6 // n)]
        for fmt in ("int8", "fp8"):
            m = Memory(kv, rng.standard_normal((n, 1, dim)), v, 32, fmt)
            q = torch.tensor(normal((new, heads, dim), 3)).to(torch.bfloat16)
            positions = np.arange(n - new, n)
            step = kv.KvStep(ints([m.order]), offsets=ints([0, new]), context=ints([n]), requests=ints([0] * new), positions=ints(positions), max_new=new)
            some = sorted({0, new // 2, new - 1})
            out, lse = m.cache.attend(q.cuda(), step)
            check_rows(m, q[some], out[some], lse[some], 8, positions[some], lambda t, h: np.arange(positions[some][t] + 1), dim ** -0.5, slack=2.0 ** -18)
            ids = rng.integers(0, n - new + 1, (new, 1, 200))
            out, lse = m.cache.attend_selected(q.cuda(), torch.tensor(ids).cuda(), step, window=0)
            check_rows(m, q[some], out[some], lse[some], 8, positions[some], lambda t, h: ids[some][t, 0], dim ** -0.5, slack=2.0 ** -18)


def test_calls_on_tensors_that_require_a_gradient_are_refused(kv):
    cache, tables = kv.KvCache(4, 2, 64, 16), kv.KvTables(1, 4, 4, 16)
    step = tables.extend(ints([3]), 3)
    x, q = torch.randn(3, 2, 64, device="cuda").half(), torch.randn(3, 4, 64, device="cuda").half()
    ids = torch.zeros(3, 2, 2, dtype=torch.int64, device="cuda")
    slopes = torch.ones(4, device="cuda", requires_grad=True)
    asks = lambda t: t.clone().requires_grad_()
    for call in (lambda: cache.append(asks(x), x, step.slots), lambda: cache.append(x, asks(x), step.slots), lambda: cache.attend(asks(q), step),
                 lambda: cache.attend_selected(asks(q), ids, step), lambda: cache.attend(q, step, slopes=slopes)):
        with pytest.raises(kv.PagError, match="gradient"):
            call()
        with torch.no_grad():
            call()


# ---- layouts --------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("max_new", [1, 20, 300])
@pytest.mark.parametrize("n", [150, 3000])
def test_strided_rows_and_tables(kv, max_new, n):
    """q and out that are slices of larger arrays, heads before tokens; a table that is a slice of a wider one.  Bit for bit what dense ones give."""
    m = Memory(kv, normal((n, 2, 64), 1), normal((n, 2, 64), 2), 32, "int8")
    heads, tokens = 6, 9
    dense = torch.tensor(normal((tokens, heads, 64), 3)).half().cuda()
    news, contexts = [4, 0, 5], [n, 0, n - 7]
    positions = list(range(n - 4, n)) + list(range(n - 12, n - 7))
    wide_table = torch.full((3, len(m.order) + 5), 1 << 30, dtype=torch.int32, device="cuda")
    wide_table[:, 2:-3] = ints([m.order] * 3)
    arrays = dict(offsets=ints([0, 4, 4, 9]), context=ints(contexts), requests=ints([0] * 4 + [2] * 5), positions=ints(positions), max_new=max_new)
    ids = torch.randint(0, n - 20, (tokens, 2, 40), generator=torch.Generator().manual_seed(1)).cuda()
    wide_ids = torch.full((2, tokens, 50), 5, dtype=torch.int64, device="cuda")
    wide_ids[:, :, 3:43] = ids.transpose(0, 1)
    one, two = kv.KvStep(ints([m.order] * 3), **arrays), kv.KvStep(wide_table[:, 2:-3], **arrays)
    want = m.cache.attend(dense, one), m.cache.attend_selected(dense, ids, one, window=5)
    check_rows(m, dense, *want[0], 11, positions, lambda t, h: np.arange(positions[t] + 1), 0.125)
    some = ids.cpu().numpy()
    check_rows(m, dense, *want[1], 11, positions, lambda t, h: np.concatenate([some[t, h // 3], np.arange(positions[t] - 4, positions[t] + 1)]), 0.125)
    fused = torch.full((tokens, 3 * heads, 80), 9.0, dtype=torch.float16, device="cuda")
    by_head = torch.full((heads, tokens, 64), 9.0, dtype=torch.float16, device="cuda")
    fused[:, heads:2 * heads, 8:72] = dense
    by_head.copy_(dense.transpose(0, 1))
    for q in (fused[:, heads:2 * heads, 8:72], by_head.transpose(0, 1)):
        rest = torch.full((tokens, 2 * heads, 72), 7.0, dtype=torch.float16, device="cuda")
        heads_first = torch.full((heads + 1, tokens, 64), 7.0, dtype=torch.float16, device="cuda")
        for out in (rest[:, heads:, :64], heads_first[1:].transpose(0, 1)):
            got = m.cache.attend(q, two, out=(out, None))
            assert got[0] is out and torch.equal(out, want[0][0])
            out.fill_(7.0)
            lse = torch.empty(tokens, heads, device="cuda")
            m.cache.attend_selected(q, wide_ids[:, :, 3:43].transpose(0, 1), two, window=5, out=(out, lse))
            assert torch.equal(out, want[1][0]) and torch.equal(lse, want[1][1])
        assert (rest[:, :heads] == 7.0).all() and (rest[:, :, 64:] == 7.0).all() and (heads_first[0] == 7.0).all()


@pytest.mark.parametrize("id_heads, k, window", [(2, 40, 0), (2, 40, 5), (6, 7, 30), (2, 3000, 64)])
def test_selected_of_several_tokens_of_a_request(kv, id_heads, k, window):
    """Each of a request's new tokens has a list and a window of its own; lists may name tokens that are new themselves."""
    n = 3100 if k > 1000 else 260
    m = Memory(kv, normal((n, 2, 64), 1), normal((n, 2, 64), 2), 16, "fp8")
    news, ends = [5, 1, 17], [n, 100, n - 50]
    requests = [r for r, a in enumerate(news) for _ in range(a)]
    positions = [p for a, e in zip(news, ends) for p in range(e - a, e)]
    rng = np.random.default_rng(k)
    ids = rng.integers(-1, n, (len(positions), id_heads, k))
    for t, p in enumerate(positions):
        ids[t, :, ::3] = rng.integers(max(0, p - 60), p + 3, ids[t, :, ::3].shape)
    q = torch.tensor(normal((len(positions), 6, 64), 3)).to(torch.bfloat16)
    step = kv.KvStep(ints([m.order] * 3), requests=ints(requests), positions=ints(positions))
    out, lse = m.cache.attend_selected(q.cuda(), torch.tensor(ids).cuda(), step, window=window)

    def keys_of(t, h):
        p, row = positions[t], ids[t, h * id_heads // 6]
        return np.concatenate([row[(row >= 0) & (row <= p - window)], np.arange(max(0, p - window + 1), p + 1)]).astype(int)

    check_rows(m, q, out, lse, 8, positions, keys_of, 0.125)


# ---- pages that come back -------------------------------------------------------------------------------------------------------


def test_release_of_long_requests(kv):
    """Thousands of pages of one request, and requests of one page on both sides of it."""
    tables = kv.KvTables(5, 7000, 9000, 16)
    add = [3, 6250 * 16, 0, 1500 * 16 + 1, 16]
    tables.commit(tables.extend(ints(add), sum(add)))
    table, count = tables.table.cpu().numpy(), int(tables.free_count)
    assert count == 9000 - (1 + 6250 + 1501 + 1) and sorted(table[table >= 0].tolist()) == list(range(9000 - count))
    free = tables.free_pages[:count].tolist()
    tables.release(ints([0, 1, 1, 1, 0]))
    free += table[1, :6250].tolist() + table[3, :1501].tolist()
    assert tables.lengths.tolist() == [3, 0, 0, 0, 16] and tables.free_pages[:int(tables.free_count)].tolist() == free


def test_release_onto_a_stack_without_room(kv):
    """Pages for which the stack has no room are not put anywhere."""
    lengths, table, free = ints([40, 16, 0]), ints([[7, 8, 9], [5, -1, -1], [1, 2, 3]]), ints([11, 12, 13, 99])
    guard = torch.full((12,), -7, dtype=torch.int32, device="cuda")
    guard[4:8] = free
    tables = kv.KvTables.from_tensors(lengths, table, guard[4:8], ints([2]), 16)
    tables.release(ints([1, 1, 1]))
    assert guard.tolist() == [-7] * 4 + [11, 12, 7, 8] + [-7] * 4 and tables.free_count.tolist() == [4] and tables.lengths.tolist() == [0, 0, 0]
