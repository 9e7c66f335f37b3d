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
