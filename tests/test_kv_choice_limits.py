"""Choices among blocks of calls up to the limits that the header names: a bounded workspace, and the same lists whether a call's tokens go in one launch or several."""
import ctypes as C

import numpy as np
import pytest
from test_kv_abi import _attention, _cache, _step, kv  # noqa: F401

torch = pytest.importorskip("torch")


def room(kv, tokens, heads, kv_heads, id_heads, blocks):
    """-> status, workspace of a choice among `blocks` blocks of 16 tokens that a request's row of the table has room for."""
    lib, size, pages = kv.load_library(), C.c_uint64(77), blocks // 2
    cache, step = _cache(kv, kv_heads=kv_heads), _step(kv, max_pages=pages, table_stride=pages, tokens=tokens)
    rc = lib.pag_kv_blocks_workspace_bytes(C.byref(cache), C.byref(step), C.byref(_attention(kv, heads=heads)), C.c_uint32(id_heads), C.c_uint32(4), C.c_uint32(16),
                                           C.byref(size), None)
    return rc, size.value


@pytest.mark.parametrize("tokens, heads, kv_heads, id_heads, blocks", [
    (40_000, 64, 8, 64, 4000), (65_536, 64, 1, 2, 65_536), (8192, 64, 8, 64, 4000), (4096, 32, 8, 32, 8192), ((1 << 23) - 1, 1, 1, 1, 2), ((1 << 23) - 1, 1, 1, 1, 1 << 16),
    ((1 << 17) - 1, 64, 64, 64, 2000), (100, 65_536, 4096, 65_536, 16)])
def test_a_choice_within_the_limits_has_a_bounded_workspace(kv, tokens, heads, kv_heads, id_heads, blocks):
    """tokens * heads below 2^23, tokens * id_heads * blocks up to 2^40: 512 MB."""
    assert tokens * heads < 1 << 23 and tokens * id_heads * blocks <= 1 << 40
    rc, size = room(kv, tokens, heads, kv_heads, id_heads, blocks)
    assert rc == 0 and size <= 512 << 20


def test_a_workspace_holds_one_tokens_scores_at_least(kv):
    assert room(kv, 5, 32, 8, 32, 1 << 23) == (0, 4 * 32 << 23)
    # and as many tokens as fit, in launches of about as many tokens each: 512 would fit, 4 launches of 500
    assert room(kv, 2000, 32, 8, 32, 8192) == (0, 4 * 32 * 8192 * 500)


@pytest.mark.parametrize("tokens, heads, kv_heads, id_heads, blocks, word", [
    (1 << 18, 4, 2, 2, 1 << 23, b"2^40"), (1 << 23, 1, 1, 1, 2, b"2^23"), (1, 64, 64, 64, 1 << 26, b"2^24")])
def test_a_choice_beyond_them_is_refused(kv, tokens, heads, kv_heads, id_heads, blocks, word):
    rc, size = room(kv, tokens, heads, kv_heads, id_heads, blocks)
    assert rc == -5 and size == 77 and word in kv.load_library().pag_last_error()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def lists_in_parts(kv, dim, heads, kv_heads, id_heads, n, width, k, some, block=16):
    """The lists of n tokens in one call, against those of `some` of them one at a time; a table with room for `width` blocks."""
    page, context = 64, 3300
    m, rng = -(-context // page), np.random.default_rng(n)
    cache = kv.KvCache(2 * m, kv_heads, dim, page)
    blocks = kv.KvBlocks(cache, block)
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(2 * m * page, kv_heads, dim, device="cuda", generator=gen)
    cache.append(x, x, torch.arange(2 * m * page, device="cuda"))
    blocks.update(torch.arange(2 * m * page, device="cuda"))
    table = np.full((2, width * block // page), -1)
    table[0, :m], table[1, :m] = rng.permutation(2 * m).reshape(2, m)
    requests, positions = rng.integers(0, 2, n), rng.integers(-1, context, n)
    q = torch.randn(n, heads, dim, device="cuda", dtype=torch.float16, generator=gen)
    out = torch.full((n, id_heads, k + 1), 77, dtype=torch.int32, device="cuda")
    got = blocks.select(q, kv.KvStep(ints(table), requests=ints(requests), positions=ints(positions)), k, window=20, id_heads=id_heads, out=out[..., :k])
    assert bool((out[..., k] == 77).all())
    for t in some:
        one = blocks.select(q[t:t + 1], kv.KvStep(ints(table[:, :m]), requests=ints(requests[t:t + 1]), positions=ints(positions[t:t + 1])), k, window=20, id_heads=id_heads)
        assert torch.equal(got[t:t + 1], one), t
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("dim, heads, kv_heads, id_heads, width, k", [(64, 8, 2, 4, 20_000, 20), (128, 40, 1, 2, 40_000, 70), (64, 4, 2, 4, 12_000, 5), (64, 4, 2, 2, 9000, 300)])
def test_tokens_that_go_in_several_launches(kv, dim, heads, kv_heads, id_heads, width, k):
    n = 10_001
    got = lists_in_parts(kv, dim, heads, kv_heads, id_heads, n, width, k, sorted({0, 1, n - 1, *range(0, n, 97)}))
    assert bool((got >= -1).all()) and bool((got < 3300 // 16 + 1).all())


@pytest.mark.gpu
def test_a_call_that_no_single_launch_has_threads_for(kv):
    """65,536 tokens over a table with room for 65,536 blocks."""
    lists_in_parts(kv, 8, 64, 1, 2, 65_536, 65_536, 4, [0, 1, 255, 256, 8191, 30_000, 65_535])


@pytest.mark.gpu
def test_several_launches_in_a_graph(kv):
    """Every replay against the same call without a graph."""
    n, heads, page, held = 6000, 8, 64, 30
    cache = kv.KvCache(held, 1, 64, page)
    blocks = kv.KvBlocks(cache, 16)
    x, at = torch.randn(held * page, 1, 64, device="cuda"), torch.arange(held * page, device="cuda")
    cache.append(x, x, at)
    blocks.update(at)
    table = np.full((1, 4000), -1)
    table[0, :held] = np.arange(held)
    step = kv.KvStep(ints(table), requests=ints([0] * n), positions=torch.randint(0, held * page, (n,), dtype=torch.int32, device="cuda"))
    q = torch.randn(n, heads, 64, device="cuda").half()
    assert 4 * heads * 16_000 * n > 512 << 20
    select = lambda: blocks.select(q, step, 9, window=5, id_heads=heads)
    select()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = select()
    for _ in range(4):
        q.copy_(torch.randn(q.shape))
        step.positions.copy_(torch.randint(0, held * page, (n,), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = select()
        torch.cuda.synchronize()
        assert torch.equal(captured, want) and bool((captured[:, :, 0] >= -1).all())
