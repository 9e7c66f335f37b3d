"""Attention over the 4-bit cache against a plain implementation in 64 bits.  Codes times their scale, as multiples of the largest power of two among 16
tokens, are 16-bit floats exactly (down to 2^-22 of it), so the tolerances are those of the 8-bit cache."""
import math

import numpy as np
import pytest

import kv_more_plain as more
import kv_plain as plain
import test_gpu_kv as base
from test_gpu_kv import DTYPES, check_attention, ints, kv, wide  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


class Memory(base.Memory):
    """base.Memory for any format."""

    def __init__(self, kv, contexts, kv_heads, dim, page, fmt, seed, spread=1.0):
        rng = np.random.default_rng(seed)
        counts = [-(-c // page) for c in contexts]
        self.pages = sum(counts) + 2
        order = rng.permutation(self.pages)
        self.table = np.full((len(contexts), max(counts + [1]) + 1), -1)
        self.page, self.fmt, self.dim, self.kv_heads, self.contexts = page, fmt, dim, kv_heads, contexts
        data_shape, exponent_shape = more.shapes(self.pages, kv_heads, page, dim, fmt)
        data, exponents = np.full(data_shape, 0x7F, np.uint8), np.full(exponent_shape, 127, np.int8)
        bytes_ = dim // 2 if fmt == "fp4" else dim
        data[..., bytes_:] = 0
        first = 0
        for b, (c, n) in enumerate(zip(contexts, counts)):
            self.table[b, :n] = order[first:first + n]
            first += n
            at = np.arange(c)
            slots = self.table[b, at // page] * page + at % page
            x = rng.standard_normal((2, c, kv_heads, dim)) * spread * 2.0 ** rng.integers(-1, 2, (2, 1, kv_heads, 1))
            x[0, ..., :: 16] *= 3
            more.append(data, exponents, dim, fmt, x[0], x[1], slots)
            if c % 16 and fmt != "fp4":
                data[self.table[b, n - 1], :, c % page:, :, :dim] = 0x7F
        self.numbers = more.numbers(data, np.minimum(exponents, 100), dim, fmt)
        self.cache = kv.KvCache.from_tensors(torch.tensor(data).cuda(), torch.tensor(exponents).cuda(), dim, fmt)


@pytest.fixture(autouse=True)
def any_format(monkeypatch):
    monkeypatch.setattr(base, "Memory", Memory)


attend_case, selected_case = base.attend_case, base.selected_case


@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attend_one_token_each(kv, dim, dtype):
    contexts = [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 300, 1000]
    attend_case(kv, contexts, [1] * len(contexts), 8, 2, dim, 32, "fp4", dtype)


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 1), (17, 1), (40, 1), (12, 4), (64, 2)])
@pytest.mark.parametrize("page", [16, 48, 128])
def test_attend_groups_and_pages(kv, heads, kv_heads, page):
    attend_case(kv, [5, 70, 333], [1, 1, 1], heads, kv_heads, 64, page, "fp4", "fp16")


@pytest.mark.parametrize("dim, heads, kv_heads, dtype", [(64, 4, 4, "bf16"), (128, 8, 2, "fp16"), (96, 6, 2, "bf16"), (192, 2, 1, "fp16"), (256, 16, 2, "bf16")])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_attend_chunks(kv, dim, heads, kv_heads, dtype, window):
    attend_case(kv, [1, 40, 70, 37, 200, 130], [1, 40, 3, 0, 17, 33], heads, kv_heads, dim, 16, "fp4", dtype, window=window, pad=3)


@pytest.mark.parametrize("softcap, slopes, window", [(30.0, False, 0), (0.0, True, 0), (2.0, True, 50), (500.0, False, 7)])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [20, 1, 60, 90]])
def test_attend_cap_and_distance(kv, softcap, slopes, window, news):
    attend_case(kv, [33, 1, 200, 90], news, 6, 2, 128, 32, "fp4", "bf16", window=window, softcap=softcap, slopes=slopes)


def test_attend_pieces_of_several_units(kv):
    attend_case(kv, [9000, 5000, 10_011], [1, 2, 1], 8, 4, 64, 64, "fp4", "fp16")
    attend_case(kv, [3000, 2000, 2011], [40, 70, 100], 8, 4, 64, 64, "fp4", "fp16")


@pytest.mark.parametrize("dim, softcap, slopes, window", [(136, 0.0, False, 0), (192, 30.0, False, 0), (192, 0.0, True, 7000), (248, 0.0, False, 0)])
def test_attend_pieces_of_wide_rows(kv, dim, softcap, slopes, window):
    attend_case(kv, [9000, 100, 10_011], [1, 2, 1], 4, 2, dim, 64, "fp4", "fp16", softcap=softcap, slopes=slopes, window=window)


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
def test_attend_two_tiles_of_rows_in_pieces(kv, dim):
    attend_case(kv, [4100, 2300, 900], [1, 2, 0], 20, 1, dim, 64, "fp4", "bf16")
    attend_case(kv, [3000, 40], [8, 8], 8, 1, dim, 64, "fp4", "fp16", window=2500, softcap=20.0)


@pytest.mark.parametrize("dim", [40, 128])
@pytest.mark.parametrize("softcap, slopes, window", [(0.0, False, 0), (30.0, False, 0), (0.0, True, 90), (5.0, True, 0)])
def test_attend_long_chunks(kv, dim, softcap, slopes, window):
    attend_case(kv, [400, 33, 0, 150], [300, 33, 0, 1], 2, 1, dim, 32, "fp4", "fp16", softcap=softcap, slopes=slopes, window=window, pad=2)


@pytest.mark.parametrize("max_new", [0, 1, 4, 16, 37, 300])
def test_attend_with_any_hint(kv, max_new):
    attend_case(kv, [2900, 40, 700], [37, 5, 1], 4, 1, 64, 64, "fp4", "fp16", max_new=max_new)


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("k, window", [(1, 0), (10, 1), (33, 16), (100, 64), (300, 0)])
def test_selected(kv, dim, k, window):
    selected_case(kv, [300, 1, 40, 130, 64, 17], 4, 2, 2, dim, k, window, "fp4", "bf16" if k % 2 else "fp16")


@pytest.mark.parametrize("heads, kv_heads, id_heads", [(1, 1, 1), (8, 2, 8), (8, 2, 4), (40, 2, 2), (12, 4, 12)])
def test_selected_heads(kv, heads, kv_heads, id_heads):
    selected_case(kv, [200, 90, 513, 33, 50], heads, kv_heads, id_heads, 64, 70, 20, "fp4", "fp16", pad=2, softcap=20.0, slopes=True)


@pytest.mark.parametrize("tokens, k, window, slopes", [(3, 1200, 300, False), (5, 2600, 64, True), (17, 2600, 64, False)])
def test_selected_longer_lists(kv, tokens, k, window, slopes):
    selected_case(kv, [3000 - 7 * i for i in range(tokens)], 16, 1, 16, 64, k, window, "fp4", "fp16", page=64, slopes=slopes)


def test_attend_pages_that_do_not_exist(kv):
    m = Memory(kv, [64, 40], 1, 64, 16, "fp4", 4)
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


@pytest.mark.parametrize("max_new, n", [(1, 1), (20, 4), (300, 40)])
@pytest.mark.parametrize("dim", [64, 192])
def test_values_and_keys_of_very_different_parts(kv, max_new, n, dim):
    """Exponents far apart from part to part and from token to token, up to numbers of 2^40: scores stay moderate (a part that is large meets zeros of q).  What lies below
    2^-24 of the largest part of 16 tokens may be lost from a number: keys and values are off by half of that, 2^-25 of the block's largest."""
    page, heads, context = 16, 2, 300
    rng = np.random.default_rng(dim + n)
    pages = -(-context // page)
    cache = kv.KvCache(pages, 1, dim, page, "fp4")
    data_shape, exponent_shape = more.shapes(pages, 1, page, dim, "fp4")
    data, exponents = np.zeros(data_shape, np.uint8), np.zeros(exponent_shape, np.int8)
    k, v = rng.standard_normal((context, 1, dim)), rng.standard_normal((context, 1, dim))
    k[:, :, 32:64] *= 2.0 ** rng.integers(0, 16, (context, 1, 1))          # q has zeros there
    v[:, :, :32] *= 2.0 ** rng.integers(-12, 12, (context, 1, 1))
    v[40:50] *= 2.0 ** 18
    k, v = (torch.tensor(x).float() for x in (k, v))
    slots = np.arange(context)
    cache.append(k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    more.append(data, exponents, dim, "fp4", wide(k), wide(v), slots)
    numbers = more.numbers(data, exponents, dim, "fp4")
    rows = numbers[slots // page, 0, slots % page]
    q = torch.tensor(rng.standard_normal((n, heads, dim))).to(torch.bfloat16)
    q[..., 32:64] = 0
    step = kv.KvStep(ints(np.arange(pages)[None]), offsets=ints([0, n]), context=ints([context]), max_new=max_new)
    out, lse = cache.attend(q.cuda(), step)
    for t in range(n):
        for h in range(heads):
            at = np.arange(context - n + t + 1)
            o, l, spread, products = plain.attend_row(wide(q[t, h]), rows[at, 0], rows[at, 1], dim ** -0.5)
            # largest |value| and |key| of any block of 16
            lost = 2.0 ** -25 * np.abs(rows[at, 0]).max() * np.abs(wide(q[t, h])).sum() * dim ** -0.5
            tol_o, tol_l = plain.tolerance(dim, 8, o, spread, products + lost * 2.0 ** 24 / dim)
            # a weight below 2^-31 of the largest times its block's scale is lost, of which there are `context`
            tol_o = tol_o + 2.0 ** -25 * np.abs(rows[at, 1]).max() + context * 2.0 ** -31 * np.abs(rows[at, 1]).max()
            assert abs(float(lse[t, h]) - l) <= tol_l + lost, (t, h)
            assert (np.abs(wide(out[t, h]) - o) <= tol_o).all(), (t, h)


@pytest.mark.parametrize("max_new, n, heads", [(1, 1, 1), (20, 4, 8), (300, 40, 1)])
def test_values_far_up_and_the_sum_of_weights(kv, max_new, n, heads):
    """Values of 2^100 in one block and of 1 and 0 in the others: the weights' sum is that of all keys, and what comes out stays finite."""
    dim, page, context = 64, 16, 200
    rng = np.random.default_rng(n)
    pages = -(-context // page)
    cache = kv.KvCache(pages, 1, dim, page, "fp4")
    data_shape, exponent_shape = more.shapes(pages, 1, page, dim, "fp4")
    data, exponents = np.zeros(data_shape, np.uint8), np.zeros(exponent_shape, np.int8)
    k, v = torch.tensor(rng.standard_normal((context, 1, dim))).float(), torch.tensor(rng.standard_normal((context, 1, dim))).float()
    v[64:80] *= 2.0 ** 100
    v[90:100] = 0.0
    slots = np.arange(context)
    cache.append(k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    more.append(data, exponents, dim, "fp4", wide(k), wide(v), slots)
    rows = more.numbers(data, exponents, dim, "fp4")[slots // page, 0, slots % page]
    q = torch.tensor(rng.standard_normal((n, heads, dim))).to(torch.bfloat16)
    step = kv.KvStep(ints(np.arange(pages)[None]), offsets=ints([0, n]), context=ints([context]), requests=ints([0] * n),
                     positions=ints(np.arange(context - n, context)), max_new=max_new)
    ids = torch.arange(context, device="cuda").expand(n, 1, context).contiguous()
    for out, lse in (cache.attend(q.cuda(), step), cache.attend_selected(q.cuda(), ids, step)):
        for t in range(n):
            for h in range(heads):
                at = np.arange(context - n + t + 1)
                o, l, spread, products = plain.attend_row(wide(q[t, h]), rows[at, 0], rows[at, 1], dim ** -0.5)
                tol_o, tol_l = plain.tolerance(dim, 8, o, spread, products)
                assert abs(float(lse[t, h]) - l) <= tol_l and (np.abs(wide(out[t, h]) - o) <= tol_o + 2.0 ** -24 * np.abs(rows[at, 1]).max()).all()


def test_rows_beyond_32_bits_of_offset(kv):
    """A cache of 5 GB: pages whose bytes lie behind the first 4 GB."""
    pages, heads, page, dim = 5 * (1 << 30) // (2 * 64 * 128), 2, 64, 128
    cache = kv.KvCache.from_tensors(torch.empty((pages, heads, page, 2, dim // 2), dtype=torch.uint8, device="cuda"),
                                    torch.empty((pages, heads, page // 16, 2, dim // 32, 16), dtype=torch.int8, device="cuda"), dim, "fp4")
    order = np.array([pages - 1, 3, pages - 70, pages // 2])
    at = np.arange(250)
    slots = torch.tensor(order[at // page] * page + at % page).cuda()
    k, v = torch.randn(250, heads, dim, device="cuda"), torch.randn(250, heads, dim, device="cuda")
    cache.append(k, v, slots)
    small = kv.KvCache(4, heads, dim, page, "fp4")
    small.append(k, v, torch.tensor(at).cuda())
    for x, y in zip(cache.read(slots), small.read(torch.tensor(at).cuda())):
        assert torch.equal(x, y)
    q = torch.randn(1, 4, dim, device="cuda").half()
    ids = torch.tensor([249, 0, 100, 64, 63, 128, -1]).cuda().view(1, 1, -1).expand(1, 2, 7)
    a, b = kv.KvStep(ints([order]), ints([0, 1]), ints([250]), ints([0]), ints([249])), kv.KvStep(ints([[0, 1, 2, 3]]), ints([0, 1]), ints([250]), ints([0]), ints([249]))
    assert all(torch.equal(x, y) for x, y in zip(cache.attend(q, a), small.attend(q, b)))
    assert all(torch.equal(x, y) for x, y in zip(cache.attend_selected(q, ids, a), small.attend_selected(q, ids, b)))


@pytest.mark.parametrize("max_new, n", [(1, 1), (20, 4), (300, 40)])
def test_the_largest_numbers_stay_finite(kv, max_new, n):
    """Values of 3e38 are held as 4 * 2^126, which is read, and averaged, as the largest finite bf16; averages of them and their negatives are finite."""
    dim, page, context = 64, 16, 100
    cache = kv.KvCache(7, 1, dim, page, "fp4")
    k, v = torch.randn(context, 1, dim, device="cuda"), torch.full((context, 1, dim), 3.0e38, device="cuda")
    v[:, :, 1::2] *= -1
    v[::2, :, 32:] *= -1
    slots = torch.arange(context, device="cuda")
    cache.append(k, v, slots)
    step = kv.KvStep(ints([[0, 1, 2, 3, 4, 5, 6]]), ints([0, n]), ints([context]), ints([0] * n), ints(range(context - n, context)), max_new=max_new)
    q = torch.randn(n, 2, dim, device="cuda").to(torch.bfloat16)
    ids = slots.expand(n, 1, context).contiguous()
    for out, lse in (cache.attend(q, step), cache.attend_selected(q, ids, step)):
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        assert (out[..., 0:32:2] == 255.0 * 2.0 ** 120).all() and (out[..., 1:32:2] == -255.0 * 2.0 ** 120).all()


def test_rows_with_infinities_and_nan_spoil_only_themselves(kv):
    m = Memory(kv, [50, 90], 2, 64, 32, "fp4", 4)
    q = torch.randn(4, 4, 64).half()
    step = kv.KvStep(ints(m.table), offsets=ints([0, 2, 4]), context=ints([50, 90]), requests=ints([0, 0, 1, 1]), positions=ints([48, 49, 88, 89]))
    ids = ints(np.tile(np.arange(3), (4, 2, 1)))
    blocks = kv.KvBlocks(m.cache, 16)
    clean = m.cache.attend(q.cuda(), step), blocks.attend(q.cuda(), ids, step, window=9)
    q[0, 1, 5], q[3, 2, 0], q[2, 0, 7] = math.nan, math.inf, -math.inf
    spoilt = torch.zeros(4, 4, dtype=torch.bool)
    spoilt[0, 1] = spoilt[3, 2] = spoilt[2, 0] = True
    for (out, lse), before in zip((m.cache.attend(q.cuda(), step), blocks.attend(q.cuda(), ids, step, window=9)), clean):
        assert torch.isnan(out.cpu()[spoilt]).all()
        assert torch.equal(out.cpu()[~spoilt], before[0].cpu()[~spoilt]) and torch.equal(lse.cpu()[~spoilt], before[1].cpu()[~spoilt])


def test_the_example_in_4_bits():
    """It runs, reads what was found and the window, and its share of the weight is a share."""
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("searched_memory", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "searched_memory.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    share, error = example.run(3000, 5, "fp4")
    assert 0.0 < share <= 1.0 + 2.0 ** -10 and math.isfinite(error)
