"""Attention over the 4-bit cache where every token and every part of its row counts: each row of q has a token of its own, which gets nearly all of its weight, so that what comes
out is that token's values, whose powers of two lie up to 2^18 apart from part to part and from token to token.  The tolerances are of the row's own numbers: of each block's weights,
values and powers of two, not of the memory's largest number; on the CPU they are shown to see one part's power of two that is off by one, and one block that is left out."""
import numpy as np
import pytest

import kv_more_plain as more
import kv_plain as plain
from test_kv_abi import kv  # noqa: F401

torch = pytest.importorskip("torch")

CONTEXT, TARGETS, PAGE = 600, 128, 16
DIMS = [64, 80, 128, 192, 256]


def apart(rng, dim):
    """128 rows of signs times a power of two for each part, and the rows that meet each of them evenly, so that none meets another one with more than 3 / 4 of that.  Of 128 and more
    numbers the second part is far above the others, and met with zeros."""
    rows, by = np.zeros((0, dim)), np.zeros((0, dim))
    parts, far = -(-dim // 32), dim >= 128
    most = 0.75 * (dim - 32 * far)
    while len(rows) < TARGETS:
        size = np.repeat(2.0 ** rng.integers(0, 2, parts), 32)[:dim]
        signs = rng.choice([-1.0, 1.0], dim)
        q = 1.0 / size
        if far:
            size[32:64], q[32:64] = 2.0 ** rng.integers(0, 18), 0.0
        if (rows @ (signs * q) <= most).all() and (by @ (signs * size) <= most).all():
            rows, by = np.concatenate([rows, [signs * size]]), np.concatenate([by, [signs * q]])
    return rows, by


class Parts:
    """Keys, values, and a row of q for each of 128 tokens among 600; the others' keys are zeros."""

    def __init__(self, dim):
        rng = np.random.default_rng(dim)
        parts = -(-dim // 32)
        each = lambda lo, hi: np.repeat(2.0 ** rng.integers(lo, hi, (CONTEXT, parts)), 32, 1)[:, :dim]
        self.dim, self.target = dim, rng.permutation(CONTEXT)[:TARGETS]
        self.k, self.v = np.zeros((CONTEXT, 1, dim)), (rng.standard_normal((CONTEXT, dim)) * each(-9, 10))[:, None].astype(np.float32).astype(np.float64)
        self.k[self.target, 0], q = apart(rng, dim)
        self.q = 6.0 * q
        data_shape, exponent_shape = more.shapes(-(-CONTEXT // PAGE), 1, PAGE, dim, "fp4")
        data, exponents = np.zeros(data_shape, np.uint8), np.zeros(exponent_shape, np.int8)
        at = np.arange(CONTEXT)
        more.append(data, exponents, dim, "fp4", self.k, self.v, at)
        rows = more.numbers(data, exponents, dim, "fp4")[at // PAGE, 0, at % PAGE]
        self.keys, self.values = rows[:, 0], rows[:, 1]
        assert (self.keys == self.k[:, 0]).all()                                                    # powers of two are codes
        e = exponents.astype(int)[at // PAGE, 0, 0, :, :, at % PAGE]                                # [tokens, 2, parts]
        self.power = [e[:, kind].max(1) for kind in range(2)]                                       # a token's largest,
        self.block = [np.array([x[t // 16 * 16:t // 16 * 16 + 16].max() for t in at]) for x in self.power]      # and its block's
        for kind in range(2):                   # what the format holds exactly
            assert ((self.block[kind][:, None] - e[:, kind] <= 22) | (e[:, kind] == -64)).all()

    def expected(self, i, listed):
        """Row i -> out, its tolerance, lse, its tolerance, the weights."""
        o, l, spread, products = plain.attend_row(self.q[i], self.keys, self.values, self.dim ** -0.5)
        w = np.exp(self.dim ** -0.5 * (self.keys @ self.q[i]) - l)
        # a weight times its values' power of two is a 16-bit float whose largest is 2^7 at least: below 2^-14 it is off by 2^-25 rather than 2^-11 of itself
        power = 2.0 ** (self.power if listed else self.block)[1]
        tol_o, tol_l = plain.tolerance(self.dim, 11, o, spread, products)
        return o, tol_o + 2.0 ** -32 * (w * power).max() * (np.abs(self.values) / power[:, None]).sum(0) + CONTEXT * 2.0 ** -24 * spread, l, tol_l, w


_made = {}


def parts_of(dim):
    if dim not in _made:
        _made[dim] = Parts(dim)
    return _made[dim]


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("dim", DIMS)
def test_the_tolerances_see_every_part(dim, listed):
    """One part of a token's values twice or half as large, one part of its keys, or its block of 16 left out: further off than twice the tolerance, for all of the tokens."""
    p = parts_of(dim)
    for i, t in enumerate(p.target):
        o, tol_o, l, tol_l, w = p.expected(i, listed)
        assert w[t] > 0.99
        block = slice(t // 16 * 16, t // 16 * 16 + 16)
        assert (w[block] @ np.abs(p.values[block]) * (np.abs(w[block] @ p.values[block]) > 2 * tol_o)).any()
        for at in range(0, dim, 32):
            part = slice(at, at + 32)
            off = np.abs(w[t] * p.values[t, part])
            assert (off / 2 > 2 * tol_o[part]).any(), (i, at)
            score = dim ** -0.5 * (p.keys[t, part] @ p.q[i, part])
            for by in (2.0, 0.5):
                change = abs(np.log1p(w[t] * np.expm1(score * (by - 1.0))))
                assert change > 2 * tol_l or not p.q[i, part].any()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def check(p, out, lse, rows, listed):
    """rows: which row of q each row of out is."""
    out, lse = out.double().cpu().numpy().reshape(-1, p.dim), lse.double().cpu().numpy().reshape(-1)
    want = {}
    for n, i in enumerate(rows):
        if i not in want:
            want[i] = p.expected(i, listed)
        o, tol_o, l, tol_l, _ = want[i]
        assert abs(lse[n] - l) <= tol_l, (n, i, lse[n] - l, tol_l)
        assert (np.abs(out[n] - o) <= tol_o).all(), (n, i, float((np.abs(out[n] - o) / tol_o).max()))


def memory(kv, p):
    cache = kv.KvCache(-(-CONTEXT // PAGE), 1, p.dim, PAGE, "fp4")
    cache.append(torch.tensor(p.k).float().cuda(), torch.tensor(p.v).float().cuda(), torch.arange(CONTEXT, device="cuda"))
    return cache


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("requests, group", [(128, 1), (8, 16), (7, 20), (4, 32), (2, 64), (1, 128), (1, 300)])
@pytest.mark.parametrize("pages", [38, 400])
def test_attend(kv, dim, requests, group, pages):
    """One tile of rows, two, the kernels for many; a workgroup for all keys of its rows, and shares."""
    p = parts_of(dim)
    rows = np.arange(requests * group) % TARGETS
    table = np.full((requests, pages), -1)
    table[:, :38] = np.arange(38)
    q = torch.tensor(p.q[rows]).half().cuda().view(requests, group, dim)
    assert (q.double().cpu().numpy().reshape(-1, dim) == p.q[rows]).all()
    step = kv.KvStep(ints(table), ints(np.arange(requests + 1)), ints([CONTEXT] * requests), max_new=1)
    check(p, *memory(kv, p).attend(q, step), rows, False)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("tokens, group, k", [(128, 1, 600), (8, 16, 700), (4, 40, 2500), (128, 1, 5000)])
def test_selected(kv, dim, tokens, group, k):
    p, rng = parts_of(dim), np.random.default_rng(k)
    rows = np.arange(tokens * group) % TARGETS
    ids = np.full((tokens, 1, k), -1)
    for t in range(tokens):
        ids[t, 0, rng.permutation(k)[:CONTEXT]] = np.arange(CONTEXT)
    step = kv.KvStep(ints(np.tile(np.arange(38), (1, 1))), requests=ints([0] * tokens), positions=ints([CONTEXT - 1] * tokens))
    out = memory(kv, p).attend_selected(torch.tensor(p.q[rows]).half().cuda().view(tokens, group, dim), torch.tensor(ids).cuda(), step)
    check(p, *out, rows, True)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("tokens, group, k", [(128, 1, 38), (8, 16, 50), (4, 40, 300), (128, 1, 300)])
def test_blocks(kv, dim, tokens, group, k):
    p, rng = parts_of(dim), np.random.default_rng(k)
    rows = np.arange(tokens * group) % TARGETS
    ids = np.full((tokens, 1, k), -1)
    for t in range(tokens):
        ids[t, 0, rng.permutation(k)[:38]] = np.arange(38)
    step = kv.KvStep(ints(np.tile(np.arange(38), (1, 1))), requests=ints([0] * tokens), positions=ints([CONTEXT - 1] * tokens))
    blocks = kv.KvBlocks(memory(kv, p), 16)
    check(p, *blocks.attend(torch.tensor(p.q[rows]).half().cuda().view(tokens, group, dim), ints(ids), step), rows, False)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("group", [1, 20, 100, 300])
def test_parts_further_apart_than_a_float_reaches(kv, dim, group):
    """Values of 2^100 and of 2^-60 in one block of 16 tokens, whose quotient is none of a float's: the small ones are zeros beside the large ones, which come out to their own
    roundings (weights 2^-11, out 2^-8), and nothing comes out that is no number."""
    context, rng = 64, np.random.default_rng(dim + group)
    large = np.arange(context) % 3 == 0
    k, v = rng.standard_normal((context, 1, dim)), rng.standard_normal((context, 1, dim)) * np.where(large, 2.0 ** 100, 2.0 ** -60)[:, None, None]
    v[:, :, 32:64] = rng.standard_normal((context, 1, 32)) * 2.0 ** -60          # in no token a large one
    cache = kv.KvCache(4, 1, dim, 16, "fp4")
    cache.append(torch.tensor(k).float().cuda(), torch.tensor(v).float().cuda(), torch.arange(context, device="cuda"))
    keys, values = (x[:, 0].double().cpu().numpy() for x in cache.read(torch.arange(context, device="cuda")))
    q = torch.randn(1, group, dim, generator=torch.Generator().manual_seed(dim)).to(torch.bfloat16)
    step = kv.KvStep(ints([[0, 1, 2, 3]]), ints([0, 1]), ints([context]), ints([0]), ints([context - 1]), max_new=1)
    ids = torch.arange(context, device="cuda").view(1, 1, -1)
    for out, lse in (cache.attend(q.cuda(), step), cache.attend_selected(q.cuda(), ids, step), kv.KvBlocks(cache, 16).attend(q.cuda(), ints([[[0, 1, 2, 3]]]), step)):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.isfinite(out).all()
        for h in range(group):
            o, l, spread, products = plain.attend_row(q[0, h].double().numpy(), keys, values, dim ** -0.5)
            tol_o, tol_l = plain.tolerance(dim, 8, o, spread, products)
            assert abs(lse[0, h] - l) <= tol_l
            assert (np.abs(out[0, h] - o)[spread > 1.0] <= tol_o[spread > 1.0]).all()
            # the others' own block lost them: 2^-25 of its largest power of two at most, which is below 2^101
            assert (np.abs(out[0, h])[32:64] <= 2.0 ** 76).all()
