"""Turned queries are written while keys, values and other queries are still being read: rows of out that lie over any of these, but for q's own in place, or over each other
are refused; rows that lie between them are not."""
import ctypes as C

import pytest
from test_kv_abi import _cache, kv  # noqa: F401
from test_kv_more_abi import _rotation

torch = pytest.importorskip("torch")

K, V, ROW = 1 << 20, 2 << 20, 128          # keys and values of 2 heads, 64 numbers of 16 bits; 3 tokens


def append(kv, heads=4, token=256, head=64, **change):
    rows = lambda at: [C.c_void_p(at), C.c_int64(token), C.c_int64(head)]
    return kv.load_library().pag_kv_append_rotated(C.byref(_cache(kv)), C.c_uint32(1), *rows(K), *rows(V), C.c_void_p(4096), C.c_uint64(3),
                                                   C.byref(_rotation(kv, heads=heads, **change)), None)


@pytest.mark.parametrize("change, word", [
    (dict(out=K), b"keys and values"), (dict(out=V), b"keys and values"), (dict(out=K + ROW), b"keys and values"), (dict(out=K - 3 * ROW), b"keys and values"),
    (dict(out=V + 16), b"keys and values"), (dict(q=K, out=K), b"keys and values"),                 # keys turned in place as queries
    (dict(q=K - 2 * ROW, out=K - 2 * ROW), b"keys and values"),                                     # queries and keys of a fused projection, side by side, in place
    (dict(out=K + 2 * ROW, out_head_stride=-64, heads=3), b"keys and values"), (dict(out=V - 10 * ROW, out_head_stride=320, heads=3), b"keys and values"),
    (dict(q=4 << 20, out=(4 << 20) + ROW), b"q itself or apart"), (dict(q=4 << 20, out=(4 << 20) - 3 * ROW), b"q itself or apart"),
    (dict(q=4 << 20, out=(4 << 20) + 16), b"q itself or apart"), (dict(out=K + 112, out_head_stride=8, heads=1), b"keys and values"),
    (dict(q=4 << 20, out=4 << 20, q_head_stride=0, out_head_stride=0), b"over each other"), (dict(q=4 << 20, out=4 << 20, q_token_stride=0, out_token_stride=0), b"over each other"),
    (dict(q=4 << 20, out=5 << 20, out_head_stride=56), b"over each other")])
def test_rows_that_lie_over_others_are_refused(kv, change, word):
    assert append(kv, **change) == -1 and word in kv.load_library().pag_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_rows_that_lie_between_others_are_not(kv, fmt):
    """Every second row of an array, rows behind and before the keys', rows of a token that are read by several heads, in place."""
    tokens, heads, dim = 37, 4, 64
    slots, at = torch.arange(tokens, device="cuda"), torch.arange(tokens, device="cuda", dtype=torch.int32)
    rotation = kv.KvRotation(torch.rand(32, device="cuda"))
    fill = lambda *shape: torch.randn(*shape, device="cuda", dtype=torch.bfloat16)

    def same(k, v, q, out):
        one, two = kv.KvCache(3, heads, dim, 16, fmt), kv.KvCache(3, heads, dim, 16, fmt)
        want = one.append_rotated(k.clone(), v.clone(), slots, at, rotation, q=q.clone())
        assert two.append_rotated(k, v, slots, at, rotation, q=q, out=out) is out and torch.equal(out, want)
        assert torch.equal(one.data, two.data) and torch.equal(one.exponents, two.exponents)

    x = fill(tokens, 4 * heads, dim)
    same(x[:, 0::4], x[:, 1::4], x[:, 2::4], x[:, 3::4])
    same(x[:, :heads], x[:, heads:2 * heads], x[:, 2 * heads:3 * heads], x[:, 2 * heads:3 * heads])
    same(x[:, 3 * heads:], x[:, heads:2 * heads], x[:, 2 * heads:3 * heads], x[:, :heads])
    y = fill(4 * heads, tokens, dim).transpose(0, 1)
    same(y[:, :heads], y[:, heads:2 * heads], y[:, 2 * heads:3 * heads], y[:, 3 * heads:])
    same(fill(tokens, heads, dim), fill(tokens, heads, dim), fill(tokens, 1, dim).expand(tokens, 6, dim), fill(tokens, 6, dim))
    z = fill(tokens, heads, dim)
    same(z, z, z, fill(tokens, heads, dim))
