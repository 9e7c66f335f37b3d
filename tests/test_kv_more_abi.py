"""The entry points of the rotated write, of the 4-bit cache and of blocks refuse what the host can see to be wrong, before any HIP call; the plain
implementation that the GPU tests compare with agrees with hand-made values."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import kv_more_plain as more
from test_kv_abi import ROOT, _attention, _cache, _step, kv  # noqa: F401

FP4 = 4


def test_struct_layouts_match_the_header(kv, tmp_path):
    src = tmp_path / "sizes.c"
    names, last = ("pag_kv_rotation", "pag_kv_blocks"), ("out_head_stride", "exponents")
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pag.h"\nint main(void){%s printf("%%d %%d %%d",PAG_KV_FP4,PAG_KV_HALVES,PAG_KV_NEIGHBOURS); return 0;}\n' % "".join(
        'printf("%%zu %%zu ",sizeof(%s),offsetof(%s,%s));' % (n, n, f) for n, f in zip(names, last)))
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    want = []
    for s, f in zip((kv._Rotation, kv._Blocks), last):
        want += [C.sizeof(s), getattr(s, f).offset]
    assert got == want + [kv._FORMATS["fp4"], kv._PAIRS["halves"], kv._PAIRS["neighbours"]]


def _rotation(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Rotation), pairs=0, turned=64, heads=4, frequencies=4096, positions=4096, q=4096, q_token_stride=256, q_head_stride=64,
             out=8192, out_token_stride=256, out_head_stride=64)
    f.update(change)
    return kv._Rotation(**f)


def _blocks(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Blocks), block_tokens=16, codes=4096, exponents=4096)
    f.update(change)
    return kv._Blocks(**f)


ROWS = [C.c_void_p(4096), C.c_int64(128), C.c_int64(64)]


def _append(kv, cache, rotation, rows=ROWS, slots=4096, tokens=1, dtype=1):
    return kv.load_library().pag_kv_append_rotated(C.byref(cache), C.c_uint32(dtype), *rows, *rows, C.c_void_p(slots), C.c_uint64(tokens),
                                                   None if rotation is None else C.byref(rotation), None)


@pytest.mark.parametrize("change, code, word", [
    (dict(struct_size=8), -1, b"struct_size"), (dict(pairs=2), -1, b"pairs"), (dict(turned=0), -5, b"turned"), (dict(turned=12), -5, b"turned"), (dict(turned=72), -5, b"turned"),
    (dict(heads=65537), -5, b"heads"), (dict(frequencies=None), -1, b"frequencies"), (dict(frequencies=4098), -1, b"aligned"), (dict(positions=None), -1, b"positions"),
    (dict(q=None), -1, b"null"), (dict(out=None), -1, b"null"), (dict(q=4104), -1, b"q and its strides"), (dict(q_head_stride=60), -1, b"q and its strides"),
    (dict(out_token_stride=252), -1, b"out and its strides"), (dict(out=4096, out_token_stride=512), -1, b"in place")])
@pytest.mark.parametrize("format", [0, FP4])
def test_a_wrong_rotation_is_refused(kv, change, code, word, format):
    assert _append(kv, _cache(kv, format=format), _rotation(kv, **change)) == code and word in kv.load_library().pag_last_error()


def test_wrong_rotated_calls_are_refused(kv):
    lib, none = kv.load_library(), [C.c_void_p(None), C.c_int64(0), C.c_int64(0)]
    assert _append(kv, _cache(kv), None) == -1 and b"rotation is null" in lib.pag_last_error()
    assert _append(kv, _cache(kv, head_dim=12), _rotation(kv)) == -5 and _append(kv, _cache(kv), _rotation(kv), dtype=3) == -1
    assert _append(kv, _cache(kv), _rotation(kv), rows=none) == -1 and _append(kv, _cache(kv), _rotation(kv), slots=None) == -1
    for tokens in ((1 << 24) + 1, 1 << 25, 1 << 26, 1 << 63):
        assert _append(kv, _cache(kv, kv_heads=1), _rotation(kv), tokens=tokens) == -5
    # nothing to do: no GPU is needed
    assert _append(kv, _cache(kv), _rotation(kv, q=None, out=None, positions=None), rows=none, slots=None, tokens=0) == 0


def test_the_4_bit_cache_and_its_limits(kv):
    lib = kv.load_library()
    for format in (2, 3, 5):
        assert lib.pag_kv_append(C.byref(_cache(kv, format=format)), C.c_uint32(1), *ROWS, *ROWS, C.c_void_p(4096), C.c_uint64(1), None) == -1
        assert b"format" in lib.pag_last_error()
    c = _cache(kv, format=FP4, exponents=4104)
    assert lib.pag_kv_read(C.byref(c), C.c_void_p(4096), C.c_uint64(1), C.c_uint32(1), *ROWS, *ROWS, None) == -1 and b"16-byte" in lib.pag_last_error()
    c = _cache(kv, format=FP4, kv_heads=1)
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *ROWS, *ROWS, C.c_void_p(4096), C.c_uint64(1 << 25), None) == -5 and b"2^25" in lib.pag_last_error()
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *ROWS, *ROWS, C.c_void_p(4096), C.c_uint64(0), None) == 0


def _select(kv, cache, blocks, step, args, id_heads=2, k=4, ids=4096):
    return kv.load_library().pag_kv_blocks_select(C.byref(cache), None if blocks is None else C.byref(blocks), C.byref(step), C.byref(args), C.c_uint32(id_heads), C.c_uint32(k),
                                                  C.c_void_p(ids), C.c_int64(8), C.c_int64(4), None)


def _attend(kv, cache, step, args, id_heads=2, k=4, block=16, ids=4096):
    return kv.load_library().pag_kv_attend_blocks(C.byref(cache), C.byref(step), C.byref(args), C.c_void_p(ids), C.c_int64(8), C.c_int64(4), C.c_uint32(id_heads),
                                                  C.c_uint32(k), C.c_uint32(block), None)


@pytest.mark.parametrize("change, word", [(dict(struct_size=8), b"struct_size"), (dict(block_tokens=0), b"block_tokens"), (dict(block_tokens=24), b"block_tokens"),
                                          (dict(block_tokens=64), b"block_tokens"), (dict(codes=None), b"null"), (dict(codes=4104), b"aligned"), (dict(exponents=None), b"null")])
def test_wrong_blocks_are_refused(kv, change, word):
    lib, b = kv.load_library(), _blocks(kv, **change)
    assert lib.pag_kv_blocks_update(C.byref(_cache(kv)), C.byref(b), C.c_void_p(4096), C.c_uint64(1), None) == -1 and word in lib.pag_last_error()
    assert _select(kv, _cache(kv), b, _step(kv), _attention(kv)) == -1 and word in lib.pag_last_error()
    if "block_tokens" in change:
        assert _attend(kv, _cache(kv), _step(kv), _attention(kv), block=change["block_tokens"]) == -1 and word in lib.pag_last_error()


@pytest.mark.parametrize("step, args, call, code, word", [
    (dict(struct_size=8), {}, {}, -1, b"struct_size"), (dict(requests=0), {}, {}, -1, b"requests"), (dict(table=None), {}, {}, -1, b"table"),
    (dict(max_pages=1 << 26, table_stride=1 << 26), {}, {}, -5, b"2^31"), ({}, dict(struct_size=8), {}, -1, b"struct_size"), ({}, dict(dtype=0), {}, -5, b"PAG_F16"),
    ({}, dict(heads=3), {}, -1, b"heads"), ({}, {}, dict(id_heads=0), -1, b"id_heads"), ({}, {}, dict(id_heads=3), -1, b"id_heads"), ({}, {}, dict(k=1 << 27), -5, b"2^30"),
    ({}, dict(window=1 << 30), {}, -5, b"2^30"), ({}, dict(q=None), {}, -1, b"null"), ({}, dict(q=4098), {}, -1, b"aligned"), ({}, dict(q_head_stride=60), {}, -1, b"strides"),
    (dict(tokens=1 << 22), {}, {}, -5, b"2^23"), (dict(request=None), {}, {}, -1, b"request"), (dict(positions=None), {}, {}, -1, b"positions"),
    ({}, {}, dict(ids=4098), -1, b"ids"), ({}, {}, dict(ids=None), -1, b"ids")])
def test_wrong_choices_and_attention_are_refused(kv, step, args, call, code, word):
    lib = kv.load_library()
    assert _select(kv, _cache(kv), _blocks(kv), _step(kv, **step), _attention(kv, **args), **call) == code and word in lib.pag_last_error()
    # the other one needs a GPU's size before it looks at its arrays
    if not (set(call) == {"ids"} or set(step) & {"request", "positions"}):
        assert _attend(kv, _cache(kv), _step(kv, **step), _attention(kv, **args), **call) == code and word in lib.pag_last_error()


def test_choices_of_nothing_and_their_workspace(kv):
    lib = kv.load_library()
    assert _select(kv, _cache(kv), None, _step(kv), _attention(kv)) == -1
    assert _select(kv, _cache(kv), _blocks(kv), _step(kv, tokens=0), _attention(kv, q=None)) == 0 and _select(kv, _cache(kv), _blocks(kv), _step(kv), _attention(kv, q=None), k=0) == 0
    assert lib.pag_kv_blocks_update(C.byref(_cache(kv)), C.byref(_blocks(kv)), None, C.c_uint64(0), None) == 0
    assert lib.pag_kv_blocks_update(C.byref(_cache(kv)), C.byref(_blocks(kv)), None, C.c_uint64(1), None) == -1
    assert lib.pag_kv_blocks_update(C.byref(_cache(kv)), C.byref(_blocks(kv)), C.c_void_p(4096), C.c_uint64(1 << 26), None) == -5
    size = C.c_uint64()
    room = lambda pages, tokens=2, id_heads=2, heads=4: (lib.pag_kv_blocks_workspace_bytes(C.byref(_cache(kv)), C.byref(_step(kv, max_pages=pages, table_stride=pages, tokens=tokens)), C.byref(
        _attention(kv, heads=heads)), C.c_uint32(id_heads), C.c_uint32(4), C.c_uint32(16), C.byref(size), None), size.value)
    assert room(512) == (0, 0) and room(513) == (0, 4 * 2 * 2 * 1026)           # 1,024 blocks fit a wave's registers
    assert room(500, id_heads=32, heads=32) == (0, 4 * 2 * 32 * 1000)          # 16 lists of 1,000 keys do not fit LDS
    assert room(440, id_heads=32, heads=32) == (0, 0)
    # such a workspace has to be there
    step = _step(kv, max_pages=513, table_stride=513)
    for args in (dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=4 * 2 * 2 * 1026 - 1), dict(workspace=4104)):
        assert _select(kv, _cache(kv), _blocks(kv), step, _attention(kv, **args)) == -1 and b"workspace" in lib.pag_last_error()
    assert _select(kv, _cache(kv), _blocks(kv), _step(kv, max_pages=1 << 24, table_stride=1 << 24, tokens=1 << 18), _attention(kv)) == -5


# ---- the plain implementation -----------------------------------------------------------------------------------------------


def test_plain_fp4_by_hand():
    x = np.array([0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 100.0, -0.75, -0.1, math.nan, -math.inf])
    assert more.encode_fp4(x).tolist() == [0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 10, 0, 0, 15]
    assert (more.decode_fp4(np.arange(16)) == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]).all()
    assert [more.least_exponent_fp4(x) for x in (7.0, 7.01, 3.5, 0.0, 6.0)] == [0, 1, -1, -64, 0]
    data, exponents = np.zeros((1, 1, 16, 2, 32), np.uint8), np.zeros((1, 1, 1, 2, 2, 16), np.int8)
    k = np.zeros((1, 1, 64))
    k[0, 0, [0, 1, 33]] = 6.0, -1.0, 14.0
    more.append(data, exponents, 64, "fp4", k, -k, [3])
    assert data[0, 0, 3, 0, 0] == 0xA7 and data[0, 0, 3, 0, 16] == 0x70 and exponents[0, 0, 0, 0, :, 3].tolist() == [0, 1]
    n = more.numbers(data, exponents, 64, "fp4")
    assert n[0, 0, 3, 0, [0, 1, 33]].tolist() == [6.0, -1.0, 12.0] and n[0, 0, 3, 1, 0] == -6.0 and (n[0, 0, 4] == 0).all()


def test_plain_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    f = np.array([math.pi / 2, math.pi], np.float64)
    assert np.allclose(more.turn(x, [1], f, "halves"), [[[-3.0, -2.0, 1.0, -4.0, 5.0]]])
    assert np.allclose(more.turn(x, [1], f, "neighbours"), [[[-2.0, 1.0, -3.0, -4.0, 5.0]]])


def test_plain_choice_by_hand():
    keys = np.array([[127.0, -2.0], [3.0, 0.4]])
    codes, e = more.summary(keys)
    assert e == 0 and codes.tolist() == [[127.0, 1.0], [3.0, -2.0]]
    q, e = more.query_codes(np.array([1.0, -0.5, math.nan, math.inf]))
    assert e == -6 and q.tolist() == [64.0, -32.0, 0.0, 127.0]
    assert more.select([(0, 1.0), (1, 5.0), (2, 5.0), (3, 0.0), (4, 5.0)], 2) == [1, 2] and more.select([(7, 1.0)], 3) == [7, -1, -1]
