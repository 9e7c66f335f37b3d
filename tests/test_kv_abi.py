"""The cache's entry points refuse what the host can see to be wrong, before any HIP call; the plain implementation that the GPU tests
compare with agrees with hand-made values."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import kv_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv():
    from paper_2603_06660_amd import binding, build
    if not os.path.exists(binding.library_path()):
        build.build()
    from paper_2603_06660_amd import kv
    return kv


def test_struct_layouts_match_the_header(kv, tmp_path):
    src = tmp_path / "sizes.c"
    names = ("pag_kv_cache", "pag_kv_tables", "pag_kv_step", "pag_kv_attention")
    last = ("exponents", "free_count", "scratch", "workspace_bytes")
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "pag.h"\nint main(void){%s return 0;}\n' % "".join(
        'printf("%%zu %%zu ",sizeof(%s),offsetof(%s,%s));' % (n, n, f) for n, f in zip(names, last)))
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    want = []
    for s, f in zip((kv._Cache, kv._Tables, kv._Step, kv._Attention), last):
        want += [C.sizeof(s), getattr(s, f).offset]
    assert got == want


def _cache(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Cache), format=0, kv_heads=2, head_dim=64, page_tokens=32, reserved=0, num_pages=4, data=4096, exponents=4096)
    f.update(change)
    return kv._Cache(**f)


def _step(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Step), requests=2, max_pages=3, table_stride=3, tokens=2, table=4096, offsets=4096, context=4096,
             request=4096, positions=4096, slots=4096, granted=4096, lengths=4096, free_count=4096, scratch=4096)
    f.update(change)
    return kv._Step(**f)


def _tables(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Tables), requests=2, max_pages=3, page_tokens=32, table_stride=3, num_pages=4, table=4096, lengths=4096,
             free_pages=4096, free_count=4096)
    f.update(change)
    return kv._Tables(**f)


def _attention(kv, **change):
    f = dict(struct_size=C.sizeof(kv._Attention), dtype=1, heads=4, scale=1.0, q=4096, q_token_stride=256, q_head_stride=64, out=4096,
             out_token_stride=256, out_head_stride=64, workspace=4096, workspace_bytes=1 << 40)
    f.update(change)
    return kv._Attention(**f)


@pytest.mark.parametrize("change, code, word", [
    (dict(struct_size=8), -1, b"struct_size"), (dict(format=2), -1, b"format"), (dict(kv_heads=0), -1, b"positive"),
    (dict(head_dim=12), -5, b"head_dim"), (dict(head_dim=264), -5, b"head_dim"), (dict(page_tokens=24), -5, b"page_tokens"),
    (dict(num_pages=1 << 27), -5, b"2^32"), (dict(num_pages=(1 << 64) - 1), -5, b"2^32"), (dict(data=None), -1, b"null"),
    (dict(data=4104), -1, b"aligned"), (dict(exponents=4097), -1, b"aligned")])
def test_a_wrong_cache_is_refused_by_every_call(kv, change, code, word):
    lib, c = kv.load_library(), C.byref(_cache(kv, **change))
    rows = [C.c_void_p(4096), C.c_int64(128), C.c_int64(64)]
    for rc in (lib.pag_kv_append(c, C.c_uint32(1), *rows, *rows, C.c_void_p(4096), C.c_uint64(1), None),
               lib.pag_kv_read(c, C.c_void_p(4096), C.c_uint64(1), C.c_uint32(1), *rows, *rows, None),
               lib.pag_kv_attend(c, C.byref(_step(kv)), C.byref(_attention(kv)), None),
               lib.pag_kv_attend_selected(c, C.byref(_step(kv)), C.byref(_attention(kv)), C.c_void_p(4096), C.c_int64(8), C.c_int64(4),
                                          C.c_uint32(2), C.c_uint32(4), None)):
        assert rc == code and word in lib.pag_last_error()


@pytest.mark.parametrize("step, args, code, word", [
    (dict(struct_size=8), {}, -1, b"struct_size"), (dict(requests=0), {}, -1, b"requests"), (dict(table=None), {}, -1, b"table"),
    (dict(table_stride=2), {}, -1, b"table"), (dict(tokens=1 << 31), {}, -5, b"2^31"), (dict(max_pages=1 << 26, table_stride=1 << 26), {}, -5, b"2^31"),
    ({}, dict(struct_size=8), -1, b"struct_size"), ({}, dict(dtype=0), -5, b"PAG_F16"), ({}, dict(heads=3), -1, b"heads"),
    ({}, dict(scale=math.nan), -1, b"finite"), ({}, dict(softcap=-1.0), -1, b"finite"), ({}, dict(q=None), -1, b"null"),
    ({}, dict(q=4098), -1, b"aligned"), ({}, dict(q_head_stride=60), -1, b"strides"), ({}, dict(out_token_stride=257), -1, b"strides"),
    ({}, dict(lse=4098), -1, b"aligned"), ({}, dict(workspace=None), -1, b"workspace")])
def test_wrong_attention_arguments_are_refused(kv, step, args, code, word):
    lib = kv.load_library()
    c, s, a = _cache(kv), _step(kv, **step), _attention(kv, **args)
    assert lib.pag_kv_attend(C.byref(c), C.byref(s), C.byref(a), None) == code and word in lib.pag_last_error()
    rc = lib.pag_kv_attend_selected(C.byref(c), C.byref(s), C.byref(a), C.c_void_p(4096), C.c_int64(8), C.c_int64(4), C.c_uint32(2), C.c_uint32(4), None)
    assert rc == code and word in lib.pag_last_error()


def test_more_than_a_launch_has_threads_for_is_refused(kv):
    lib, c, a = kv.load_library(), _cache(kv), _attention(kv)
    rows = [C.c_void_p(4096), C.c_int64(128), C.c_int64(64)]
    for tokens in (1 << 26, 1 << 27, 1 << 63):                 # of 2 heads
        assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *rows, *rows, C.c_void_p(4096), C.c_uint64(tokens), None) == -5 and b"2^27" in lib.pag_last_error()
        assert lib.pag_kv_read(C.byref(c), C.c_void_p(4096), C.c_uint64(tokens), C.c_uint32(1), *rows, *rows, None) == -5 and b"2^27" in lib.pag_last_error()
    for change in (dict(tokens=1 << 21), dict(requests=1 << 22)):
        rc = lib.pag_kv_attend_selected(C.byref(c), C.byref(_step(kv, **change)), C.byref(a), C.c_void_p(4096), C.c_int64(8), C.c_int64(4), C.c_uint32(2),
                                        C.c_uint32(4), None)
        assert rc == -5 and b"2^23" in lib.pag_last_error()


def test_null_arguments_and_empty_calls(kv):
    lib = kv.load_library()
    c, s, a, t = _cache(kv), _step(kv), _attention(kv), _tables(kv)
    none = C.c_void_p(None)
    rows, nothing = [C.c_void_p(4096), C.c_int64(128), C.c_int64(64)], [none, C.c_int64(0), C.c_int64(0)]
    assert lib.pag_kv_attend(None, C.byref(s), C.byref(a), None) == -1
    assert lib.pag_kv_attend(C.byref(c), None, C.byref(a), None) == -1
    assert lib.pag_kv_attend(C.byref(c), C.byref(s), None, None) == -1
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *nothing, *rows, C.c_void_p(4096), C.c_uint64(1), None) == -1
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(3), *rows, *rows, C.c_void_p(4096), C.c_uint64(1), None) == -1
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), C.c_void_p(4096), C.c_int64(124), C.c_int64(64), *rows, C.c_void_p(4096), C.c_uint64(1), None) == -1
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *rows, *rows, C.c_void_p(4096), C.c_uint64(1 << 40), None) == -5
    assert lib.pag_kv_read(C.byref(c), none, C.c_uint64(1), C.c_uint32(1), *rows, *rows, None) == -1
    for bad in (dict(struct_size=1), dict(requests=0), dict(max_pages=0), dict(num_pages=0), dict(lengths=None), dict(free_count=None)):
        t = _tables(kv, **bad)
        assert lib.pag_kv_extend(C.byref(t), C.c_void_p(4096), C.byref(s), None) == -1, bad
        assert lib.pag_kv_release(C.byref(t), C.c_void_p(4096), None) == -1, bad
    t = _tables(kv)
    assert lib.pag_kv_extend(C.byref(_tables(kv, page_tokens=8)), C.c_void_p(4096), C.byref(s), None) == -5
    assert lib.pag_kv_extend(C.byref(t), none, C.byref(s), None) == -1 and lib.pag_kv_release(C.byref(t), none, None) == -1
    for bad in (dict(requests=3), dict(table=8192), dict(granted=None), dict(slots=None), dict(scratch=None)):
        assert lib.pag_kv_extend(C.byref(t), C.c_void_p(4096), C.byref(_step(kv, **bad)), None) == -1, bad
    # nothing to do: no GPU is needed either
    assert lib.pag_kv_append(C.byref(c), C.c_uint32(1), *nothing, *nothing, none, C.c_uint64(0), None) == 0
    assert lib.pag_kv_read(C.byref(c), none, C.c_uint64(5), C.c_uint32(1), *nothing, *nothing, None) == 0
    assert lib.pag_kv_attend(C.byref(c), C.byref(_step(kv, tokens=0)), C.byref(_attention(kv, q=None, out=None)), None) == 0
    for id_heads, k, code in ((3, 4, -1), (0, 4, -1), (1, 4, -1), (2, 1 << 31, -5)):
        rc = lib.pag_kv_attend_selected(C.byref(c), C.byref(_step(kv, tokens=0)), C.byref(a), C.c_void_p(4096), C.c_int64(8), C.c_int64(4),
                                        C.c_uint32(id_heads), C.c_uint32(k), None)
        assert rc == code


def test_binding_refuses_what_is_not_on_a_gpu(kv):
    import torch
    with pytest.raises(kv.PagError):
        kv.KvCache(4, 2, 64, device="cpu")
    with pytest.raises(kv.PagError):
        kv.KvCache.from_tensors(torch.zeros(1, 1, 16, 2, 64, dtype=torch.uint8), torch.zeros(1, 1, 1, 2, dtype=torch.int8), 64)
    with pytest.raises(kv.PagError):
        kv.KvCache.from_tensors(None, None, 64, "int4")
    with pytest.raises(kv.PagError):
        kv.KvTables.from_tensors(None, torch.zeros(2, 3, dtype=torch.int32), None, None, 16)
    with pytest.raises(kv.PagError):
        kv.KvStep(torch.zeros(2, 3, dtype=torch.int32))


# ---- the plain implementation -----------------------------------------------------------------------------------------------


def test_plain_codes():
    n = plain.fp8_numbers()
    assert n[0x7E] == 448 and n[0x01] == 2.0 ** -9 and n[0x38] == 1.0 and n[0xB8] == -1.0 and math.isnan(n[0x7F])
    finite = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    assert (plain.encode(n[finite], "fp8") == finite).all()                                   # every number is its own code
    # halfway cases go to the even code: 1.0625 between 1 and 1.125, 1.1875 between 1.125 and 1.25
    assert plain.encode(np.array([1.0625, 1.1875, -1.0625, 500.0, np.inf, np.nan]), "fp8").tolist() == [0x38, 0x3A, 0xB8, 0x7E, 0x7E, 0]
    assert plain.encode(np.array([0.5, 1.5, -2.5, 200.0, -np.inf, np.nan]), "int8").view(np.int8).tolist() == [0, 2, -2, 127, -127, 0]
    assert [plain.least_exponent(x, "int8") for x in (127.0, 127.5, 0.0, 63.5)] == [0, 1, -64, -1]
    assert [plain.least_exponent(x, "fp8") for x in (448.0, 448.5, 1.75)] == [0, 1, -8]


def test_plain_attention_by_hand():
    keys, values = np.array([[1.0, 0.0], [0.0, 1.0]]), np.array([[2.0, 0.0], [0.0, 4.0]])
    out, lse, spread, products = plain.attend_row(np.array([math.log(3.0), 0.0]), keys, values, 1.0)
    assert np.allclose(out, [1.5, 1.0]) and np.isclose(lse, math.log(4.0)) and np.allclose(spread, out) and np.isclose(products, math.log(3.0))
    out, lse, _, _ = plain.attend_row(np.array([9.0, 9.0]), keys, values, 1.0, slope=math.log(3.0), distance=np.array([0.0, 1.0]))
    assert np.allclose(out, [1.5, 1.0]) and np.isclose(lse, 9.0 + math.log(4.0 / 3.0))
    out, lse, _, _ = plain.attend_row(np.array([9.0, 9.0]), keys[:0], values[:0], 1.0)
    assert (out == 0).all() and lse == -math.inf


def test_plain_tables_by_hand():
    table = np.full((3, 3), -1)
    table[0, 0] = 7
    e = plain.extend([3, 0, 0], table, [5, 6, 9], 3, [2, 9, 1], 4, 13)
    # request 0 takes page 9, request 1 wants three pages and two are left, request 2 is refused with it
    assert table.tolist() == [[7, 9, -1], [-1] * 3, [-1] * 3] and e["granted"] == [1, 0, 0] and e["free_count"] == [2]
    assert e["slots"] == [31, 36] + [-1] * 11 and e["positions"][:3] == [3, 4, -1] and e["context"] == [5, 0, 0]
    assert e["offsets"] == [0, 2, 11, 12] and e["requests"] == [0, 0] + [1] * 9 + [2, -1]
