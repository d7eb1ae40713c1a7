"""What the serving calls refuse, and answer, before they look at any device."""
import ctypes

import pytest

import paper_2505_00232_b200 as P
from paper_2505_00232_b200 import binding

lib, BAD = binding.lib, P.QL_ERR_INVALID_ARG
BUFFER = ctypes.create_string_buffer(4096)
AT = (ctypes.addressof(BUFFER) + 255) & ~255                              # 256-byte aligned; never read: every call below is refused, or has nothing to do


def tables(cos=AT, sin=AT + 1024, first=0, n_pos=4, rot=64, base=1e4, scaling=None, device=0):
    return lib.qlinear_rope_tables(cos, sin, first, n_pos, rot, base, None if scaling is None else ctypes.byref(binding.qlinear_rope_scaling(*scaling)), device, None)


@pytest.mark.parametrize("change", [
    {"cos": None}, {"sin": None}, {"cos": AT + 4}, {"sin": AT}, {"first": -1}, {"n_pos": -1}, {"first": 2 ** 31 - 3}, {"rot": 0}, {"rot": 24}, {"rot": 528}, {"base": 1.0}, {"base": 0.5},
    {"base": float("nan")}, {"base": float("inf")}, {"device": -1}, {"scaling": (5, 8192, 2.0, 1.0, 4.0)}, {"scaling": (-1, 8192, 2.0, 1.0, 4.0)}, {"scaling": (1, 8192, 0.5, 1.0, 4.0)},
    {"scaling": (2, 8192, float("nan"), 1.0, 4.0)}, {"scaling": (3, 0, 2.0, 1.0, 4.0)}, {"scaling": (3, 8192, 2.0, 4.0, 4.0)}, {"scaling": (4, 8192, 2.0, 0.0, 4.0)},
    {"scaling": (4, 8192, 2.0, 1.0, float("inf"))}])
def test_tables_refused(change):
    assert tables(**change) == BAD


def test_tables_of_nothing():
    assert tables(n_pos=0, cos=None, sin=None) == binding.QL_OK


@pytest.mark.parametrize("scaling,rot,n_pos,device", [("other", 64, 4, None), (None, 64, -1, None), (None, -16, 4, None), (None, 64, 4, "cpu")])
def test_tables_refused_in_python(scaling, rot, n_pos, device):
    with pytest.raises(P.QLinearError) as e:
        P.qlinear_rope_tables(n_pos, rot, scaling=scaling, device=device)
    assert e.value.status == BAD


@pytest.mark.parametrize("desc,size", [((10, 16, 8, 128), 8 * 2304), ((10, 64, 2, 64), 8 * 1152), ((1, 1024, 1, 256), 64 * 4608), ((2 ** 27 - 1, 16, 1, 64), 1152),
                                       ((2 ** 27, 16, 1, 64), 0), ((0, 16, 8, 128), 0), ((10, 8, 8, 128), 0), ((10, 48, 8, 128), 0), ((10, 2048, 8, 128), 0), ((10, 16, 0, 128), 0), ((10, 16, 1025, 128), 0),
                                       ((10, 16, 8, 32), 0), ((10, 16, 8, 96), 0)])
def test_page_bytes(desc, size):
    """Half a byte for an element of the keys and the values, two for every 32 of them: 0.5625 in all; 0 for what has no cache."""
    d = binding.qlinear_paged_desc(*desc)
    assert lib.qlinear_paged_page_bytes(ctypes.byref(d)) == size
    assert size == 0 or size == desc[1] * desc[2] * desc[3] * 2 * 9 // 16
    if size == 0:
        h = ctypes.c_void_p()
        assert lib.qlinear_paged_create(ctypes.byref(d), AT, 0, ctypes.byref(h)) == P.QL_ERR_UNSUPPORTED and not h.value


def test_no_handle():
    d, h = binding.qlinear_paged_desc(10, 16, 8, 128), ctypes.c_void_p()
    assert lib.qlinear_paged_page_bytes(None) == 0
    assert lib.qlinear_paged_create(None, AT, 0, ctypes.byref(h)) == BAD
    assert lib.qlinear_paged_create(ctypes.byref(d), None, 0, ctypes.byref(h)) == BAD
    assert lib.qlinear_paged_create(ctypes.byref(d), AT + 16, 0, ctypes.byref(h)) == BAD
    assert lib.qlinear_paged_create(ctypes.byref(d), AT, 0, None) == BAD
    batch = (AT, 4, 4, AT, AT, 1, 1)
    assert lib.qlinear_paged_append(None, None, 0, AT, 1024, AT, 1024, None, 0, 0, *batch, None, None, 0, 0, 0, None) == BAD
    assert lib.qlinear_paged_read(None, *batch, AT, AT, None) == BAD
    assert lib.qlinear_paged_attention_workspace(None, 8, 1, 1) == 0
    assert lib.qlinear_paged_attention(None, AT, 1024, AT + 64, 1024, 8, *batch, 1, 1.0, 0.0, 0, AT, 4096, None) == BAD


def logits(x=AT, ld=8, out=AT, out_ld=8, rows=2, vocab=8, fp32=0, tokens=AT, n_tokens=4, start=AT, n_prompt=AT, rep=AT, pres=AT, freq=AT, ids=AT, values=AT, b_start=AT, n_biases=4, mask=AT, mask_ld=1, device=0):
    return lib.qlinear_adjust_logits(x, ld, out, out_ld, rows, vocab, fp32, tokens, n_tokens, start, n_prompt, rep, pres, freq, ids, values, b_start, n_biases, mask, mask_ld, device, None)


@pytest.mark.parametrize("change", [
    {"x": None}, {"out": None}, {"ld": 7}, {"out_ld": 7}, {"out_ld": 16}, {"rows": -1}, {"rows": 65536}, {"vocab": 0}, {"fp32": 2}, {"n_tokens": -1}, {"n_biases": -1}, {"device": -1}, {"tokens": None},
    {"start": None}, {"ids": None}, {"values": None}, {"b_start": None}, {"mask_ld": 0}, {"x": AT + 1}, {"tokens": AT + 2}, {"rep": AT + 2}, {"mask": AT + 2}, {"values": AT + 1}])
def test_logits_refused(change):
    assert logits(**change) == BAD


def test_logits_of_nothing():
    assert logits(rows=0) == binding.QL_OK


@pytest.mark.parametrize("change", [{"n_pos": 2 ** 32}, {"rot": 2 ** 32 + 64}, {"first": 2 ** 32}, {"first": 2 ** 31}, {"first": -2 ** 32}, {"scaling": "yarn", "factor": 2.0, "original": 2 ** 32 + 8192}])
def test_tables_of_numbers_beyond_32_bits(change):
    """Refused: their lower 32 bits would be another call."""
    with pytest.raises(P.QLinearError) as e:
        P.qlinear_rope_tables(**{"n_pos": 4, "rot": 64, **change})
    assert e.value.status == BAD


@pytest.mark.parametrize("args", [(2 ** 32 + 4, 16, 2, 64), (4, 2 ** 32 + 16, 2, 64), (4, 16, 2 ** 32 + 2, 64), (4, 16, 2, 2 ** 32 + 64)])
def test_caches_of_numbers_beyond_32_bits(args):
    with pytest.raises(P.QLinearError) as e:
        P.PagedKV(*args)
    assert e.value.status == BAD
