"""What the entry points of the 8-bit cache refuse, without a GPU, and the definitions that they are tested with."""
import ctypes
import pathlib

import numpy as np
import pytest
import torch

from oracle import serving
from paper_2606_29563_gb300 import build as kbuild
from paper_2606_29563_gb300 import kvec

BF = torch.bfloat16
BAD, UNSUPPORTED = kvec.KVEC_ERR_INVALID_ARG, kvec.KVEC_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def lib():
    kbuild.build()
    return kvec.load()


def cache(**over):
    c = dict(dtype=kvec.KVEC_BF16, page_size=64, num_pages=10, max_pages=4, k_pages=4096, v_pages=8192, weights=16,
             page_table=64, lens=128)
    c.update(over)
    return kvec.kvec_paged_cache(**c)


def rotate_args(**over):
    a = dict(dtype=kvec.KVEC_BF16, num_tokens=1, q=16, k=16, v=16, q_stride=4096, k_stride=1024, v_stride=1024, eps=1e-6,
             rot_dim=128, max_positions=10, rot_table=16, positions=16, q_out=32)
    a.update(over)
    return kvec.kvec_rotate_args(**a)


def refused(call, status, words):
    with pytest.raises(kvec.KvecError) as e:
        call()
    assert e.value.status == status and words in str(e.value), str(e.value)


GOOD = kvec.kvec_paged_scales(16, 32)


def calls(c, s):
    return [lambda: kvec.kvec_rotate_append_quant(None, rotate_args(), 1, None, c, s),
            lambda: kvec.kvec_paged_decode_quant(None, 1, 16, c, s, 64, 0, 0, 16, 16, 0),
            lambda: kvec.kvec_paged_evict_quant(None, 1, c, s, 16, 4, 64, 8, 0, 0, 16, 16)]


@pytest.mark.parametrize("scales,words", [
    (None, "k_scales"), (kvec.kvec_paged_scales(None, 16), "k_scales"), (kvec.kvec_paged_scales(16, None), "k_scales"),
    (kvec.kvec_paged_scales(8, 16), "16-byte"), (kvec.kvec_paged_scales(16, 4), "16-byte"),
])
def test_bad_scales(scales, words):
    for call in calls(cache(), scales):
        refused(call, BAD, words)
    if scales is not None:
        refused(lambda: kvec.kvec_paged_read(None, 1, cache(), scales, None, 16, 5, 16, 16), BAD, words)


@pytest.mark.parametrize("over,status,words", [
    (dict(dtype=2), BAD, "dtype"), (dict(page_size=8), UNSUPPORTED, "page_size"), (dict(num_pages=0), BAD, "num_pages"),
    (dict(max_pages=2 ** 14 + 1), BAD, "max_pages"), (dict(k_pages=None), BAD, "NULL"), (dict(v_pages=8), BAD, "16-byte"),
    (dict(page_table=2), BAD, "4-byte"), ({}, BAD, "handle is NULL"),
])
def test_bad_caches(over, status, words):
    for call in calls(cache(**over), GOOD):
        refused(call, status, words)
    for s in (GOOD, None):
        refused(lambda: kvec.kvec_paged_read(None, 1, cache(**over), s, None, 16, 5, 16, 16), status, words)


def test_bad_arguments():
    refused(lambda: kvec.kvec_rotate_append_quant(None, rotate_args(), 1, None, None, GOOD), BAD, "cache is NULL")
    refused(lambda: kvec.kvec_rotate_append_quant(None, rotate_args(dtype=kvec.KVEC_FP16), 1, None, cache(), GOOD), BAD, "differs")
    refused(lambda: kvec.kvec_rotate_append_quant(None, None, 1, None, cache(), GOOD), BAD, "args")
    refused(lambda: kvec.kvec_paged_decode_quant(None, 1, 16, cache(), GOOD, 257, 0, 0, 16, 16, 0), BAD, "max_len")
    refused(lambda: kvec.kvec_paged_decode_quant(None, 1, 16, cache(), GOOD, 64, -1, 0, 16, 16, 0), BAD, "window")
    refused(lambda: kvec.kvec_paged_evict_quant(None, 1, cache(weights=None), GOOD, 16, 4, 64, 8, 0, 0, 16, 16), BAD, "weights")
    refused(lambda: kvec.kvec_paged_evict_quant(None, 1, cache(), GOOD, 16, 4, 64, 8, 5, 4, 16, 16), BAD, "sinks")
    refused(lambda: kvec.kvec_paged_read(None, 1, cache(), GOOD, None, 16, -1, 16, 16), BAD, "num_rows")
    refused(lambda: kvec.kvec_paged_read(None, 1, None, None, None, 16, 1, 16, 16), BAD, "cache is NULL")


def selector(Hq=8, Hkv=2):
    """The binding's own checks need no handle."""
    s = kvec.KvecSelector.__new__(kvec.KvecSelector)
    s._torch, s.params, s.handle, s.device = torch, kvec.make_params(Hq, Hkv), None, torch.device("cpu")
    s._lib, s._decode_bytes, s._current = kvec.load(), {}, lambda index: 0
    return s


def tensors(Hkv=2, page=16, pages=6, batch=2):
    k = torch.zeros((pages, Hkv, page, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    return dict(k_pages=k, v_pages=k.clone(), page_table=torch.zeros((batch, 3), dtype=torch.int32),
                lens=torch.zeros(batch, dtype=torch.int32), weights=torch.zeros((pages, Hkv, page)),
                k_scales=torch.ones((pages, Hkv, page)), v_scales=torch.ones((pages, Hkv, page)), dtype=BF)


@pytest.mark.parametrize("name,value", [
    ("dtype", None), ("dtype", torch.float32), ("k_scales", None), ("v_scales", None), ("k_scales", torch.ones((6, 2, 8))),
    ("v_scales", torch.ones((6, 2, 16), dtype=torch.float16)), ("k_scales", torch.ones((6, 16, 2)).transpose(1, 2)),
    ("v_pages", torch.zeros((6, 2, 16, 128), dtype=BF)), ("k_pages", torch.zeros((6, 2, 16, 128), dtype=BF)),
    ("k_pages", torch.zeros((6, 2, 16, 128), dtype=torch.uint8)),
    ("k_pages", torch.zeros((6, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e5m2)),
])
def test_the_binding_checks_a_cache(name, value):
    kvec.PagedCache(**tensors())
    with pytest.raises(kvec.KvecError):
        kvec.PagedCache(**{**tensors(), name: value})


def test_the_binding_keeps_formats_apart():
    bf = torch.zeros((6, 2, 16, 128), dtype=BF)
    plain = dict(k_pages=bf, v_pages=bf.clone(), page_table=torch.zeros((2, 3), dtype=torch.int32), lens=torch.zeros(2, dtype=torch.int32))
    kvec.PagedCache(**plain, dtype=BF)
    for over in (dict(k_scales=torch.ones((6, 2, 16))), dict(v_scales=torch.ones((6, 2, 16))), dict(dtype=torch.float16)):
        with pytest.raises(kvec.KvecError):
            kvec.PagedCache(**plain, **over)


def test_the_binding_checks_a_read():
    sel, c, cu = selector(), kvec.PagedCache(**tensors()), torch.zeros(3, dtype=torch.int32)
    refused(lambda: sel.paged_read(c, cu, 4), BAD, "handle is NULL")
    for bad in (dict(cu_rows=cu.long()), dict(cu_rows=cu[:2]), dict(num_rows=-1), dict(num_rows=2 ** 31), dict(first=cu),
                dict(first=torch.zeros(2)), dict(k_out=torch.zeros((4, 2, 128))), dict(v_out=torch.zeros((5, 2, 128), dtype=BF)),
                dict(k_out=torch.zeros((4, 2, 256), dtype=BF)[..., ::2])):
        with pytest.raises(kvec.KvecError) as e:
            sel.paged_read(**{**dict(cache=c, cu_rows=cu, num_rows=4), **bad})
        assert "handle" not in str(e.value)
    with pytest.raises(kvec.KvecError):
        selector(8, 4).paged_read(c, cu, 4)


def test_the_header_names_every_entry_point():
    header = (pathlib.Path(__file__).parents[1] / "include" / "kvec.h").read_text()
    for name in ("kvec_rotate_append_quant", "kvec_paged_decode_quant_bytes", "kvec_paged_decode_quant", "kvec_paged_evict_quant",
                 "kvec_paged_read", "kvec_shared_decode_bytes", "kvec_shared_decode", "kvec_shared_decode_quant_bytes",
                 "kvec_shared_decode_quant"):
        assert name in kvec.EXPORTED and f" {name}(" in header and callable(getattr(kvec, name))
    assert kvec.kvec_paged_decode_quant_bytes(None, 1, 64, 0, 0, True) == 0


def test_the_binding_checks_queries_of_an_eight_bit_cache():
    sel, c = selector(), kvec.PagedCache(**tensors())
    refused(lambda: sel.paged_decode(torch.zeros((2, 8, 128), dtype=BF), c), BAD, "handle is NULL")
    with pytest.raises(kvec.KvecError):
        sel.paged_decode(torch.zeros((2, 8, 128), dtype=torch.float16), c)
    q, k = torch.zeros((2, 8, 128), dtype=torch.float16), torch.zeros((2, 2, 128), dtype=torch.float16)
    refused(lambda: sel.rotate_append(q, k, k, torch.zeros(2, dtype=torch.int32), torch.zeros((4, 128)), c), BAD, "differs")


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(kvec.kvec_paged_scales) == 16


# ---------------------------------------------------------------- the definitions themselves

def test_e4m3_definition():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = every[~np.isnan(every)]
    assert np.array_equal(serving.e4m3(every), every)
    pos = np.unique(np.abs(every))
    mid = (pos[1:] + pos[:-1]) / 2
    eps = 1e-9
    assert np.array_equal(serving.e4m3(mid * (1 - eps)), pos[:-1]) and np.array_equal(serving.e4m3(mid * (1 + eps)), pos[1:])
    even = np.where(np.arange(len(mid)) % 2 == 0, pos[:-1], pos[1:])   # codes alternate: the even one of the two
    assert np.array_equal(serving.e4m3(mid), even) and np.array_equal(serving.e4m3(-mid), -even)
    assert serving.e4m3(1e9) == 448 and serving.e4m3(449.0) == 448 and serving.e4m3(0.0) == 0


def test_scales_and_reads():
    y = np.zeros((2, 128))
    y[1, 3] = -896.0
    assert serving.scale_of(y).tolist() == [2.0 ** -126, 2.0]
    k = np.arange(3 * 1 * 4 * 2, dtype=float).reshape(3, 1, 4, 2)
    a, b = serving.paged_read(k, -k, np.array([[2, 0], [1, -1]]), [6, 8], [3, 2], [0, 4, 8], 9, 5.0)
    assert np.array_equal(a[:4, 0], np.stack([k[2, 0, 3], k[0, 0, 0], k[0, 0, 1], 0 * k[0, 0, 0]]))   # slot 6 is past the length
    assert np.array_equal(b[4:8, 0], -np.stack([k[1, 0, 2], k[1, 0, 3], 0 * k[0, 0, 0], 0 * k[0, 0, 0]])) and np.all(a[8] == 5.0)
