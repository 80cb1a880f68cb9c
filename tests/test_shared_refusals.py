"""What kvec_shared_decode refuses, without a GPU, and its definition."""
import ctypes

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


def prefix(**over):
    p = dict(num_groups=2, max_pages=3, page_table=64, lens=128, cu_seqs=256)
    p.update(over)
    return kvec.kvec_shared_prefix(**p)


def refused(call, status, words):
    with pytest.raises(kvec.KvecError) as e:
        call()
    assert e.value.status == status and words in str(e.value), str(e.value)


@pytest.mark.parametrize("c,p,max_len,max_prefix,status,words", [
    (dict(dtype=3), {}, 64, 64, BAD, "dtype"), (dict(page_size=8), {}, 64, 64, UNSUPPORTED, "page_size"),
    (dict(lens=None), {}, 64, 64, BAD, "NULL"), ({}, None, 64, 64, BAD, "prefix is NULL"),
    ({}, {}, 0, 64, BAD, "max_len"), ({}, {}, 257, 64, BAD, "max_len"),
    ({}, {}, 64, 0, BAD, "max_prefix"), ({}, {}, 64, 193, BAD, "max_prefix"), ({}, {}, 64, -1, BAD, "max_prefix"),
    ({}, dict(num_groups=0), 64, 64, BAD, "num_groups"), ({}, dict(num_groups=65536), 64, 64, BAD, "num_groups"),
    ({}, dict(num_groups=-1), 64, 64, BAD, "num_groups"),
    ({}, dict(max_pages=0), 64, 64, BAD, "max_pages"), ({}, dict(max_pages=2 ** 14 + 1), 64, 64, BAD, "max_pages"),
    ({}, dict(max_pages=2 ** 31 - 1), 64, 64, BAD, "max_pages"),
    ({}, dict(page_table=None), 64, 64, BAD, "NULL"), ({}, dict(lens=None), 64, 64, BAD, "NULL"),
    ({}, dict(cu_seqs=None), 64, 64, BAD, "NULL"), ({}, dict(cu_seqs=2), 64, 64, BAD, "4-byte"),
    ({}, {}, 64, 64, BAD, "handle is NULL"), ({}, {}, 256, 192, BAD, "handle is NULL"),
])
def test_bad_calls(c, p, max_len, max_prefix, status, words):
    refused(lambda: kvec.kvec_shared_decode(None, 2, 16, cache(**c), None if p is None else prefix(**p), max_len, max_prefix,
                                            16, 256, 0), status, words)
    assert kvec.kvec_shared_decode_bytes(None, 2, 64, True) == 0


def selector(Hq=8, Hkv=2):
    s = kvec.KvecSelector.__new__(kvec.KvecSelector)
    s._torch, s.params, s.handle, s.device = torch, kvec.make_params(Hq, Hkv), None, torch.device("cpu")
    s._lib, s._decode_bytes, s._current = kvec.load(), {}, lambda index: 0
    return s


def tensors(groups=2):
    return dict(page_table=torch.zeros((groups, 3), dtype=torch.int32), lens=torch.zeros(groups, dtype=torch.int32),
                cu_seqs=torch.zeros(groups + 1, dtype=torch.int32))


@pytest.mark.parametrize("name,value", [
    ("page_table", torch.zeros(2, dtype=torch.int32)), ("page_table", torch.zeros((2, 3), dtype=torch.int64)),
    ("page_table", torch.zeros((2, 0), dtype=torch.int32)), ("page_table", torch.zeros((3, 2), dtype=torch.int32).t()),
    ("lens", torch.zeros(3, dtype=torch.int32)), ("lens", torch.zeros(2)), ("cu_seqs", torch.zeros(2, dtype=torch.int32)),
    ("cu_seqs", torch.zeros(6, dtype=torch.int32)[::2]), ("cu_seqs", torch.zeros(3, dtype=torch.int64)),
])
def test_the_binding_checks_a_prefix(name, value):
    kvec.SharedPrefix(**tensors())
    with pytest.raises(kvec.KvecError):
        kvec.SharedPrefix(**{**tensors(), name: value})


def test_the_binding_checks_a_call():
    sel = selector()
    k = torch.zeros((6, 2, 16, 128), dtype=BF)
    c = kvec.PagedCache(k, k.clone(), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    p, q = kvec.SharedPrefix(**tensors()), torch.zeros((2, 8, 128), dtype=BF)
    refused(lambda: sel.shared_decode(q, c, p), BAD, "handle is NULL")
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(out=q.float()), dict(max_len=2 ** 31), dict(max_prefix=2 ** 32 + 16),
                dict(max_len=-1), dict(max_prefix=49), dict(max_len=49)):
        with pytest.raises(kvec.KvecError) as e:
            sel.shared_decode(**{**dict(q=q, cache=c, prefix=p), **bad})
        assert "handle" not in str(e.value)
    e = torch.zeros((6, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    one = torch.ones((6, 2, 16))
    eight = kvec.PagedCache(e, e.clone(), c.page_table, c.lens, k_scales=one, v_scales=one.clone(), dtype=BF)
    refused(lambda: sel.shared_decode(q, eight, p), UNSUPPORTED, "16 bits")


    other = kvec.PagedCache(k.clone(), k.clone(), c.page_table, c.lens)
    refused(lambda: sel.shared_decode(q, eight, kvec.SharedPrefix(**tensors(), pool=other)), BAD, "handle is NULL")
    refused(lambda: sel.shared_decode(q, c, kvec.SharedPrefix(**tensors(), pool=other)), BAD, "same pages")
    refused(lambda: sel.shared_decode(q, c, kvec.SharedPrefix(**tensors(), pool=c)), BAD, "handle is NULL")
    with pytest.raises(kvec.KvecError):
        kvec.SharedPrefix(**tensors(), pool=eight)
    half = kvec.PagedCache(k.half(), k.half(), c.page_table, c.lens)
    refused(lambda: sel.shared_decode(q, eight, kvec.SharedPrefix(**tensors(), pool=half)), BAD, "dtype")


def test_bad_calls_over_eight_bits():
    scales = kvec.kvec_paged_scales(16, 32)
    call = lambda c=cache(), s=scales, pool=cache(), p=prefix(), most=64: kvec.kvec_shared_decode_quant(
        None, 2, 16, c, s, pool, p, 64, most, 16, 256, 0)
    for bad, words in ((dict(s=None), "k_scales"), (dict(s=kvec.kvec_paged_scales(8, 16)), "16-byte"), (dict(pool=None), "cache is NULL"),
                       (dict(pool=cache(dtype=kvec.KVEC_FP16)), "dtype"), (dict(pool=cache(k_pages=None)), "NULL"),
                       (dict(p=None), "prefix is NULL"), (dict(most=193), "max_prefix"), (dict(pool=cache(page_size=16), most=49), "max_prefix"),
                       ({}, "handle is NULL")):
        refused(lambda: call(**bad), BAD, words)
    assert kvec.kvec_shared_decode_quant_bytes(None, 2, 64, True) == 0


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(kvec.kvec_shared_prefix) == 8 + 3 * 8


def test_shared_decode_definition():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((2, 6, 2, 4, 8))
    q = rng.standard_normal((3, 4, 8))
    own, prefix = np.array([[3, -1], [1, 0], [2, -1]]), np.array([[5, 4]])
    w = np.zeros((6, 2, 4))
    out = serving.shared_decode(q, k, v, w, own, [2, 5, 3], 8, prefix, [6], [0, 2], 8, 0.3)
    # The same with the prefix's slots in front of each sequence's own, page by page where it fills its pages.
    full = serving.shared_decode(q, k, v, None, own, [2, 5, 3], 8, prefix, [8], [0, 2], 8, 0.3)
    joined = serving.paged_decode(q, k, v, None, np.array([[5, 4, 3, -1], [5, 4, 1, 0], [2, -1, -1, -1]]), [10, 13, 3], 16, 0, 0, 0.3)
    assert np.allclose(full, joined)
    kk, vv = np.concatenate([k[5], k[4][:, :2], k[3][:, :2]], 1), np.concatenate([v[5], v[4][:, :2], v[3][:, :2]], 1)
    e = np.exp(0.3 * kk[1] @ q[0, 3])
    assert np.allclose(out[0, 3], e @ vv[1] / e.sum())
    assert np.all(w[[4, 5]] == 0) and np.all(w[3, :, 2:] == 0) and np.all(w[3, :, :2] > 0) and w[2, :, :3].sum() > 3.99
