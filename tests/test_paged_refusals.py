"""What the paged-cache entry points refuse, without a GPU: the checks of a call's sizes come before the
handle's, so a call without a handle tells which check it met.  And the fp64 definitions against closed forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import serving
from paper_2606_29563_gb300 import build as kbuild
from paper_2606_29563_gb300 import kvec


@pytest.fixture(scope="module", autouse=True)
def lib():
    kbuild.build()
    return kvec.load()


def cache(**over):
    c = dict(dtype=kvec.KVEC_BF16, page_size=64, num_pages=10, max_pages=4, k_pages=4096, v_pages=8192, weights=16,
             page_table=64, lens=128)
    c.update(over)
    return kvec.kvec_paged_cache(**c)


def refused(call, status, words):
    with pytest.raises(kvec.KvecError) as e:
        call()
    assert e.value.status == status and words in str(e.value), str(e.value)


BAD_CACHES = [
    (dict(dtype=2), kvec.KVEC_ERR_INVALID_ARG, "dtype"),
    (dict(dtype=-1), kvec.KVEC_ERR_INVALID_ARG, "dtype"),
    (dict(page_size=0), kvec.KVEC_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=8), kvec.KVEC_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=48), kvec.KVEC_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=512), kvec.KVEC_ERR_UNSUPPORTED, "page_size"),
    (dict(num_pages=0), kvec.KVEC_ERR_INVALID_ARG, "num_pages"),
    (dict(max_pages=0), kvec.KVEC_ERR_INVALID_ARG, "max_pages"),
    (dict(max_pages=2 ** 14 + 1), kvec.KVEC_ERR_INVALID_ARG, "max_pages"),
    (dict(max_pages=2 ** 31 - 1), kvec.KVEC_ERR_INVALID_ARG, "max_pages"),
    (dict(k_pages=None), kvec.KVEC_ERR_INVALID_ARG, "NULL"),
    (dict(lens=None), kvec.KVEC_ERR_INVALID_ARG, "NULL"),
    (dict(v_pages=8), kvec.KVEC_ERR_INVALID_ARG, "16-byte"),
    (dict(weights=4), kvec.KVEC_ERR_INVALID_ARG, "16-byte"),
    (dict(page_table=2), kvec.KVEC_ERR_INVALID_ARG, "4-byte"),
]


@pytest.mark.parametrize("over,status,words", BAD_CACHES)
def test_bad_caches(over, status, words):
    c = cache(**over)
    refused(lambda: kvec.kvec_paged_decode(None, 1, 16, c, 64, 0, 0, 16, 16, 0), status, words)
    if "weights" not in over or over["weights"]:
        refused(lambda: kvec.kvec_paged_evict(None, 1, c, 16, 4, 64, 8, 0, 0, 16, 16), status, words)
    refused(lambda: kvec.kvec_rotate_append(None, rotate_args(), 1, None, c), status, words)


def rotate_args(**over):
    a = dict(dtype=kvec.KVEC_BF16, num_tokens=1, q=16, k=16, v=16, q_stride=4096, k_stride=1024, v_stride=1024, eps=1e-6,
             rot_dim=128, max_positions=10, rot_table=16, positions=16, q_out=32)
    a.update(over)
    return kvec.kvec_rotate_args(**a)


@pytest.mark.parametrize("over,words", [
    (dict(dtype=5), "dtype"), (dict(dtype=kvec.KVEC_FP16), "differs"), (dict(num_tokens=-1), "num_tokens"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(rot_dim=8), "rot_dim"), (dict(rot_dim=144), "rot_dim"), (dict(rot_dim=-16), "rot_dim"),
    (dict(interleaved=2), "interleaved"), (dict(rot_table=None), "rot_table"), (dict(max_positions=0), "max_positions"),
    (dict(q_stride=4), "strides"), (dict(k_stride=-8), "strides"), (dict(v_stride=1 << 41), "strides"),
    ({}, "handle is NULL"),
])
def test_bad_rotations(over, words):
    refused(lambda: kvec.kvec_rotate_append(None, rotate_args(**over), 1, None, cache()), kvec.KVEC_ERR_INVALID_ARG, words)


@pytest.mark.parametrize("args,words", [
    ((0, 0, 0), "max_len"), ((257, 0, 0), "max_len"), ((64, -1, 0), "window"), ((64, 0, -1), "sinks"), ((64, 0, 0), "handle"),
])
def test_bad_decodes(args, words):
    refused(lambda: kvec.kvec_paged_decode(None, 1, 16, cache(), *args, 16, 16, 0), kvec.KVEC_ERR_INVALID_ARG, words)
    assert kvec.kvec_paged_decode_bytes(None, 1, 64, True) == 0


@pytest.mark.parametrize("new_pages,max_len,budget,sinks,recent,words", [
    (4, 0, 8, 0, 0, "max_len"), (4, 300, 8, 0, 0, "max_len"), (4, 64, 0, 0, 0, "budget"), (4, 64, 2 ** 20 + 1, 0, 0, "budget"),
    (4, 64, 8, -1, 0, "sinks"), (4, 64, 8, 0, -1, "sinks"), (4, 64, 8, 5, 4, "sinks"),
    (4, 64, 2 ** 20, 2 ** 31 - 1, 2 ** 31 - 1, "sinks"), (0, 64, 8, 0, 0, "new_table"), (1, 256, 65, 0, 0, "new_table"),
    (4, 64, 8, 0, 0, "handle"),
])
def test_bad_evictions(new_pages, max_len, budget, sinks, recent, words):
    refused(lambda: kvec.kvec_paged_evict(None, 1, cache(), 16, new_pages, max_len, budget, sinks, recent, 16, 16),
            kvec.KVEC_ERR_INVALID_ARG, words)
    refused(lambda: kvec.kvec_paged_evict(None, 1, cache(weights=None), 16, 4, 64, 8, 0, 0, 16, 16),
            kvec.KVEC_ERR_INVALID_ARG, "weights")


def selector(Hq=8, Hkv=2):
    """The binding's own checks need no handle."""
    s = kvec.KvecSelector.__new__(kvec.KvecSelector)
    s._torch, s.params, s.handle, s.device = torch, kvec.make_params(Hq, Hkv), None, torch.device("cpu")
    s._lib, s._decode_bytes = kvec.load(), {}
    return s


def tensors(dtype=torch.bfloat16, Hkv=2, page=16, pages=6, batch=2):
    k = torch.zeros((pages, Hkv, page, 128), dtype=dtype)
    return dict(k_pages=k, v_pages=k.clone(), page_table=torch.zeros((batch, 3), dtype=torch.int32),
                lens=torch.zeros(batch, dtype=torch.int32), weights=torch.zeros((pages, Hkv, page)))


@pytest.mark.parametrize("name,value", [
    ("k_pages", torch.zeros((6, 2, 16, 128))), ("v_pages", torch.zeros((5, 2, 16, 128), dtype=torch.bfloat16)),
    ("v_pages", torch.zeros((6, 2, 16, 128), dtype=torch.float16)), ("page_table", torch.zeros((2, 3), dtype=torch.int64)),
    ("page_table", torch.zeros(2, dtype=torch.int32)), ("page_table", torch.zeros((3, 2), dtype=torch.int32).t()),
    ("lens", torch.zeros(3, dtype=torch.int32)), ("lens", torch.zeros(2)), ("weights", torch.zeros((6, 2, 8))),
    ("weights", torch.zeros((6, 2, 16), dtype=torch.float16)),
    ("k_pages", torch.zeros((6, 16, 2, 128), dtype=torch.bfloat16).transpose(1, 2)),
])
def test_the_binding_checks_a_cache(name, value):
    with pytest.raises(kvec.KvecError):
        kvec.PagedCache(**{**tensors(), name: value})


def test_the_binding_checks_a_call():
    sel, c = selector(), kvec.PagedCache(**tensors())
    bf = torch.bfloat16
    for q in (torch.zeros((2, 8, 128)), torch.zeros((1, 8, 128), dtype=bf), torch.zeros((2, 4, 128), dtype=bf),
              torch.zeros((2, 8, 256), dtype=bf)[..., ::2]):
        with pytest.raises(kvec.KvecError):
            sel.paged_decode(q, c)
    with pytest.raises(kvec.KvecError):
        selector(8, 4).paged_decode(torch.zeros((2, 8, 128), dtype=bf), c)       # other KV heads than the pages
    for table in (torch.zeros((2, 3)), torch.zeros((1, 3), dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32).t()):
        with pytest.raises(kvec.KvecError):
            sel.paged_evict(c, table, 16)
    q, k = torch.zeros((2, 8, 128), dtype=bf), torch.zeros((2, 2, 128), dtype=bf)
    pos, tab = torch.zeros(2, dtype=torch.int32), torch.zeros((4, 128))
    for bad in (dict(q=q.float()), dict(k=k[:1]), dict(v=k.half()), dict(positions=pos.long()), dict(rot_table=tab.double()),
                dict(q=torch.zeros((2, 8, 256), dtype=bf)[..., :128]), dict(q_norm=torch.zeros(128)),
                dict(cu_tokens=torch.zeros(3)), dict(cu_tokens=torch.zeros(2, dtype=torch.int32)), dict(q_out=q.float())):
        with pytest.raises(kvec.KvecError):
            sel.rotate_append(**{**dict(q=q, k=k, v=k, positions=pos, rot_table=tab, cache=c), **bad})


# ---------------------------------------------------------------- the definitions themselves

def test_rotation_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 1, 1, 128))
    ang = lambda p: p * 10000.0 ** (-np.arange(0, 128, 2) / 128)
    rows = lambda p: np.concatenate([np.cos(ang(p)), np.sin(ang(p))])[None]
    for inter in (False, True):
        a = serving.rotate(x, None, 0.0, rows(7.0), inter)
        assert np.allclose((a * a).sum(), (x * x).sum())
        dot = lambda p, q: (serving.rotate(x, None, 0.0, rows(p), inter) * serving.rotate(y, None, 0.0, rows(q), inter)).sum()
        assert np.isclose(dot(3.0, 11.0), dot(100.0, 108.0)) and np.isclose(dot(5.0, 5.0), (x * y).sum())
    n = serving.rotate(x, np.full(128, 2.0), 0.0, None, False)
    assert np.isclose((n * n).mean(), 4.0)


def test_decode_definition():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 5, 2, 4, 8))
    table, q = np.array([[3, 1, -1]]), rng.standard_normal((1, 4, 8))
    w = np.zeros((5, 2, 4))
    out = serving.paged_decode(q, k, v, w, table, [7], 12, 0, 0, 0.3)
    kk = np.concatenate([k[3], k[1][:, :3]], 1)
    vv = np.concatenate([v[3], v[1][:, :3]], 1)
    for hq in range(4):
        e = np.exp(0.3 * kk[hq // 2] @ q[0, hq])
        assert np.allclose(out[0, hq], e @ vv[hq // 2] / e.sum())
    assert np.allclose(w.sum(), 4) and np.all(w[[0, 2, 4]] == 0) and np.all(w[1, :, 3] == 0)
    # A window of one slot and no first ones: that slot's value.
    assert np.allclose(serving.paged_decode(q, k, v, None, table, [7], 12, 1, 0, 0.3)[0, 0], v[1, 0, 2])
    # Zero queries: the mean of what is visible.
    m = serving.paged_decode(0 * q, k, v, None, table, [7], 12, 2, 1, 0.3)
    assert np.allclose(m[0, 3], (v[3, 1, 0] + v[1, 1, 1] + v[1, 1, 2]) / 3)


def test_evict_definition():
    w = np.zeros((4, 1, 4))
    w[0, 0], w[2, 0] = [5, 1, 9, 9], [0, 9, 3, 2]
    k = np.arange(4 * 4 * 2, dtype=float).reshape(4, 1, 4, 2)
    v, k0 = k + 100, k.copy()
    lens, kept = serving.evict(k, v, w, np.array([[2, 0]]), [8], np.array([[3, -1]]), 8, 4, 1, 1)
    # Slots' weights: 0 9 3 2 | 5 1 9 9; slot 0 and slot 7 stay, then 1 and 6 (both 9, before 4 with 5).
    assert lens.tolist() == [4] and kept[0, 0].tolist() == [0, 1, 6, 7]
    assert np.array_equal(k[3, 0], k0[[2, 2, 0, 0], 0, [0, 1, 2, 3]]) and w[3, 0].tolist() == [0, 9, 9, 9]
    assert np.array_equal(k[:3], k0[:3])


def test_struct_layouts_match_the_header():
    # Natural alignment: four ints and five pointers; 8 + 3 pointers + 3 int64 + 2 pointers + float and 3 ints + 4 pointers.
    assert ctypes.sizeof(kvec.kvec_paged_cache) == 4 * 4 + 5 * 8
    assert ctypes.sizeof(kvec.kvec_rotate_args) == 8 + 3 * 8 + 3 * 8 + 2 * 8 + 16 + 4 * 8


# ---------------------------------------------------------------- prefill attention

@pytest.mark.parametrize("over,words", [
    (dict(dtype=2), "dtype"), (dict(batch=0), "batch"), (dict(batch=70000), "batch"), (dict(window=-1), "window"),
    (dict(sinks=-1), "window"), (dict(cu_q=None), "NULL"), (dict(cu_q=[1, 5]), "cu_q[0]"), (dict(cu_k=[2, 5]), "cu_q[0]"),
    (dict(cu_q=[0, -1]), "-1 queries"), (dict(cu_k=[0, 2 ** 20 + 1]), "keys"), (dict(cu_q=[0, 2 ** 31 - 1]), "queries"),
    ({}, "handle is NULL"),
])
def test_bad_prefills(over, words):
    a = dict(dtype=kvec.KVEC_FP16, batch=1, window=0, sinks=0, cu_q=[0, 5], cu_k=[0, 5])
    a.update(over)
    host = {n: None if a[n] is None else (ctypes.c_int32 * len(a[n]))(*a[n]) for n in ("cu_q", "cu_k")}
    at = {n: None if x is None else ctypes.addressof(x) for n, x in host.items()}
    refused(lambda: kvec.kvec_prefill_attention(None, a["dtype"], a["batch"], at["cu_q"], 16, at["cu_k"], 16, 16, 16, 16,
                                                a["window"], a["sinks"], 16, None), kvec.KVEC_ERR_INVALID_ARG, words)


def test_the_binding_checks_a_prefill():
    sel, bf = selector(), torch.bfloat16
    q, k = torch.zeros((5, 8, 128), dtype=bf), torch.zeros((5, 2, 128), dtype=bf)
    cu = torch.tensor([0, 5], dtype=torch.int32)
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(k=torch.zeros((5, 4, 128), dtype=bf)), dict(v=k[:, :, :64]),
                dict(q=torch.zeros((5, 8, 256), dtype=bf)[..., :128]), dict(cu_q_host=cu.long()), dict(cu_q_dev=cu[:1]),
                dict(cu_q_host=torch.tensor([0, 6], dtype=torch.int32)), dict(v=k[:4]), dict(out=q.float()),
                dict(lse=torch.zeros(5, 8, dtype=torch.float64)), dict(lse=torch.zeros(5, 2))):
        with pytest.raises(kvec.KvecError):
            sel.prefill_attention(**{**dict(q=q, k=k, v=k, cu_q_host=cu, cu_q_dev=cu), **bad})


def test_prefill_definition():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((6, 2, 8)), rng.standard_normal((9, 1, 8)), rng.standard_normal((9, 1, 8))
    out, lse = serving.prefill(q, k, v, [0, 4, 6], [0, 8, 9], 0, 0, 0.4)
    e = np.exp(0.4 * k[:6, 0] @ q[1, 1])                     # row 1 of the first sequence is at position 5
    assert np.allclose(out[1, 1], e @ v[:6, 0] / e.sum()) and np.isclose(lse[1, 1], np.log(e.sum()))
    assert np.all(out[4] == 0) and np.all(np.isneginf(lse[4]))   # two queries, one key: the first sees nothing
    assert np.allclose(out[5], v[8]) and np.allclose(lse[5, 0], 0.4 * q[5, 0] @ k[8, 0])
    mean, _ = serving.prefill(0 * q, k, v, [0, 4, 6], [0, 8, 9], 2, 1, 0.4)
    assert np.allclose(mean[3, 0], (v[0, 0] + v[6, 0] + v[7, 0]) / 3)


def test_the_binding_remembers_few_sizes():
    # A loop that passes the longest length of each step meets a new bound every time.
    sel = selector()
    sel._current = lambda index: 0
    c = kvec.PagedCache(**{**tensors(), "page_table": torch.zeros((2, 2000), dtype=torch.int32)})
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    for n in range(1, 3000):
        refused(lambda: sel.paged_decode(q, c, max_len=n), kvec.KVEC_ERR_INVALID_ARG, "handle is NULL")
    assert 1 <= len(sel._decode_bytes) <= 256


@pytest.mark.parametrize("far", [2 ** 31, 2 ** 32, 2 ** 32 + 16, 2 ** 40])
def test_the_binding_refuses_sizes_past_32_bits(far):
    # Their lower 32 bits would count: 2^32 as no window, 2^32 + 16 as 16.
    sel, c = selector(), kvec.PagedCache(**tensors())
    sel._current = lambda index: 0
    bf, cu = torch.bfloat16, torch.tensor([0, 2], dtype=torch.int32)
    q, k, table = torch.zeros((2, 8, 128), dtype=bf), torch.zeros((2, 2, 128), dtype=bf), torch.zeros((2, 3), dtype=torch.int32)
    for bad in ("max_len", "window", "sinks"):
        refused(lambda: sel.paged_decode(q, c, **{bad: far}), kvec.KVEC_ERR_INVALID_ARG, "2^31")
    for bad in ("max_len", "sinks", "recent"):
        refused(lambda: sel.paged_evict(c, table, 16, **{bad: far}), kvec.KVEC_ERR_INVALID_ARG, "2^31")
    for bad in ("window", "sinks"):
        refused(lambda: sel.prefill_attention(q, k, k, cu, cu, **{bad: far}), kvec.KVEC_ERR_INVALID_ARG, "2^31")
    # The largest that is taken reaches the library.
    refused(lambda: sel.paged_decode(q, c, window=2 ** 31 - 1, sinks=2 ** 31 - 1), kvec.KVEC_ERR_INVALID_ARG, "handle is NULL")
