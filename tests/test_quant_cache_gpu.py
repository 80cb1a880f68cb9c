"""GPU parity of the operators over a paged cache of 8 bits (kvec_rotate_append_quant, kvec_paged_decode_quant,
kvec_paged_evict_quant, kvec_paged_read) with their definitions in fp64 (oracle/serving.py).

Tolerances.  u is half a step of the 16-bit type relative to the value (bf16 2^-8, fp16 2^-11).
* A row's scale: fp32 arithmetic, the rotated row is off by up to 4e-6 of its largest value (as in the tests of the
  16-bit cache), and one rounding of the quotient: 5e-6 relative.
* Stored numbers: half a step of e4m3 beside z = y / s (2^-4 |z|, 2^-10 below 2^-6), and what z is off by: 448 times
  (4e-6 + 5e-6).  The steps beside a power of two are covered, as 2^-4 |z| is half the wider step.
* Decode outputs: keys and values are the exact products; logits and sums as for the 16-bit cache, 2e-5 of the largest
  value; a weight times its value's scale counts with 2^-22 of itself and 2^-39 of the largest; then one rounding to
  the type: u |ref| + (2^-22 + n 2^-39 + 2e-5) max|v|.
* Accumulated weights: 2e-5 of the step's sum, and a rounding of the new value.
* Rows read back: the product in fp32 (2^-24) and one rounding to the type, u + 2^-23; below fp16's normal numbers half of
  their step, 2^-25.
* Kept slots, lengths, and moved numbers and scales are equal, byte for byte.
"""
import numpy as np
import pytest
import torch

from oracle import serving
from paper_2606_29563_gb300 import kvec

pytestmark = pytest.mark.gpu
D = 128
E4M3 = torch.float8_e4m3fn
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2606_29563_gb300 import build as kbuild
    kbuild.build()


_SELECTORS = {}


def selector(Hq, Hkv):
    key = (Hq, Hkv)
    if key not in _SELECTORS:
        _SELECTORS[key] = kvec.KvecSelector(kvec.make_params(Hq, Hkv, num_ext_heads=1, max_batch=300, max_seqlen=64, max_layers=1))
    return _SELECTORS[key]


def f64(x):
    return None if x is None else x.detach().cpu().to(torch.float64).numpy()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def raw(x):
    return x.view(torch.uint8).cpu()


def values(pages, scales):
    return f64(pages) * f64(scales)[..., None]


def make_cache(lens, Hkv, page, dtype, gen, max_pages=None, spare=0, weights=True, spread=0.5):
    """Shuffled pages for the sequences' slots, -1 past them; in every slot past a length NaN numbers and scales."""
    counts = [-(-max(n, 0) // page) for n in lens]
    max_pages = max(1, max(counts)) if max_pages is None else max_pages
    pages = sum(counts) + spare + 1
    perm = torch.randperm(pages, generator=gen).tolist()
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = torch.tensor(perm[at:at + c], dtype=torch.int32)
        at += c
    used = torch.zeros((pages, page), dtype=torch.bool)
    for s, n in enumerate(lens):
        for j in range(max(n, 0)):
            used[table[s, j // page], j % page] = True
    hole = ~used[:, None, :].expand(pages, Hkv, page)
    parts = []
    for bad in (float("nan"), float("inf")):
        x = torch.randn((pages, Hkv, page, D), generator=gen) * (torch.randn((pages, Hkv, page, 1), generator=gen) * spread).exp()
        scale = x.abs().amax(-1) / 448
        x = (x / scale[..., None]).to(E4M3)
        raw_x = x.view(torch.uint8)
        raw_x[hole] = 0x7f
        scale[hole] = bad
        parts += [x.cuda(), scale.cuda()]
    w = torch.randn((pages, Hkv, page), generator=gen).exp() if weights else None
    cache = kvec.PagedCache(parts[0], parts[2], table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                            None if w is None else w.cuda(), k_scales=parts[1], v_scales=parts[3], dtype=dtype)
    return cache, perm[at:]


def rot_table(positions, rot, theta=10000.0):
    inv = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


# ---------------------------------------------------------------- rotate_append

def check_stored(numbers, scales, ref, name):
    """Rows ref [...][d] in fp64 against numbers (e4m3) and scales."""
    want = serving.scale_of(ref)
    got = f64(scales)
    assert np.all(np.abs(got - want) <= 5e-6 * want), f"{name}: a scale is off"
    z = ref / got[..., None]
    tol = np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -10) + 448 * 9e-6
    bad = ~(np.abs(f64(numbers) - z) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} numbers off"


def check_append(cache, before, table, lens, cu, positions, most, k, v):
    """The cache after an append against `before` (clones of pages, scales, weights) and the rotated rows k, v."""
    num_pages, page = cache.k_pages.shape[0], cache.page_size
    written = torch.zeros((num_pages, page), dtype=torch.bool)
    for s in range(len(lens)):
        for t in range(cu[s], cu[s + 1]):
            at = serving.place(table[s], lens[s] - (cu[s + 1] - t), page, num_pages) if 0 <= positions[t] < most else None
            if at is None:
                continue
            written[at[0], at[1]] = True
            check_stored(cache.k_pages[at[0], :, at[1]], cache.k_scales[at[0], :, at[1]], k[t], f"key {t}")
            check_stored(cache.v_pages[at[0], :, at[1]], cache.v_scales[at[0], :, at[1]], v[t], f"value {t}")
    left = ~written[:, None, :].expand(cache.k_scales.shape)
    for got, old in zip((cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales), before):
        assert torch.equal(raw(got).reshape(*left.shape, -1)[left], raw(old).reshape(*left.shape, -1)[left])
    if cache.weights is not None:
        assert torch.equal(cache.weights.cpu()[left], before[4].cpu()[left]) and torch.all(cache.weights.cpu()[~left] == 0)


def clones(cache):
    return [None if x is None else x.clone() for x in (cache.k_pages, cache.v_pages, cache.k_scales, cache.v_scales, cache.weights)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,new,held,page,rot,interleaved,norm", [
    (4, 4, [1], [0], 16, 128, False, True),
    (32, 8, [1, 1, 1], [15, 16, 700], 16, 128, False, True),
    (28, 4, [3, 0, 17, 1], [0, 5, 31, 64], 32, 64, True, False),
    (8, 1, [40, 300], [100, 0], 64, 16, True, True),
    (7, 7, [5, 6], [2, 3], 256, 0, False, True),
    (5, 5, [130], [1000], 128, 96, False, False),
])
def test_append(dtype, Hq, Hkv, new, held, page, rot, interleaved, norm):
    gen = torch.Generator().manual_seed(Hq * 100 + page + rot)
    lens = [a + b for a, b in zip(new, held)]
    cache, _ = make_cache(lens, Hkv, page, dtype, gen)
    T = sum(new)
    qkv = (torch.randn((T, Hq + 2 * Hkv, D), generator=gen) * 3).to(dtype).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    positions = torch.tensor([h + i for n, h in zip(new, held) for i in range(n)], dtype=torch.int32)
    tab = rot_table(max(lens), rot) if rot else None
    norms = [(torch.randn(D, generator=gen) * 0.3 + 1).to(dtype).cuda() if norm else None for _ in range(2)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = f64(tab)[positions.numpy()] if rot else None
    ref_q = serving.rotate(f64(q), f64(norms[0]), 1e-6, rows, interleaved)
    ref_k = serving.rotate(f64(k), f64(norms[1]), 1e-6, rows, interleaved)
    before = clones(cache)
    k_out = torch.empty((T, Hkv, D), dtype=dtype, device="cuda")
    one_each = new == [1] * len(new)
    q_out, k_got = selector(Hq, Hkv).rotate_append(
        q, k, v, positions.cuda(), None if tab is None else tab.cuda(), cache,
        None if one_each else torch.from_numpy(cu).cuda(), q_norm=norms[0], k_norm=norms[1], interleaved=interleaved,
        k_out=k_out)
    torch.cuda.synchronize()
    for got, ref in ((q_out, ref_q), (k_got, ref_k)):
        assert np.all(np.abs(f64(got) - ref) <= half_step(dtype) * np.abs(ref) + 4e-6 * np.abs(ref).max(axis=-1, keepdims=True))
    check_append(cache, before, cache.page_table.cpu().numpy(), lens, cu, positions.tolist(), max(lens), ref_k, f64(v))


def test_padding_rows_and_missing_pages_are_left_alone():
    dtype, Hq, Hkv, page = torch.bfloat16, 8, 2, 16
    gen = torch.Generator().manual_seed(11)
    cache, _ = make_cache([20, 3, 9], Hkv, page, dtype, gen, max_pages=2)
    table = cache.page_table.clone()
    table[0, 1], table[2, 0] = 10 ** 6, -7
    lens = [20, 3, 40]
    cache = kvec.PagedCache(cache.k_pages, cache.v_pages, table, torch.tensor(lens, dtype=torch.int32).cuda(), cache.weights,
                            k_scales=cache.k_scales, v_scales=cache.v_scales, dtype=dtype)
    T, cu = 16, [0, 6, 8, 12]
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=gen).to(dtype).cuda()
    positions = torch.tensor([14, 15, 16, 17, 18, 19, -1, 2, 36, 37, 38, 39, 0, 0, 0, 0], dtype=torch.int32)
    tab = rot_table(38, 128)
    rows = f64(tab)[np.clip(positions.numpy(), 0, 37)]
    ref_k = serving.rotate(f64(x[:, Hq:Hq + Hkv]), None, 1e-6, rows, False)
    before = clones(cache)
    q_out = torch.full((T, Hq, D), 77.0, dtype=dtype, device="cuda")
    selector(Hq, Hkv).rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], positions.cuda(), tab.cuda(), cache,
                                    torch.tensor(cu, dtype=torch.int32).cuda(), q_out=q_out)
    torch.cuda.synchronize()
    left = [t for t in range(T) if t >= 12 or not 0 <= positions[t] < 38]
    assert torch.all(q_out[left] == 77.0)
    check_append(cache, before, table.cpu().numpy(), lens, cu, positions.tolist(), 38, ref_k, f64(x[:, Hq + Hkv:]))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_at_the_ends_of_the_range(dtype):
    # Zeros, the type's least and largest numbers, one large value among small ones; rows with infinities and NaN read as NaN.
    gen = torch.Generator().manual_seed(3)
    cache, _ = make_cache([9], 1, 16, dtype, gen)
    rows = torch.randn((9, 2, D), generator=gen)
    rows[0] = 0.0
    rows[1] = 0.0
    rows[1, :, 5] = 5.9604644775390625e-8 if dtype == torch.float16 else 9.183549615799121e-41   # subnormal
    rows[2] *= torch.finfo(dtype).tiny
    rows[3] = torch.finfo(dtype).max
    rows[4] *= 1e-4
    rows[4, :, 17] = 1e4
    rows[5, 0, 3], rows[5, 1, 99] = float("inf"), float("-inf")
    rows[6, 0, 0], rows[6, 1, 127] = float("nan"), float("nan")
    rows[7] = -1.0
    x = rows.to(dtype).cuda()
    sel, pos, cu = selector(1, 1), torch.arange(9, dtype=torch.int32).cuda(), torch.tensor([0, 9], dtype=torch.int32).cuda()
    sel.rotate_append(x[:, :1], x[:, :1], x[:, 1:], pos, None, cache, cu)
    k, v = sel.paged_read(cache, cu, 9)
    torch.cuda.synchronize()
    fine = [0, 1, 2, 3, 4, 7, 8]
    at = int(cache.page_table[0, 0])
    for pages, scales, src in ((cache.k_pages, cache.k_scales, x[:, :1]), (cache.v_pages, cache.v_scales, x[:, 1:])):
        check_stored(pages[at, 0, fine], scales[at, 0, fine], f64(src)[fine, 0], "row")
        assert torch.all(pages[at, 0, [0]].float() == 0) and float(scales[at, 0, 0]) == 2.0 ** -126
        assert torch.all(pages[at, 0, 3].float() == 448)
    for got in (k, v):
        assert torch.all(torch.isnan(got[5:7])) and torch.all(torch.isfinite(got[fine]))


@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 1333), (8, 2, 1334), (32, 8, 1250), (32, 8, 1251), (28, 4, 3333), (28, 4, 3334), (40, 8, 14285), (40, 8, 14286)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_on_both_sides_of_the_layout_rule(Hq, Hkv, T, interleaved):
    # Every layout stores the same bytes as a few tokens at a time: 16000, 60000, 120000 and 800000 rows.
    gen = torch.Generator(device="cuda").manual_seed(T)
    dtype, page, new = torch.bfloat16, 32, [T // 3, T - T // 3]
    counts = [-(-n // page) for n in new]
    table = torch.full((2, max(counts)), -1, dtype=torch.int32)
    perm = torch.randperm(sum(counts), generator=torch.Generator().manual_seed(T)).to(torch.int32)
    table[0, :counts[0]], table[1, :counts[1]] = perm[:counts[0]], perm[counts[0]:]
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((2, D), generator=gen, device="cuda") * 0.2 + 1).to(dtype)
    pos = torch.cat([torch.arange(n) for n in new]).int().cuda()
    tab = rot_table(max(new), 128).cuda()
    sel, got = selector(Hq, Hkv), []
    for step in (T, 97):
        k, v = (torch.zeros((sum(counts), Hkv, page, D), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
        weights, ks, vs = (torch.ones((sum(counts), Hkv, page), device="cuda") for _ in range(3))
        q = torch.empty((T, Hq, D), dtype=dtype, device="cuda")
        for t0 in range(0, T, step):
            t1 = min(t0 + step, T)
            cu = torch.tensor([0, new[0], T]).clamp(t0, t1) - t0
            held = torch.tensor([min(t1, new[0]), max(t1 - new[0], 0)], dtype=torch.int32).cuda()
            sel.rotate_append(x[t0:t1, :Hq], x[t0:t1, Hq:Hq + Hkv], x[t0:t1, Hq + Hkv:], pos[t0:t1], tab,
                              kvec.PagedCache(k, v, table.cuda(), held, weights, k_scales=ks, v_scales=vs, dtype=dtype),
                              cu.int().cuda(), q_norm=w[0], k_norm=w[1], q_out=q[t0:t1], interleaved=interleaved)
        got.append((q, raw(k), raw(v), ks, vs, weights))
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- paged_decode

def check_decode(sel, q, cache, lens, max_len=None, window=0, sinks=0, u=None):
    dtype = q.dtype
    u = half_step(dtype) if u is None else u
    max_len = cache.capacity if max_len is None else max_len
    with np.errstate(invalid="ignore"):
        kp, vp = values(cache.k_pages, cache.k_scales), values(cache.v_pages, cache.v_scales)
    w0 = f64(cache.weights)
    w = None if w0 is None else w0.copy()
    ref = serving.paged_decode(f64(q), kp, vp, w, cache.page_table.cpu().numpy(), lens, max_len, window, sinks, 1 / np.sqrt(D))
    out = sel.paged_decode(q, cache, max_len, window=window, sinks=sinks)
    kvec.kvec_sync_status(sel.handle)
    got = f64(out)
    n = max(1, min(max_len, max(lens)))
    vmax = np.abs(vp[np.isfinite(vp)]).max(initial=0.0)
    tol = u * np.abs(ref) + (2.0 ** -22 + n * 2.0 ** -39 + 2e-5) * vmax
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} outputs off, by up to {np.nanmax(np.abs(got - ref)):.3e}; rows {np.argwhere(bad.any(-1))[:8].tolist()}"
    if w is not None:
        gw = f64(cache.weights)
        bad = ~(np.abs(gw - w) <= 2e-5 * (w - w0) + 2.0 ** -24 * np.abs(w) + 1e-9)
        assert not bad.any(), f"{bad.sum()} weights off, by up to {np.nanmax(np.abs(gw - w)):.3e}: {np.argwhere(bad)[:6].tolist()}"
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,page,lens,weights", [
    (4, 4, 16, [1], True),
    (8, 4, 16, [15, 16, 17], True),
    (32, 8, 32, [512], True),
    (28, 4, 64, [200, 0, 137, 1], True),
    (16, 2, 128, [513, 300], False),
    (8, 1, 256, [1000, 255, 256, 257], True),
    (32, 8, 16, [4097], True),
    (28, 4, 64, [3000, 5, 0, 1777, 64], True),
])
def test_decode_matches_the_definition(dtype, Hq, Hkv, page, lens, weights):
    gen = torch.Generator().manual_seed(sum(lens) + Hq)
    cache, _ = make_cache(lens, Hkv, page, dtype, gen, weights=weights)
    q = torch.randn((len(lens), Hq, D), generator=gen).to(dtype).cuda()
    out = check_decode(selector(Hq, Hkv), q, cache, lens)
    for s, n in enumerate(lens):
        assert n or torch.all(out[s] == 0)
    check_decode(selector(Hq, Hkv), q, cache, lens)   # again, on the grown weights


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 3), (16, 4), (17, 16), (64, 20), (5000, 7), (333, 400)])
@pytest.mark.parametrize("lens", [[700, 1, 16, 399, 0], [2500]])
def test_window_and_sinks(lens, window, sinks):
    gen = torch.Generator().manual_seed(window * 31 + sinks)
    dtype, page = torch.bfloat16, 32
    cache, _ = make_cache(lens, 4, page, dtype, gen)
    for s, n in enumerate(lens):
        for j in range(min(sinks, n), max(0, n - window)):   # pages that the window has left behind
            at = int(cache.page_table[s, j // page])
            cache.k_pages.view(torch.uint8)[at, :, j % page] = 0x7f
            cache.v_pages.view(torch.uint8)[at, :, j % page] = 0xff
            cache.k_scales[at, :, j % page] = float("inf") if j % 2 else float("nan")
            cache.v_scales[at, :, j % page] = float("nan") if j % 2 else float("inf")
    q = torch.randn((len(lens), 12, D), generator=gen).to(dtype).cuda()
    check_decode(selector(12, 4), q, cache, lens, window=window, sinks=sinks)


@pytest.mark.parametrize("batch,scale,Hq,Hkv", [(3, 1, 32, 8), (75, 1, 8, 8), (290, 2, 8, 4), (70, 9, 28, 4), (60, 40, 8, 4)])
def test_batches_on_every_path(batch, scale, Hq, Hkv):
    # Clusters of CTAs, a CTA a pair, shares of the list of all blocks.
    gen = torch.Generator().manual_seed(batch * scale + Hq)
    lens = [scale * (0, 1, 15, 16, 17, 63, 64, 65, 128, 130, 255, 257, 31, 7, 300, 48)[(5 * b + b // 16) % 16] for b in range(batch)]
    if scale == 40:
        lens = [600 + (37 * b) % 100 for b in range(batch)]
    cache, _ = make_cache(lens, Hkv, 16, torch.bfloat16, gen)
    q = torch.randn((batch, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    check_decode(selector(Hq, Hkv), q, cache, lens)


def test_max_len_and_missing_pages():
    gen = torch.Generator().manual_seed(3)
    lens, dtype = [70, 70, 70], torch.float16
    cache, _ = make_cache(lens, 2, 16, dtype, gen)
    cache.page_table[1, 2] = -1
    cache.page_table[2, 0] = 2 ** 30
    q = torch.randn((3, 8, D), generator=gen).to(dtype).cuda()
    for max_len in (80, 33):
        check_decode(selector(8, 2), q, cache, lens, max_len=max_len)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [40, 3000])
def test_scales_of_any_size(dtype, n):
    # Values' scales over sixty powers of two in turn up and down the sequence, zero, and negative; large and small queries.
    # (Outputs are rounded to the type last: ones past its range are not asked for.)
    gen = torch.Generator().manual_seed(n)
    cache, _ = make_cache([n, n, n], 2, 16, dtype, gen, spread=0.1)
    most = 8.0 if dtype == torch.float16 else 2.0 ** 40
    for s, order in enumerate((1, -1, 0)):
        for j in range(n):
            at, ofs = int(cache.page_table[s, j // 16]), j % 16
            e = order * (60.0 * j / n - 30.0) if order else 60.0 * (j * 7 % n) / n - 30.0
            cache.v_scales[at, :, ofs] *= 2.0 ** min(e, np.log2(most)) * (0.0 if j % 11 == 5 else -1.0 if j % 5 == 3 else 1.0)
    q = torch.randn((3, 8, D), generator=gen)
    q[1] *= 1e-3
    q[2, :, 0] *= 100
    check_decode(selector(8, 2), q.to(dtype).cuda(), cache, [n, n, n])


# Each output against its own size: sum_j p_j |s_j v8_j|, not the largest value in the cache.  A weight times its value's scale
# counts but for 2^-22 of itself, or 2^-39 of the head's largest such product: with sum_j p_j |s_j| for that one, n slots
# and numbers up to 448, n 448 2^-39 of it.  Then the logits' 2e-5, and the rounding to the type (fp16 below its normal numbers half
# of their step, 2^-25).

def check_each_output(sel, q, cache, lens):
    kp, vp = values(cache.k_pages, cache.k_scales), values(cache.v_pages, cache.v_scales)
    scales = np.broadcast_to(np.abs(f64(cache.v_scales))[..., None], vp.shape)
    ref, size, top = (serving.paged_decode(f64(q), kp, x, None, cache.page_table.cpu().numpy(), lens, cache.capacity, 0, 0,
                                           1 / np.sqrt(D)) for x in (vp, np.abs(vp), scales))
    out = f64(sel.paged_decode(q, cache))
    kvec.kvec_sync_status(sel.handle)
    n = max(lens)
    tol = half_step(q.dtype) * np.abs(ref) + (2.0 ** -22 + 2e-5) * size + n * 448 * 2.0 ** -39 * top
    tol += 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    past = np.abs(ref) >= 2.0 * torch.finfo(q.dtype).max      # rounded to the type, these are infinite
    assert np.array_equal(out[past], np.sign(ref[past]) * np.inf)
    bad = ~(np.abs(out - ref) <= tol) & ~past
    assert not bad.any(), f"{bad.sum()} outputs off, by up to {np.abs((out - ref) / size)[bad].max():.3e} of their size"


def set_slot(cache, s, j, key, value_scale):
    """Slot j of sequence s: a key of `key` in column 0 and zeros, and a factor on its value's scale."""
    at, ofs = int(cache.page_table[s, j // cache.page_size]), j % cache.page_size
    numbers = torch.zeros(D)
    numbers[0] = 1.0
    cache.k_pages.view(torch.uint8)[at, :, ofs] = numbers.to(E4M3).view(torch.uint8).cuda()
    cache.k_scales[at, :, ofs] = key
    cache.v_scales[at, :, ofs] *= value_scale


ON_EVERY_PATH = [(8, 2, [40]), (8, 2, [700, 1]), (28, 4, [9000]), (8, 4, [600 + (37 * b) % 100 for b in range(60)])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,lens", ON_EVERY_PATH)
@pytest.mark.parametrize("where", ["before", "behind", "between"])
def test_a_large_scale_without_weight_costs_the_others_nothing(dtype, Hq, Hkv, lens, where):
    # Some slots' scales are 2^40 times the others', their logits 104 (base 2) below: what they add is 2^-64 of the rest.
    gen = torch.Generator().manual_seed(sum(lens) + len(where))
    cache, _ = make_cache(lens, Hkv, 32, dtype, gen, weights=False)
    for s, n in enumerate(lens):
        few = min(n // 3, 100)
        for j in {"before": range(few), "behind": range(n - few, n), "between": range(3, n, max(7, n // 60))}[where]:
            set_slot(cache, s, j, -104.0, 2.0 ** 40)
    q = torch.randn((len(lens), Hq, D), generator=gen)
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    check_each_output(selector(Hq, Hkv), q.to(dtype).cuda(), cache, lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,lens", ON_EVERY_PATH)
@pytest.mark.parametrize("rise", [60.0, 90.0, -90.0])
def test_weights_and_scales_that_make_up_for_each_other(dtype, Hq, Hkv, lens, rise):
    # Logits that rise (or fall) along the sequence by so many powers of two, scales that fall by as many: every slot adds as much
    # as every other, whatever maximum the weights refer to.  (The logits' five roundings are off by 5 2^-24 90 ln 2 = 1.9e-5 at most.)
    gen = torch.Generator().manual_seed(sum(lens) + int(rise))
    cache, _ = make_cache(lens, Hkv, 32, dtype, gen, weights=False, spread=0.1)
    for s, n in enumerate(lens):
        for j in range(n):
            x = rise * (j + 1) / n
            set_slot(cache, s, j, x, 2.0 ** (max(rise, 0.0) - x - 4.0))
    q = torch.zeros((len(lens), Hq, D))
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    check_each_output(selector(Hq, Hkv), q.to(dtype).cuda(), cache, lens)


def test_queries_of_any_size():
    # bf16 queries far outside fp16's range, with keys' scales that bring the logits back.
    gen = torch.Generator().manual_seed(9)
    cache, _ = make_cache([300] * 4, 2, 16, torch.bfloat16, gen, spread=0.1)
    q = torch.randn((4, 8, D), generator=gen)
    for s, e in enumerate((60, -60, 16, -14)):
        q[s] *= 2.0 ** e
        for p in cache.page_table[s].tolist():
            cache.k_scales[p] *= 2.0 ** -e
    q[3, 2:] = 0.0
    check_decode(selector(8, 2), q.to(torch.bfloat16).cuda(), cache, [300] * 4)


@pytest.mark.parametrize("n", [40, 2100])
def test_unbounded_values_in_sight(n):
    # A NaN number or scale in sight makes its outputs NaN; an infinite scale makes them infinite by their numbers' signs.
    gen = torch.Generator().manual_seed(n)
    cache, _ = make_cache([n], 2, 16, torch.bfloat16, gen)
    q = torch.randn((1, 8, D), generator=gen).to(torch.bfloat16).cuda()
    place = lambda j: (int(cache.page_table[0, j // 16]), j % 16)
    (a, i), (b, j) = place(n - 1), place(3)
    cache.v_pages.view(torch.uint8)[a, 0, i, 77] = 0x7f
    cache.v_scales[b, 1, j] = float("inf")
    signs = f64(cache.v_pages[b, 1, j])
    out = f64(selector(8, 2).paged_decode(q, cache))[0]
    kvec.kvec_sync_status(selector(8, 2).handle)
    assert np.all(np.isnan(out[:4, 77])) and np.isfinite(np.delete(out[:4], 77, axis=1)).all()
    want = np.where(signs == 0, np.nan, np.sign(signs) * np.inf)
    assert np.array_equal(out[4:], np.broadcast_to(want, (4, D)), equal_nan=True)


def test_page_offsets_past_32_bits():
    Hkv, page, pages = 8, 256, 17000
    k = torch.zeros((pages, Hkv, page, D), dtype=torch.uint8, device="cuda")
    assert k.numel() > 2 ** 32
    v, w = torch.zeros_like(k), torch.zeros((pages, Hkv, page), device="cuda")
    ks, vs = torch.ones_like(w), torch.ones_like(w)
    gen = torch.Generator().manual_seed(1)
    small, _ = make_cache([512], Hkv, page, torch.bfloat16, gen, weights=True)
    small.weights.zero_()
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    for at, src in zip((pages - 1, 0), small.page_table[0].tolist()):
        k[at], v[at] = small.k_pages.view(torch.uint8)[src], small.v_pages.view(torch.uint8)[src]
        ks[at], vs[at] = small.k_scales[src], small.v_scales[src]
    lens = torch.tensor([400], dtype=torch.int32).cuda()
    cache = kvec.PagedCache(k.view(E4M3), v.view(E4M3), table, lens, w, k_scales=ks, v_scales=vs, dtype=torch.bfloat16)
    small.lens.copy_(lens)
    q = torch.randn((1, 32, D), generator=gen).to(torch.bfloat16).cuda()
    sel = selector(32, 8)
    assert torch.equal(sel.paged_decode(q, cache), sel.paged_decode(q, small))
    cu = torch.tensor([0, 400], dtype=torch.int32).cuda()
    for a, b in zip(sel.paged_read(cache, cu, 400), sel.paged_read(small, cu, 400)):
        assert torch.equal(a, b)
    fresh = torch.tensor([[pages - 2]], dtype=torch.int32, device="cuda")
    _, kept = sel.paged_evict(cache, fresh, 100, sinks=2, recent=10)
    idx = kept[0].long()
    for pool in (k, v, ks, vs, w):
        rows = torch.cat([pool[-1], pool[0]], dim=1)
        for h in range(Hkv):
            assert torch.equal(pool[-2][h, :100], rows[h][idx[h]])
    x = torch.randn((1, 48, D), generator=gen).to(torch.bfloat16).cuda()
    one = kvec.PagedCache(k.view(E4M3), v.view(E4M3), table[:, :1].contiguous(), torch.tensor([256], dtype=torch.int32).cuda(), w,
                          k_scales=ks, v_scales=vs, dtype=torch.bfloat16)
    sel.rotate_append(x[:, :32], x[:, 32:40], x[:, 40:], torch.tensor([0], dtype=torch.int32).cuda(), None, one)
    check_stored(k[-1][:, 255].view(E4M3), ks[-1][:, 255], f64(x[0, 32:40]), "key")


# ---------------------------------------------------------------- paged_evict

@pytest.mark.parametrize("Hkv,page,lens,budget,sinks,recent", [
    (4, 16, [1], 1, 0, 0),
    (2, 16, [40, 16, 0, 17], 16, 0, 0),
    (8, 32, [576], 512, 4, 32),
    (4, 64, [1000, 300, 512, 513], 512, 4, 100),
    (1, 256, [900, 2], 899, 0, 0),
    (1, 64, [17000, 34000], 12000, 0, 500),
])
def test_evict_moves_numbers_scales_and_weights(Hkv, page, lens, budget, sinks, recent):
    gen = torch.Generator().manual_seed(sum(lens) + budget)
    spare = sum(-(-min(n, budget) // page) for n in lens)
    cache, free = make_cache(lens, Hkv, page, torch.bfloat16, gen, spare=spare)
    table = torch.full((len(lens), -(-min(budget, cache.capacity) // page)), -1, dtype=torch.int32)
    for s in range(len(lens)):
        c = -(-min(lens[s], budget) // page)
        table[s, :c] = torch.tensor(free[:c], dtype=torch.int32)
        free = free[c:]
    kb, vb = raw(cache.k_pages).numpy().astype(float), raw(cache.v_pages).numpy().astype(float)
    ks, vs, w = f64(cache.k_scales), f64(cache.v_scales), f64(cache.weights)
    old, w0 = cache.page_table.cpu().numpy(), w.copy()
    ref_lens, ref_kept = serving.evict(kb, vb, w, old, lens, table.numpy(), cache.capacity, budget, sinks, recent)
    serving.evict(ks[..., None], vs[..., None], w0, old, lens, table.numpy(), cache.capacity, budget, sinks, recent)
    new_lens, kept = selector(Hkv * 2, Hkv).paged_evict(cache, table.cuda(), budget, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    assert np.array_equal(new_lens.cpu().numpy(), ref_lens) and np.array_equal(kept.cpu().numpy(), ref_kept)
    assert np.array_equal(raw(cache.k_pages).numpy(), kb) and np.array_equal(raw(cache.v_pages).numpy(), vb)
    assert np.array_equal(f64(cache.k_scales), ks, equal_nan=True) and np.array_equal(f64(cache.v_scales), vs, equal_nan=True)
    assert np.array_equal(f64(cache.weights), w)


# ---------------------------------------------------------------- paged_read

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,page,lens,first,extra", [
    (1, 16, [1], None, 0),
    (8, 32, [512], [511], 0),
    (4, 64, [200, 0, 137, 1], [0, 0, 100, 0], 3),
    (3, 16, [33, 500], None, 17),
    (2, 256, [1000, 255, 300], [3, 255, 290], 0),
])
@pytest.mark.parametrize("eight", [True, False])
def test_read_matches_the_definition(dtype, Hkv, page, lens, first, extra, eight):
    gen = torch.Generator().manual_seed(sum(lens) + page)
    cache, _ = make_cache(lens, Hkv, page, dtype, gen)
    if eight:
        kp, vp = values(cache.k_pages, cache.k_scales), values(cache.v_pages, cache.v_scales)
    else:
        k = torch.randn(cache.k_pages.shape, generator=gen).to(dtype).cuda()
        v = torch.randn(cache.k_pages.shape, generator=gen).to(dtype).cuda()
        cache = kvec.PagedCache(k, v, cache.page_table, cache.lens)
        kp, vp = f64(k), f64(v)
    cache.page_table[-1, 0] = -1 if len(lens) > 1 else cache.page_table[-1, 0]
    at = first or [0] * len(lens)
    over = 2 if len(lens) > 1 else 0      # rows past the first sequence's length are zeros
    counts = [n - f for n, f in zip(lens, at)]
    counts[0] += over
    cu = np.concatenate([[0], np.cumsum(counts)])
    rows = int(cu[-1]) + extra
    ref = serving.paged_read(kp, vp, cache.page_table.cpu().numpy(), lens, at, cu, rows, 77.0)
    out = [torch.full((rows, Hkv, D), 77.0, dtype=dtype, device="cuda") for _ in range(2)]
    got = selector(Hkv, Hkv).paged_read(cache, torch.tensor(cu, dtype=torch.int32).cuda(), rows,
                                        first=None if first is None else torch.tensor(first, dtype=torch.int32).cuda(),
                                        k_out=out[0], v_out=out[1])
    torch.cuda.synchronize()
    for x, r in zip(got, ref):
        if eight:
            assert np.all(np.abs(f64(x) - r) <= (half_step(dtype) + 2.0 ** -23) * np.abs(r) + (2.0 ** -25 if dtype == torch.float16 else 0))
        else:
            assert np.array_equal(f64(x), r)


def test_read_of_no_rows_and_of_slots_before_the_first():
    cache, _ = make_cache([5], 2, 16, torch.bfloat16, torch.Generator().manual_seed(0))
    cu = torch.tensor([0, 0], dtype=torch.int32).cuda()
    k, v = selector(4, 2).paged_read(cache, cu, 0)
    assert k.shape == v.shape == (0, 2, D)
    before = torch.tensor([-3], dtype=torch.int32).cuda()    # slots below 0 are zeros
    five = torch.tensor([0, 5], dtype=torch.int32).cuda()
    k, _ = selector(4, 2).paged_read(cache, five, 5, first=before)
    assert torch.all(k[:3] == 0) and torch.all(torch.isfinite(k)) and torch.any(k[3:] != 0)
    with pytest.raises(kvec.KvecError):   # one place for both
        selector(4, 2).paged_read(cache, five, 5, k_out=k, v_out=k)


# ---------------------------------------------------------------- together, captured, on other streams

def test_a_serving_loop_over_eight_bits():
    """Prompt stored in two chunks, the second one's attention over rows read back, decoding, eviction, decoding again:
    each step against the definition on what the cache holds."""
    gen = torch.Generator().manual_seed(77)
    dtype, Hq, Hkv, page = torch.bfloat16, 28, 4, 32
    first, second, steps, budget = [150, 70], [60, 33], 3, 128
    total = [a + b + steps for a, b in zip(first, second)]
    counts, spare = [-(-n // page) for n in total], [-(-budget // page) + 1] * 2
    pages = sum(counts) + sum(spare)
    perm = torch.randperm(pages, generator=gen).to(torch.int32)
    width = max(counts)
    table = torch.full((2, width), -1, dtype=torch.int32)
    table[0, :counts[0]], table[1, :counts[1]] = perm[:counts[0]], perm[counts[0]:sum(counts)]
    k = torch.zeros((pages, Hkv, page, D), dtype=torch.uint8, device="cuda").view(E4M3)
    v = torch.zeros((pages, Hkv, page, D), dtype=torch.uint8, device="cuda").view(E4M3)
    ks, vs, w = (torch.zeros((pages, Hkv, page), device="cuda") for _ in range(3))
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache = kvec.PagedCache(k, v, table.cuda(), lens, w, k_scales=ks, v_scales=vs, dtype=dtype)
    sel, tab = selector(Hq, Hkv), rot_table(400, D).cuda()

    def step(new, held):
        x = torch.randn((sum(new), Hq + 2 * Hkv, D), generator=gen).to(dtype).cuda()
        pos = torch.tensor([h + i for n, h in zip(new, held) for i in range(n)], dtype=torch.int32).cuda()
        cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32)
        lens.copy_(torch.tensor([a + b for a, b in zip(new, held)], dtype=torch.int32))
        q = sel.rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pos, tab, cache, cu.cuda())
        return q, cu

    step(first, [0, 0])
    q, cu_q = step(second, first)
    held = [a + b for a, b in zip(first, second)]
    cu_k = torch.tensor([0, held[0], sum(held)], dtype=torch.int32)
    keys, vals = sel.paged_read(cache, cu_k.cuda(), sum(held))
    out, _ = sel.prefill_attention(q, keys, vals, cu_q, cu_q.cuda(), cu_k, cu_k.cuda())
    kvec.kvec_sync_status(sel.handle)
    ref, _ = serving.prefill(f64(q), f64(keys), f64(vals), cu_q.tolist(), cu_k.tolist(), 0, 0, D ** -0.5)
    vmax = np.abs(f64(vals)).max()
    # Weights rounded to the type beside the output's own rounding, and the logits' 2e-5.
    assert np.all(np.abs(f64(out) - ref) <= half_step(dtype) * np.abs(ref) + (half_step(dtype) + 4e-5) * vmax)
    for i in range(steps):
        q, _ = step([1, 1], held)
        held = [n + 1 for n in held]
        check_decode(sel, q, cache, held)
    fresh = torch.full((2, spare[0]), -1, dtype=torch.int32)
    free = perm[sum(counts):]
    fresh[0], fresh[1] = free[:spare[0]], free[spare[0]:]
    new_lens, _ = sel.paged_evict(cache, fresh.cuda(), budget, sinks=4, recent=16)
    small = kvec.PagedCache(k, v, fresh.cuda(), new_lens, w, k_scales=ks, v_scales=vs, dtype=dtype)
    now = new_lens.tolist()
    assert now == [min(n, budget) for n in held]
    check_decode(sel, q, small, now)


def test_calls_on_two_streams_and_in_a_graph():
    gen = torch.Generator().manual_seed(21)
    lens = [900, 33, 2000]
    sel = selector(28, 4)
    cu = torch.tensor([0, 900, 933, 2933], dtype=torch.int32).cuda()
    cases, want = [], []
    for _ in range(2):
        cache, _ = make_cache(lens, 4, 64, torch.bfloat16, gen)
        q = torch.randn((3, 28, D), generator=gen).to(torch.bfloat16).cuda()
        cases.append((q, cache, cache.weights.clone()))
    for q, cache, w0 in cases:
        want.append((sel.paged_decode(q, cache), cache.weights.clone(), sel.paged_read(cache, cu, 2933)))
        cache.weights.copy_(w0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        outs = [(sel.paged_decode(q, cache, stream=st), sel.paged_read(cache, cu, 2933, stream=st))
                for (q, cache, _), st in zip(cases, streams)]
        torch.cuda.synchronize()
        for (q, cache, w0), (out, kv), (ref, w, ref_kv) in zip(cases, outs, want):
            assert torch.equal(out, ref) and torch.equal(cache.weights, w)
            assert torch.equal(kv[0], ref_kv[0]) and torch.equal(kv[1], ref_kv[1])
            cache.weights.copy_(w0)
        torch.cuda.synchronize()
    graphs = []
    for q, cache, _ in cases:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out, kv = sel.paged_decode(q, cache), sel.paged_read(cache, cu, 2933)
        graphs.append((gr, out, kv))
    torch.cuda.synchronize()
    for k in range(3):
        for gr, _, _ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for (q, cache, w0), (_, out, kv), (ref, w, ref_kv) in zip(cases, graphs, want):
            assert torch.equal(out, ref) and (k or torch.equal(cache.weights, w)) and torch.equal(kv[0], ref_kv[0])


def test_a_wait_that_runs_out_is_reported():
    gen = torch.Generator().manual_seed(2)
    cache, _ = make_cache([300, 40], 2, 16, torch.bfloat16, gen)
    q, sel = torch.randn((2, 8, D), generator=gen).to(torch.bfloat16).cuda(), selector(8, 2)
    kvec.kvec_set_test_fault(4)
    try:
        sel.paged_decode(q, cache)
        with pytest.raises(kvec.KvecError) as e:
            kvec.kvec_sync_status(sel.handle)
        assert e.value.status == kvec.KVEC_ERR_DEVICE_TIMEOUT
    finally:
        kvec.kvec_set_test_fault(0)
    cache.weights.zero_()   # what a call that gave up leaves, the weights among it, is invalid
    check_decode(sel, q, cache, [300, 40])
