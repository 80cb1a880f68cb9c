"""GPU parity of the operators over the paged cache (kvec_rotate_append, kvec_paged_decode,
kvec_paged_evict) with their definitions in fp64 (oracle/serving.py).

Tolerances.  u is half a step of the 16-bit type relative to the value (bf16 2^-8, fp16 2^-11).
* Rotated rows: fp32 arithmetic on exact inputs, a handful of roundings and the sum of 128 squares
  (below 2e-6 of the row's largest rotated value R), then one rounding: u |ref| + 4e-6 R.
* Decode outputs: a weight counts as its rounding and the rounding of the rest, off by u^2 p
  (fp16 also by 2^-25 of the largest weight, of which a row of n slots has at most n / sum); logits
  are fp32 sums of exact products, 2e-5 as for the contiguous cache; then one rounding:
  u |ref| + (u^2 + n 2^-25 [fp16] + 2e-5) max|v|, n 2^-25 < 5e-4 at the lengths here.
* Accumulated weights: 2e-5 relative to the step's p summed over the group (the logits' errors), and one
  fp32 rounding of the new value, 2^-24.
* Kept slots, lengths and moved rows are equal.
"""
import numpy as np
import pytest
import torch

from oracle import serving
from paper_2606_29563_gb300 import kvec

pytestmark = pytest.mark.gpu
D = 128
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2606_29563_gb300 import build as kbuild
    kbuild.build()


_SELECTORS = {}


def selector(Hq, Hkv, scale=0.0):
    key = (Hq, Hkv, scale)
    if key not in _SELECTORS:
        _SELECTORS[key] = kvec.KvecSelector(kvec.make_params(Hq, Hkv, num_ext_heads=1, max_batch=300, max_seqlen=64,
                                                             max_layers=1, softmax_scale=scale))
    return _SELECTORS[key]


def f64(x):
    return None if x is None else x.detach().cpu().to(torch.float64).numpy()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def make_cache(lens, Hkv, page, dtype, gen, max_pages=None, spare=0, weights=True, poison=True):
    """Shuffled pages for the sequences' slots, -1 past them; NaN in every slot past a sequence's length."""
    counts = [-(-max(n, 0) // page) for n in lens]
    max_pages = max(1, max(counts)) if max_pages is None else max_pages
    pages = sum(counts) + spare + 1
    perm = torch.randperm(pages, generator=gen).tolist()
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = torch.tensor(perm[at:at + c], dtype=torch.int32)
        at += c
    k = torch.randn((pages, Hkv, page, D), generator=gen).to(dtype)
    v = torch.randn((pages, Hkv, page, D), generator=gen).to(dtype)
    w = torch.randn((pages, Hkv, page), generator=gen).exp() if weights else None
    if poison:
        used = torch.zeros((pages, page), dtype=torch.bool)
        for s, n in enumerate(lens):
            for j in range(max(n, 0)):
                used[table[s, j // page], j % page] = True
        hole = ~used[:, None, :].expand(pages, Hkv, page)
        k[hole] = float("nan")
        v[hole] = float("inf")
    free = perm[at:]
    cache = kvec.PagedCache(k.cuda(), v.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                            None if w is None else w.cuda())
    return cache, free


# ---------------------------------------------------------------- rotate_append

def rot_table(positions, rot, theta=10000.0):
    inv = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def check_rows(got, ref, dtype, name):
    got, u = f64(got), half_step(dtype)
    tol = u * np.abs(ref) + 4e-6 * np.abs(ref).max(axis=-1, keepdims=True) + 1e-30
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{name}: {bad.sum()} values off, by up to {np.abs(got - ref).max():.3e}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,new,held,page,rot,interleaved,norm", [
    (4, 4, [1], [0], 16, 128, False, True),              # the first token of a sequence
    (32, 8, [1, 1, 1], [15, 16, 700], 16, 128, False, True),
    (28, 4, [3, 0, 17, 1], [0, 5, 31, 64], 32, 64, True, False),   # a sequence without new tokens
    (8, 1, [40, 300], [100, 0], 64, 16, True, True),
    (16, 8, [130], [1000], 128, 96, False, True),
    (7, 7, [5, 6], [2, 3], 256, 0, False, True),         # no rotation
    (32, 8, [200, 33], [0, 0], 16, 48, True, False),
])
def test_rotate_append(dtype, Hq, Hkv, new, held, page, rot, interleaved, norm):
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
    kp, vp, w = f64(cache.k_pages), f64(cache.v_pages), f64(cache.weights)
    serving.append(kp, vp, w, cache.page_table.cpu().numpy(), lens, cu, positions.tolist(), max(lens), ref_k, f64(v))
    k_out = torch.empty((T, Hkv, D), dtype=dtype, device="cuda")
    one_each = new == [1] * len(new)
    q_out, k_got = selector(Hq, Hkv).rotate_append(
        q, k, v, positions.cuda(), None if tab is None else tab.cuda(), cache,
        None if one_each else torch.from_numpy(cu).cuda(), q_norm=norms[0], k_norm=norms[1], interleaved=interleaved,
        k_out=k_out)
    torch.cuda.synchronize()
    check_rows(q_out, ref_q, dtype, "q_out")
    check_rows(k_got, ref_k, dtype, "k_out")
    assert np.array_equal(f64(cache.v_pages), vp, equal_nan=True)
    assert np.array_equal(f64(cache.weights), w, equal_nan=True)
    got = f64(cache.k_pages)
    old = np.isnan(kp)
    assert np.array_equal(np.isnan(got), old)
    check_rows(torch.from_numpy(np.where(old, 0, got)), np.where(old, 0, kp), dtype, "k_pages")


@pytest.mark.parametrize("dtype", TYPES)
def test_rotate_without_a_cache_and_in_place(dtype):
    gen = torch.Generator().manual_seed(7)
    q = torch.randn((19, 8, D), generator=gen).to(dtype).cuda()
    k = torch.randn((19, 2, D), generator=gen).to(dtype).cuda()
    pos, tab = torch.randint(0, 5000, (19,), generator=gen, dtype=torch.int32), rot_table(5000, 128)
    rows = f64(tab)[pos.numpy()]
    ref_q, ref_k = (serving.rotate(f64(x), None, 1e-6, rows, False) for x in (q, k))
    sel = selector(8, 2)
    q1, k1 = sel.rotate_append(q, k, None, pos.cuda(), tab.cuda(), cu_tokens=torch.tensor([0, 19], dtype=torch.int32).cuda())
    check_rows(q1, ref_q, dtype, "q")
    check_rows(k1, ref_k, dtype, "k")
    sel.rotate_append(q, k, None, pos.cuda(), tab.cuda(), cu_tokens=torch.tensor([0, 19], dtype=torch.int32).cuda(), q_out=q, k_out=k)
    assert torch.equal(q, q1) and torch.equal(k, k1)


def test_padding_rows_and_missing_pages_are_left_alone():
    dtype, Hq, Hkv, page = torch.bfloat16, 8, 2, 16
    gen = torch.Generator().manual_seed(11)
    lens = [20, 3, 9]
    cache, _ = make_cache(lens, Hkv, page, dtype, gen, max_pages=2)
    table = cache.page_table.clone()
    table[0, 1] = 10 ** 6      # no such page: slots 16 .. 19 of sequence 0 go nowhere
    table[2, 0] = -7
    lens_d = torch.tensor([20, 3, 40], dtype=torch.int32, device="cuda")   # sequence 2 is past its capacity of 32
    cache = kvec.PagedCache(cache.k_pages, cache.v_pages, table, lens_d, cache.weights)
    T, cu = 16, [0, 6, 8, 12]  # four rows behind the last sequence
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=gen).to(dtype).cuda()
    positions = torch.tensor([14, 15, 16, 17, 18, 19, -1, 2, 36, 37, 38, 39, 0, 0, 0, 0], dtype=torch.int32)
    tab = rot_table(38, 128)   # positions 38 and 39 lie outside
    kp, vp, w = f64(cache.k_pages), f64(cache.v_pages), f64(cache.weights)
    rows = f64(tab)[np.clip(positions.numpy(), 0, 37)]
    ref_q = serving.rotate(f64(x[:, :Hq]), None, 1e-6, rows, False)
    ref_k = serving.rotate(f64(x[:, Hq:Hq + Hkv]), None, 1e-6, rows, False)
    serving.append(kp, vp, w, table.cpu().numpy(), [20, 3, 40], cu, positions.tolist(), 38, ref_k, f64(x[:, Hq + Hkv:]))
    q_out = torch.full((T, Hq, D), 77.0, dtype=dtype, device="cuda")
    selector(Hq, Hkv).rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], positions.cuda(), tab.cuda(), cache,
                                    torch.tensor(cu, dtype=torch.int32).cuda(), q_out=q_out)
    torch.cuda.synchronize()
    written = [t for t in range(12) if 0 <= positions[t] < 38]
    left = [t for t in range(T) if t not in written]
    check_rows(q_out[written], ref_q[written], dtype, "q")
    assert torch.all(q_out[left] == 77.0)
    got, old = f64(cache.k_pages), np.isnan(kp)
    assert np.array_equal(np.isnan(got), old) and np.array_equal(f64(cache.v_pages), vp, equal_nan=True)
    check_rows(torch.from_numpy(np.where(old, 0, got)), np.where(old, 0, kp), dtype, "k_pages")
    assert np.array_equal(f64(cache.weights), w)


# ---------------------------------------------------------------- paged_decode

def check_decode(sel, q, cache, lens, max_len=None, window=0, sinks=0, scale=None, table=None):
    dtype, u = q.dtype, half_step(q.dtype)
    max_len = cache.capacity if max_len is None else max_len
    kp, vp, w0 = f64(cache.k_pages), f64(cache.v_pages), f64(cache.weights)
    w = None if w0 is None else w0.copy()
    ref = serving.paged_decode(f64(q), kp, vp, w, cache.page_table.cpu().numpy(), lens, max_len, window, sinks,
                               1 / np.sqrt(D) if scale is None else scale)
    out = sel.paged_decode(q, cache, max_len, window=window, sinks=sinks)
    kvec.kvec_sync_status(sel.handle)
    got = f64(out)
    vmax = 8.0   # of the normal values here (a draw above it has odds of 1e-15)
    assert np.abs(vp[np.isfinite(vp)]).max(initial=0.0) < vmax
    n = max(1, min(max_len, max(lens)))
    tol = u * np.abs(ref) + (u * u + (n * 2.0 ** -25 if dtype == torch.float16 else 0.0) + 2e-5) * vmax
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} outputs off, by up to {np.nanmax(np.abs(got - ref)):.3e}; rows {np.argwhere(bad.any(-1))[:8].tolist()}"
    if w is not None:
        gw = f64(cache.weights)
        bad = ~(np.abs(gw - w) <= 2e-5 * (w - w0) + 2.0 ** -24 * np.abs(w) + 1e-9)
        assert not bad.any(), f"{bad.sum()} weights off, by up to {np.nanmax(np.abs(gw - w)):.3e}: {np.argwhere(bad)[:6].tolist()}"
        assert np.array_equal(gw == w0, w == w0) or np.all((gw == w0) | (w != w0))
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,page,lens,weights", [
    (4, 4, 16, [1], True),
    (8, 4, 16, [15, 16, 17], True),
    (32, 8, 32, [512], True),
    (28, 4, 64, [200, 0, 137, 1], True),       # seven query heads; an empty cache gives zeros
    (16, 2, 128, [513, 300], False),
    (8, 1, 256, [1000, 255, 256, 257], True),
    (32, 8, 16, [4097], True),                 # shared by many CTAs
    (28, 4, 64, [3000, 5, 0, 1777, 64], True),
])
def test_decode_matches_the_definition(dtype, Hq, Hkv, page, lens, weights):
    gen = torch.Generator().manual_seed(sum(lens) + Hq)
    cache, _ = make_cache(lens, Hkv, page, dtype, gen, weights=weights)
    q = (torch.randn((len(lens), Hq, D), generator=gen) * 2).to(dtype).cuda()
    out = check_decode(selector(Hq, Hkv), q, cache, lens)
    for s, n in enumerate(lens):
        if n == 0:
            assert torch.all(out[s] == 0)
    check_decode(selector(Hq, Hkv), q, cache, lens)   # again, on the grown weights


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 3), (16, 4), (17, 16), (64, 20), (100, 0), (5000, 7), (333, 400)])
@pytest.mark.parametrize("lens", [[700, 1, 16, 399, 0], [2500]])
def test_window_and_sinks(lens, window, sinks):
    # Slots outside the window hold infinities and NaN: pages that the window has left behind.
    gen = torch.Generator().manual_seed(window * 31 + sinks)
    dtype, page = torch.bfloat16, 32
    cache, _ = make_cache(lens, 4, page, dtype, gen)
    for s, n in enumerate(lens):
        for j in range(min(sinks, n), max(0, n - window)):
            at = int(cache.page_table[s, j // page])
            cache.k_pages[at, :, j % page] = float("nan")
            cache.v_pages[at, :, j % page] = float("-inf") if j % 2 else float("nan")
    q = torch.randn((len(lens), 12, D), generator=gen).to(dtype).cuda()
    check_decode(selector(12, 4), q, cache, lens, window=window, sinks=sinks)


@pytest.mark.parametrize("batch", [3, 40, 75, 160, 290])
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (32, 8)])
def test_batches_on_both_sides_of_the_cluster_rule(batch, Hq, Hkv):
    gen = torch.Generator().manual_seed(batch + Hq)
    lens = [(0, 1, 15, 16, 17, 63, 64, 65, 128, 130, 255, 257, 31, 7, 300, 48)[(5 * b + b // 16) % 16] for b in range(batch)]
    cache, _ = make_cache(lens, Hkv, 16, torch.bfloat16, gen)
    q = torch.randn((batch, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    check_decode(selector(Hq, Hkv), q, cache, lens)


def test_max_len_and_bad_lengths_and_pages():
    gen = torch.Generator().manual_seed(3)
    dtype, page = torch.float16, 16
    lens = [70, 70, 70]
    cache, _ = make_cache(lens, 2, page, dtype, gen)
    table = cache.page_table.clone()
    table[1, 2] = -1            # slots 32 .. 47 of sequence 1 are on no page
    table[2, 0] = 2 ** 30
    for lens, max_len in (([70, 70, 70], 80), ([-5, 10 ** 9, 33], 80), ([70, 70, 70], 33), ([70, 48, 16], 48)):
        c = kvec.PagedCache(cache.k_pages, cache.v_pages, table, torch.tensor(lens, dtype=torch.int32).cuda(), cache.weights)
        # Lengths past the pages meet NaN in the slots behind the real ones: cut the reference the same way.
        if lens[1] == 10 ** 9:
            c.k_pages[torch.isnan(c.k_pages)] = 0.25
            c.v_pages[torch.isinf(c.v_pages)] = 0.5
        q = torch.randn((3, 8, D), generator=gen).to(dtype).cuda()
        check_decode(selector(8, 2), q, c, lens, max_len=max_len)


def test_minus_infinite_logits_have_no_weight():
    gen = torch.Generator().manual_seed(5)
    lens = [40, 600, 17]
    cache, _ = make_cache(lens, 2, 16, torch.bfloat16, gen)
    q = torch.ones((3, 8, D), dtype=torch.bfloat16, device="cuda")
    for s, hit in ((0, range(0, 20)), (1, range(0, 600, 2)), (2, range(17))):   # sequence 2: every one
        for j in hit:
            cache.k_pages[int(cache.page_table[s, j // 16]), :, j % 16, 0] = float("-inf")
    out = check_decode(selector(8, 2), q, cache, lens)
    assert torch.all(out[2] == 0)


def test_a_softmax_scale_of_the_handle():
    gen = torch.Generator().manual_seed(9)
    cache, _ = make_cache([100], 2, 16, torch.bfloat16, gen)
    q = torch.randn((1, 4, D), generator=gen).to(torch.bfloat16).cuda()
    check_decode(selector(4, 2, 0.25), q, cache, [100], scale=0.25)


def test_page_offsets_past_32_bits():
    # Rows whose byte offset in the pool is past 2^32: the last page of 20 million rows.
    Hkv, page, pages = 8, 256, 9000
    k = torch.zeros((pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    assert k.numel() * 2 > 2 ** 32
    v, w = torch.zeros_like(k), torch.zeros((pages, Hkv, page), device="cuda")
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(1)
    for at in (pages - 1, 0):
        k[at] = torch.randn((Hkv, page, D), generator=gen).to(k.dtype).cuda()
        v[at] = torch.randn((Hkv, page, D), generator=gen).to(k.dtype).cuda()
    cache = kvec.PagedCache(k, v, table, torch.tensor([400], dtype=torch.int32).cuda(), w)
    q = torch.randn((1, 32, D), generator=gen).to(k.dtype).cuda()
    small = kvec.PagedCache(torch.stack([k[0], k[-1]]), torch.stack([v[0], v[-1]]), torch.tensor([[1, 0]], dtype=torch.int32).cuda(),
                            cache.lens, torch.zeros((2, Hkv, page), device="cuda"))
    out = check_decode(selector(32, 8), q, small, [400])
    assert torch.equal(selector(32, 8).paged_decode(q, cache), out)
    assert torch.equal(w[-1], small.weights[1]) and torch.equal(w[0], small.weights[0])
    fresh = torch.tensor([[pages - 2]], dtype=torch.int32, device="cuda")
    new_lens, kept = selector(32, 8).paged_evict(cache, fresh, 100, sinks=2, recent=10)
    idx = kept[0].long()
    rows_k = torch.cat([k[-1], k[0]], dim=1)
    for h in range(Hkv):
        assert torch.equal(k[-2][h, :100], rows_k[h][idx[h]])
    x = torch.randn((1, 48, D), generator=gen).to(k.dtype).cuda()
    selector(32, 8).rotate_append(x[:, :32], x[:, 32:40], x[:, 40:], torch.tensor([0], dtype=torch.int32).cuda(), None,
                                  kvec.PagedCache(k, v, table[:, :1].contiguous(), torch.tensor([256], dtype=torch.int32).cuda(), w))
    assert torch.equal(k[-1][:, 255], x[0, 32:40]) and torch.equal(v[-1][:, 255], x[0, 40:])


# ---------------------------------------------------------------- paged_evict

def check_evict(sel, cache, free, lens, budget, sinks, recent, page, max_len=None):
    max_len = cache.capacity if max_len is None else max_len
    need = -(-min(budget, max_len) // page)
    table = torch.full((len(lens), need), -1, dtype=torch.int32)
    for s in range(len(lens)):
        c = -(-min(max(lens[s], 0), max_len, budget) // page)
        table[s, :c] = torch.tensor(free[:c], dtype=torch.int32)
        free = free[c:]
    kp, vp, w = f64(cache.k_pages), f64(cache.v_pages), f64(cache.weights)
    ref_lens, ref_kept = serving.evict(kp, vp, w, cache.page_table.cpu().numpy(), lens, table.numpy(), max_len, budget, sinks, recent)
    new_lens, kept = sel.paged_evict(cache, table.cuda(), budget, sinks=sinks, recent=recent, max_len=max_len)
    torch.cuda.synchronize()
    assert np.array_equal(new_lens.cpu().numpy(), ref_lens)
    assert np.array_equal(kept.cpu().numpy(), ref_kept)
    assert np.array_equal(f64(cache.k_pages), kp, equal_nan=True)
    assert np.array_equal(f64(cache.v_pages), vp, equal_nan=True)
    assert np.array_equal(f64(cache.weights), w, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,page,lens,budget,sinks,recent", [
    (4, 16, [1], 1, 0, 0),
    (2, 16, [40, 16, 0, 17], 16, 0, 0),
    (8, 32, [576], 512, 4, 32),
    (4, 64, [1000, 300, 512, 513], 512, 4, 100),
    (2, 128, [700], 7, 3, 4),                  # nothing left to rank
    (1, 256, [900, 2], 899, 0, 0),
    (3, 16, [3000], 1000, 1, 1),
    (2, 64, [9000], 4000, 4, 64),
    (1, 64, [17000, 30000], 12000, 0, 500),
])
def test_evict_matches_the_definition(dtype, Hkv, page, lens, budget, sinks, recent):
    gen = torch.Generator().manual_seed(sum(lens) + budget)
    spare = sum(-(-min(n, budget) // page) for n in lens)
    cache, free = make_cache(lens, Hkv, page, dtype, gen, spare=spare)
    check_evict(selector(Hkv * 2, Hkv), cache, free, lens, budget, sinks, recent, page)


def test_evict_a_row_longer_than_the_registers_hold():
    gen = torch.Generator().manual_seed(2)
    lens, page = [33000, 40001, 20], 256
    cache, free = make_cache(lens, 1, page, torch.bfloat16, gen, spare=400, poison=False)
    cache.weights.copy_((cache.weights * 50).round() / 50)     # many equal ones
    check_evict(selector(2, 1), cache, free, lens, 30000, 4, 100, page)


@pytest.mark.parametrize("n", [100, 5000, 33001])
def test_ties_and_special_weights(n):
    # Equal weights, zeros of both signs, infinities, NaN, and every value the same.
    gen = torch.Generator().manual_seed(n)
    cache, free = make_cache([n, n], 2, 64, torch.float16, gen, spare=2 * (n // 128 + 2), poison=False)
    vals = torch.tensor([0.0, -0.0, 1.0, 1.0, 2.0, float("inf"), float("nan"), -1.0, float("-inf"), 1e-42])
    cache.weights.copy_(vals[torch.randint(0, 10, cache.weights.shape, generator=gen)])
    one = int(cache.page_table[1, 0])
    for p in cache.page_table[1].tolist():
        cache.weights[p, 1] = 3.5
    assert one >= 0
    for budget, sinks, recent in ((n // 2, 0, 0), (n // 3, 2, 9), (1, 0, 0)):
        check_evict(selector(4, 2), cache, free, [n, n], budget, sinks, recent, 64)


def test_evict_with_slots_on_no_page():
    gen = torch.Generator().manual_seed(4)
    cache, free = make_cache([100, 100], 2, 16, torch.bfloat16, gen, spare=20, poison=False)
    cache.page_table[0, 2] = -1
    cache.page_table[1, 0] = 10 ** 8
    check_evict(selector(4, 2), cache, free, [100, 100], 90, 4, 10, 16)
    check_evict(selector(4, 2), cache, free, [100, 100], 40, 0, 10, 16, max_len=64)


# ---------------------------------------------------------------- captured, on other streams, twice at once

def test_calls_on_two_streams_and_in_a_graph():
    gen = torch.Generator().manual_seed(21)
    lens = [900, 33, 2000]
    sel = selector(28, 4)
    cases = []
    for _ in range(2):
        cache, _ = make_cache(lens, 4, 64, torch.bfloat16, gen)
        q = torch.randn((3, 28, D), generator=gen).to(torch.bfloat16).cuda()
        cases.append((q, cache, cache.weights.clone()))
    want = []
    for q, cache, w0 in cases:
        want.append((sel.paged_decode(q, cache), cache.weights.clone()))
        cache.weights.copy_(w0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        outs = [sel.paged_decode(q, cache, stream=st) for (q, cache, _), st in zip(cases, streams)]
        torch.cuda.synchronize()
        for (q, cache, w0), out, (ref, w) in zip(cases, outs, want):
            assert torch.equal(out, ref) and torch.equal(cache.weights, w)
            cache.weights.copy_(w0)
        torch.cuda.synchronize()
    graphs = []
    for q, cache, _ in cases:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = sel.paged_decode(q, cache)
        graphs.append((gr, out))
    torch.cuda.synchronize()
    for k in range(3):
        for gr, _ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for (q, cache, w0), (_, out), (ref, w) in zip(cases, graphs, want):
            assert torch.equal(out, ref) and (k or torch.equal(cache.weights, w))


@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 999), (8, 2, 1001), (32, 8, 3126), (32, 8, 3127), (16, 8, 18755), (40, 8, 12000)])
def test_rotate_append_on_both_sides_of_the_layout_rule(Hq, Hkv, T):
    # Every layout gives the same rows, bit for bit, as one token at a time: 12000, 150000 and 600000 rows.
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
        k, v = (torch.zeros((sum(counts), Hkv, page, D), dtype=dtype, device="cuda") for _ in range(2))
        weights = torch.ones((sum(counts), Hkv, page), device="cuda")
        q = torch.empty((T, Hq, D), dtype=dtype, device="cuda")
        for t0 in range(0, T, step):
            t1 = min(t0 + step, T)
            cu = torch.tensor([0, new[0], T]).clamp(t0, t1) - t0
            held = torch.tensor([min(t1, new[0]), max(t1 - new[0], 0)], dtype=torch.int32).cuda()
            sel.rotate_append(x[t0:t1, :Hq], x[t0:t1, Hq:Hq + Hkv], x[t0:t1, Hq + Hkv:], pos[t0:t1], tab,
                              kvec.PagedCache(k, v, table.cuda(), held, weights), cu.int().cuda(), q_norm=w[0], k_norm=w[1],
                              q_out=q[t0:t1])
        got.append((q, k, v, weights))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    rows = f64(tab)[pos[:50].cpu().numpy()]
    check_rows(got[0][0][:50], serving.rotate(f64(x[:50, :Hq]), f64(w[0]), 1e-6, rows, False), dtype, "q")


def test_windows_and_first_slots_of_any_size():
    gen = torch.Generator().manual_seed(6)
    cache, _ = make_cache([77, 3000], 2, 16, torch.bfloat16, gen, weights=False)
    q = torch.randn((2, 4, D), generator=gen).to(torch.bfloat16).cuda()
    sel, most = selector(4, 2), 2 ** 31 - 1
    whole = sel.paged_decode(q, cache)
    for window, sinks in ((most, 0), (most, most), (1, most), (2 ** 20, 5)):
        assert torch.equal(sel.paged_decode(q, cache, window=window, sinks=sinks), whole)


def test_rotation_without_sequences_takes_any_number_of_tokens():
    gen = torch.Generator().manual_seed(8)
    q, k = (torch.randn((1000, h, D), generator=gen).to(torch.float16).cuda() for h in (4, 2))
    pos, tab = torch.arange(1000, dtype=torch.int32).cuda(), rot_table(1000, 128).cuda()
    got = selector(4, 2).rotate_append(q, k, None, pos, tab)
    cu = torch.tensor([0, 1000], dtype=torch.int32).cuda()
    want = selector(4, 2).rotate_append(q, k, None, pos, tab, cu_tokens=cu)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("batch,scale,Hq,Hkv", [(290, 2, 8, 4), (70, 9, 28, 4), (300, 3, 32, 8)])
def test_many_sequences_on_the_list_path(batch, scale, Hq, Hkv):
    # Rows past 512 slots share the list of all blocks; empty ones lie between them and at its ends.
    gen = torch.Generator().manual_seed(batch * scale)
    lens = [scale * (0, 1, 15, 16, 17, 63, 64, 65, 128, 130, 255, 257, 31, 7, 300, 48)[(5 * b + b // 16) % 16] for b in range(batch)]
    cache, _ = make_cache(lens, Hkv, 32, torch.bfloat16, gen)
    assert cache.capacity > 512
    q = torch.randn((batch, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    check_decode(selector(Hq, Hkv), q, cache, lens)


@pytest.mark.parametrize("lens", [[5, 0, 17], [0, 0, 0], [1], [0, 300], [40, 33, 2, 0, 0, 1, 99]])
@pytest.mark.parametrize("weights", [False, True])
def test_a_bound_far_above_the_lengths(lens, weights):
    # The work is divided by max_len: most CTAs have no block, and pairs are shared with empty shares between.
    gen = torch.Generator().manual_seed(len(lens) + sum(lens))
    cache, _ = make_cache(lens, 2, 64, torch.float16, gen, max_pages=16384 // 64, weights=weights)
    q = torch.randn((len(lens), 14, D), generator=gen).to(torch.float16).cuda()
    out = check_decode(selector(14, 2), q, cache, lens)
    for s, n in enumerate(lens):
        assert n or torch.all(out[s] == 0)


def lengths_of(kind, batch):
    if kind == "alike":                                   # a CTA each
        return [600 + (37 * b) % 100 for b in range(batch - 2)] + [0, 555]
    if kind == "one long":                                # the list of all blocks
        return [5000] + [30 + b for b in range(batch - 1)]
    return [(b * 389) % 1500 if b % 3 else b % 20 for b in range(batch)]


@pytest.mark.parametrize("kind", ["alike", "one long", "mixed"])
@pytest.mark.parametrize("Hq,Hkv,batch,window,sinks", [(8, 4, 60, 0, 0), (28, 4, 70, 0, 0), (16, 8, 30, 530, 20)])
def test_pairs_about_as_many_as_ctas(kind, Hq, Hkv, batch, window, sinks):
    gen = torch.Generator().manual_seed(batch + window)
    lens = lengths_of(kind, batch)
    cache, _ = make_cache(lens, Hkv, 64, torch.bfloat16, gen)
    q = torch.randn((batch, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    check_decode(selector(Hq, Hkv), q, cache, lens, window=window, sinks=sinks)


def test_a_captured_call_takes_lengths_of_every_kind():
    # The way the work is divided follows the lengths on the device.
    gen = torch.Generator().manual_seed(50)
    batch, Hq, Hkv = 60, 8, 4
    kinds = [lengths_of(k, batch) for k in ("alike", "one long", "mixed")]
    cache, _ = make_cache([max(x) for x in zip(*kinds)], Hkv, 64, torch.bfloat16, gen)
    q = torch.randn((batch, Hq, D), generator=gen).to(torch.bfloat16).cuda()
    sel, first = selector(Hq, Hkv), cache.weights.clone()
    out = torch.empty_like(q)
    sel.paged_decode(q, cache, 5000, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sel.paged_decode(q, cache, 5000, out=out)
    for lens in kinds[1:] + kinds[:2]:
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.weights.copy_(first)
        graph.replay()
        kvec.kvec_sync_status(sel.handle)
        got, weights = out.clone(), cache.weights.clone()
        cache.weights.copy_(first)
        want = check_decode(sel, q, cache, lens, max_len=5000)
        assert torch.equal(got, want) and torch.equal(weights, cache.weights)


def test_rotate_of_rows_that_overlap():
    # Tokens 8 elements apart, as documented: the outputs made for them are packed all the same.
    gen = torch.Generator().manual_seed(60)
    base = torch.randn(2000, generator=gen).to(torch.bfloat16).cuda()
    q, k = torch.as_strided(base, (6, 4, D), (8, D, 1)), torch.as_strided(base, (6, 2, D), (16, D, 1))
    pos, tab = torch.arange(6, dtype=torch.int32).cuda(), rot_table(16, D).cuda()
    got = selector(4, 2).rotate_append(q, k, None, pos, tab)
    want = selector(4, 2).rotate_append(q.contiguous(), k.contiguous(), None, pos, tab)
    assert all(x.is_contiguous() for x in got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,window,sinks", [([40], 0, 0), ([500, 33], 0, 0), ([6000, 77], 0, 0), ([900, 2100], 64, 3)])
def test_unbounded_values_in_sight(dtype, lens, window, sinks):
    # What is infinite or NaN in V and seen gives sum p v as it is defined: an infinity stays one, two of different
    # signs and NaN give NaN.  (q and k of normal values: each weight is above 2^-25 of the largest.)
    gen = torch.Generator().manual_seed(sum(lens) + window)
    cache, _ = make_cache(lens, 2, 16, dtype, gen)
    q = torch.randn((len(lens), 8, D), generator=gen).to(dtype).cuda()
    for s, n in enumerate(lens):
        last, before, first = n - 1, n - 20, 0 if window == 0 or sinks else n - 2
        for slot, col, value in ((last, 3, "inf"), (before, 9, "-inf"), (first, 70, "nan"), (last, 127, "inf"), (before, 127, "-inf")):
            cache.v_pages[int(cache.page_table[s, slot // 16]), 1, slot % 16, col] = float(value)
    w0 = f64(cache.weights)
    w = w0.copy()
    with np.errstate(invalid="ignore"):
        ref = serving.paged_decode(f64(q), f64(cache.k_pages), f64(cache.v_pages), w, cache.page_table.cpu().numpy(), lens,
                                   cache.capacity, window, sinks, 1 / np.sqrt(D))
    sel, u = selector(8, 2), half_step(dtype)
    got = f64(sel.paged_decode(q, cache, window=window, sinks=sinks))
    kvec.kvec_sync_status(sel.handle)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    assert np.isinf(ref).sum() == len(lens) * 4 * 2 and np.isnan(ref).sum() == len(lens) * 4 * 2
    fine = np.isfinite(ref)
    n = max(lens)
    tol = u * np.abs(ref[fine]) + (u * u + (n * 2.0 ** -25 if dtype == torch.float16 else 0.0) + 2e-5) * 8.0
    assert np.all(np.abs(got[fine] - ref[fine]) <= tol)
    assert np.all(np.abs(f64(cache.weights) - w) <= 2e-5 * (w - w0) + 2.0 ** -24 * np.abs(w) + 1e-9)


def test_scratch_goes_by_what_is_in_sight():
    # With a window no more than its slots wait in scratch, and the call stays within the bytes that it asks for.
    gen = torch.Generator().manual_seed(70)
    lens, window, sinks = [900, 40, 3000], 100, 20
    cache, _ = make_cache(lens, 2, 64, torch.bfloat16, gen, max_pages=131072 // 64)
    q = torch.randn((3, 16, D), generator=gen).to(torch.bfloat16).cuda()
    sel, first = selector(16, 2), cache.weights.clone()
    whole = kvec.kvec_paged_decode_bytes(sel.handle, 3, 131072, True)
    need = kvec.kvec_paged_decode_window_bytes(sel.handle, 3, 131072, window, sinks, True)
    fixed = kvec.kvec_paged_decode_window_bytes(sel.handle, 3, 131072, window, sinks, False)
    assert fixed == kvec.kvec_paged_decode_bytes(sel.handle, 3, 131072, False)
    assert whole - fixed == 3 * 16 * 131072 * 4 and need - fixed == 3 * 16 * (100 // 16 + 2 + 2) * 16 * 4
    assert kvec.kvec_paged_decode_window_bytes(sel.handle, 3, 131072, 0, 7, True) == whole
    assert kvec.kvec_paged_decode_window_bytes(sel.handle, 3, 131072, -1, 0, True) == 0
    assert kvec.kvec_paged_decode_window_bytes(sel.handle, 3, 131072, 9, -1, True) == 0
    out = torch.empty_like(q)

    def run(scratch, size):
        cache.weights.copy_(first)
        kvec.kvec_paged_decode(sel.handle, 3, q.data_ptr(), cache.c, 131072, window, sinks, out.data_ptr(), scratch.data_ptr(),
                               size, torch.cuda.current_stream().cuda_stream)
        kvec.kvec_sync_status(sel.handle)
        return out.clone(), cache.weights.clone()

    large = run(torch.empty(whole, dtype=torch.uint8, device="cuda"), whole)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    small = run(room, need)
    assert torch.equal(small[0], large[0]) and torch.equal(small[1], large[1]) and torch.all(room[need:] == 0xA5)
    with pytest.raises(kvec.KvecError):
        run(room, need - 1)
    cache.weights.copy_(first)
    check_decode(sel, q, cache, lens, max_len=131072, window=window, sinks=sinks)


def test_a_windowed_call_takes_little_memory():
    # 64 caches with room for 131072 slots each: the logits of all of them would take 1.07 GB.
    gen = torch.Generator().manual_seed(71)
    cache, _ = make_cache([50] * 64, 8, 64, torch.bfloat16, gen, max_pages=131072 // 64)
    q = torch.randn((64, 32, D), generator=gen).to(torch.bfloat16).cuda()
    sel = selector(32, 8)
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    sel.paged_decode(q, cache, window=512, sinks=4)
    assert torch.cuda.max_memory_allocated() - held < 10 << 20   # 64 * 32 * (512 + 3 * 16) * 4 = 4.6 MB, and 2.6 MB
