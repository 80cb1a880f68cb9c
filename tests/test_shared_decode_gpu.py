"""GPU parity of the attention of single tokens behind shared prefixes (kvec_shared_decode) with its definition in fp64
(oracle/serving.py).

Tolerances.  u is half a step of the 16-bit type relative to the value (bf16 2^-8, fp16 2^-11).  The weights of a prefix's
slots are rounded to the type before they meet the values: at most u max|v| (fp16 also 2^-25 of the row's first maximum
for each of n slots, n 2^-25 max|v|); logits are fp32 sums of exact products and exponentials approximate, 2e-5 in each of
the two parts that are joined; the result is rounded once: u |ref| + (u + 4e-5 + n 2^-25 [fp16]) max|v|.
Accumulated weights of own slots: 4e-5 of the step's sum (both parts' logits), and a rounding of the new value.
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


def selector(Hq, Hkv):
    key = (Hq, Hkv)
    if key not in _SELECTORS:
        _SELECTORS[key] = kvec.KvecSelector(kvec.make_params(Hq, Hkv, num_ext_heads=1, max_batch=300, max_seqlen=64, max_layers=1))
    return _SELECTORS[key]


def f64(x):
    return None if x is None else x.detach().cpu().to(torch.float64).numpy()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def make(prefixes, groups, lens, Hkv, page, dtype, gen, weights=True, pages=None, own_pages=None):
    """Shuffled pages for prefixes and own slots; NaN and infinities in every slot that none of them holds."""
    spans = [-(-n // page) for n in prefixes], [-(-n // page) for n in lens]
    count = sum(spans[0]) + sum(spans[1]) + 1
    perm = torch.randperm(count, generator=gen).tolist()
    tables, at = [], 0
    for counts, least in zip(spans, (pages, own_pages)):
        table = torch.full((len(counts), max(1, max(counts)) if least is None else least), -1, dtype=torch.int32)
        for s, c in enumerate(counts):
            table[s, :c] = torch.tensor(perm[at:at + c], dtype=torch.int32)
            at += c
        tables.append(table)
    k = torch.randn((count, Hkv, page, D), generator=gen).to(dtype)
    v = torch.randn((count, Hkv, page, D), generator=gen).to(dtype)
    hole = torch.ones((count, page), dtype=torch.bool)
    for table, ns in zip(tables, (prefixes, lens)):
        for s, n in enumerate(ns):
            for j in range(n):
                hole[table[s, j // page], j % page] = False
    hole = hole[:, None, :].expand(count, Hkv, page)
    k[hole] = float("nan")
    v[hole] = float("inf")
    w = torch.randn((count, Hkv, page), generator=gen).exp().cuda() if weights else None
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    cache = kvec.PagedCache(k.cuda(), v.cuda(), tables[1].cuda(), ints(lens), w)
    return cache, kvec.SharedPrefix(tables[0].cuda(), ints(prefixes), ints([0] + np.cumsum(groups).tolist()))


def check(sel, q, cache, prefix, max_len=None, max_prefix=None, **kw):
    dtype, u = q.dtype, half_step(q.dtype)
    max_len = cache.capacity if max_len is None else max_len
    max_prefix = prefix.max_pages * cache.page_size if max_prefix is None else max_prefix
    vp, w0 = f64(cache.v_pages), f64(cache.weights)
    w = None if w0 is None else w0.copy()
    lens, plens = cache.lens.tolist(), prefix.lens.tolist()
    ref = serving.shared_decode(f64(q), f64(cache.k_pages), vp, w, cache.page_table.cpu().numpy(), lens, max_len,
                                prefix.page_table.cpu().numpy(), plens, prefix.cu_seqs.tolist(), max_prefix, 1 / np.sqrt(D))
    out = sel.shared_decode(q, cache, prefix, max_len, max_prefix=max_prefix, **kw)
    kvec.kvec_sync_status(sel.handle)
    got = f64(out)
    vmax = np.abs(vp[np.isfinite(vp)]).max(initial=0.0)
    n = max(min(max(plens), max_prefix), 0) + max(min(max(lens), max_len), 1)
    tol = u * np.abs(ref) + (u + 4e-5 + (n * 2.0 ** -25 if dtype == torch.float16 else 0.0)) * vmax
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} outputs off, by up to {np.nanmax(np.abs(got - ref)):.3e}; rows {np.argwhere(bad.any(-1))[:8].tolist()}"
    if w is not None:
        gw = f64(cache.weights)
        bad = ~(np.abs(gw - w) <= 4e-5 * (w - w0) + 2.0 ** -24 * np.abs(w) + 1e-9)
        assert not bad.any(), f"{bad.sum()} weights off, by up to {np.nanmax(np.abs(gw - w)):.3e}: {np.argwhere(bad)[:6].tolist()}"
    return out


def queries(batch, Hq, dtype, gen):
    return (torch.randn((batch, Hq, D), generator=gen) * 2).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,page,prefixes,groups,lens", [
    (4, 4, 16, [1], [1], [1]),
    (8, 4, 16, [15], [2], [3, 0]),                             # a sequence without own slots
    (32, 8, 32, [128], [3], [1, 40, 16]),
    (28, 4, 64, [500], [4], [1, 17, 40, 23]),
    (28, 4, 16, [300], [73], [(7 * i) % 50 for i in range(73)]),    # two pairs of tiles and one query more
    (16, 2, 128, [129, 0, 700], [5, 3, 17], [(11 * i) % 90 for i in range(25)]),   # a group without a prefix
    (8, 1, 256, [1000, 37], [0, 6], [5, 9, 255, 256, 257, 0]),  # a group without sequences
    (7, 7, 64, [127, 640], [129, 2], [(3 * i) % 40 for i in range(131)]),
    (32, 8, 16, [4097], [9], [2, 600, 33, 0, 1, 5, 1100, 64, 16]),
])
def test_matches_the_definition(dtype, Hq, Hkv, page, prefixes, groups, lens):
    gen = torch.Generator().manual_seed(sum(lens) + sum(prefixes) + Hq)
    cache, prefix = make(prefixes, groups, lens, Hkv, page, dtype, gen)
    q = queries(len(lens), Hq, dtype, gen)
    check(selector(Hq, Hkv), q, cache, prefix)
    check(selector(Hq, Hkv), q, cache, prefix)   # again, on the grown weights


@pytest.mark.parametrize("kind", ["clusters", "a CTA a pair", "shares", "one long", "none of their own"])
@pytest.mark.parametrize("weights", [True, False])
def test_every_path_of_the_own_slots(kind, weights):
    gen = torch.Generator().manual_seed(len(kind))
    Hq, Hkv, page, batch = 8, 4, 32, 60
    lens = {"clusters": [(9 * b) % 130 for b in range(batch)], "a CTA a pair": [600 + (37 * b) % 100 for b in range(batch - 1)] + [0],
            "shares": [(b * 389) % 1500 if b % 3 else b % 20 for b in range(batch)],
            "one long": [5000] + [0, 30] * 29 + [7], "none of their own": [0] * batch}[kind]
    cache, prefix = make([333, 64], [41, 14], lens, Hkv, page, torch.bfloat16, gen, weights=weights)   # five without a prefix
    check(selector(Hq, Hkv), queries(batch, Hq, torch.bfloat16, gen), cache, prefix)


@pytest.mark.parametrize("groups,length", [(70, 20), (33, 300), (150, 130)])
def test_many_groups(groups, length):
    gen = torch.Generator().manual_seed(groups)
    sizes = [(5 * r) % 4 for r in range(groups)]
    prefixes = [(length * r) // 3 % (2 * length) for r in range(groups)]
    lens = [1 + (3 * b) % 30 for b in range(sum(sizes))]
    cache, prefix = make(prefixes, sizes, lens, 2, 16, torch.float16, gen)
    check(selector(8, 2), queries(len(lens), 8, torch.float16, gen), cache, prefix)

def many_groups(n, gen, Hkv=1, size=lambda r: 1):
    """n groups behind prefixes that fill their pages, of pages that many of them share (they are only read)."""
    dtype, pages = torch.bfloat16, 200
    sel = kvec.KvecSelector(kvec.make_params(4 * Hkv, Hkv, num_ext_heads=1, max_batch=n, max_seqlen=64, max_layers=1))
    k, v = (torch.randn((pages, Hkv, 16, D), generator=gen).to(dtype).cuda() for _ in range(2))
    sizes = [size(r) for r in range(n)]
    batch = sum(sizes)
    prefixes = torch.tensor([16 * (r % 4) for r in range(n)], dtype=torch.int32)
    lens = torch.tensor([(7 * b) % 40 for b in range(batch)], dtype=torch.int32).cuda()
    prefix = kvec.SharedPrefix(torch.randint(pages, (n, 3), generator=gen, dtype=torch.int32).cuda(), prefixes.cuda(),
                               torch.tensor([0] + np.cumsum(sizes).tolist(), dtype=torch.int32).cuda())
    cache = kvec.PagedCache(k, v, torch.randint(pages, (batch, 3), generator=gen, dtype=torch.int32).cuda(), lens)
    return sel, queries(batch, 4 * Hkv, dtype, gen), cache, prefix, sizes


@pytest.mark.parametrize("n,size", [(700, lambda r: r % 3), (5000, lambda r: 1), (3000, lambda r: (r % 700 == 5) * 300 + (r < 50))])
def test_thousands_of_groups(n, size):
    # Against every sequence on its own over its prefix's pages and then its own: the same within the roundings.
    gen = torch.Generator().manual_seed(n)
    sel, q, cache, prefix, sizes = many_groups(n, gen, 2, size)
    of = torch.repeat_interleave(torch.arange(n), torch.tensor(sizes)).cuda()
    held = prefix.lens[of]
    at, own = torch.arange(6, device="cuda")[None, :], held[:, None] // 16
    table = torch.where(at < own, prefix.page_table[of].gather(1, at.clamp(max=2).expand(len(of), -1)),
                        cache.page_table.gather(1, (at - own).clamp(0, 2))).to(torch.int32).contiguous()
    whole = kvec.PagedCache(cache.k_pages, cache.v_pages, table, cache.lens + held)
    a, b = f64(sel.shared_decode(q, cache, prefix)), f64(sel.paged_decode(q, whole))
    kvec.kvec_sync_status(sel.handle)
    u = half_step(q.dtype)
    vmax = float(cache.v_pages.float().abs().max())
    assert np.all(np.abs(a - b) <= 2 * u * np.abs(b) + (u + 6e-5) * vmax)
    sel.close()


def test_time_grows_with_the_groups():
    # Eight times as many take eight times as long (17 where each sequence's place was summed up by every lane alone).
    times = []
    for n in (1024, 8192):
        sel, q, cache, prefix, _ = many_groups(n, torch.Generator().manual_seed(n))
        times.append(device_time(lambda: sel.shared_decode(q, cache, prefix)))
        kvec.kvec_sync_status(sel.handle)
        sel.close()
    assert times[1] < 13 * times[0], times



@pytest.mark.parametrize("Hkv,prefixes,groups", [
    (8, [1280] * 13, [1, 2] * 6 + [3]),          # 104 items of ten blocks: shares of a list
    (8, [1280] * 9 + [100], [1] * 10),           # 80 items: a chunk a CTA would be a fourth longer than the mean
    (4, [4000, 128, 129], [70, 1, 40]),          # chunks of several pairs
    (1, [20000], [130]),                         # more CTAs than an item of each length needs
    (2, [16], [300 // 4]),                       # one block each
])
def test_divisions_of_the_prefixes(Hkv, prefixes, groups):
    gen = torch.Generator().manual_seed(sum(prefixes) + Hkv)
    lens = [(3 * b) % 20 for b in range(sum(groups) + 1)]
    cache, prefix = make(prefixes, groups, lens, Hkv, 64, torch.bfloat16, gen)
    check(selector(4 * Hkv, Hkv), queries(len(lens), 4 * Hkv, torch.bfloat16, gen), cache, prefix)


def test_missing_pages_and_bounds():
    gen = torch.Generator().manual_seed(4)
    cache, prefix = make([200, 1000], [3, 4], [20, 0, 33, 50, 1, 2, 3], 2, 16, torch.bfloat16, gen, own_pages=8)
    q = queries(7, 8, torch.bfloat16, gen)
    prefix.page_table[0, 3] = -1                       # in the middle of a block
    prefix.page_table[1, 40:] = 10 ** 9                # whole blocks, and the last slots
    prefix.page_table[1, 7] = -5
    cache.page_table[3, 1] = -1
    check(selector(8, 2), q, cache, prefix)
    check(selector(8, 2), q, cache, prefix, max_len=30, max_prefix=777)
    prefix.page_table[0] = -1                          # a prefix on no page at all
    check(selector(8, 2), q, cache, prefix)
    # Lengths outside their bounds count as these.
    prefix.lens.copy_(torch.tensor([-7, 100], dtype=torch.int32))
    cache.lens.copy_(torch.tensor([-1, 0, 33, 50, 1, 2, 3], dtype=torch.int32))
    check(selector(8, 2), q, cache, prefix)


def test_large_pages_end_inside_blocks():
    for page in (128, 256):
        gen = torch.Generator().manual_seed(page)
        cache, prefix = make([page - 1, page + 1, 5 * page + 130], [2, 1, 20], [3] * 23, 2, page, torch.bfloat16, gen)
        check(selector(16, 2), queries(23, 16, torch.bfloat16, gen), cache, prefix)


def test_unbounded_values_in_sight():
    # Infinities and NaN of a prefix's values reach the rows that see them, in blocks seen wholly and in part.
    gen = torch.Generator().manual_seed(6)
    cache, prefix = make([300, 300], [3, 2], [9] * 5, 2, 16, torch.bfloat16, gen)
    for slot, col, value in ((5, 3, "inf"), (299, 9, "-inf"), (290, 70, "nan"), (299, 3, "inf")):
        cache.v_pages[int(prefix.page_table[0, slot // 16]), 1, slot % 16, col] = float(value)
    out = f64(selector(8, 2).shared_decode(queries(5, 8, torch.bfloat16, gen), cache, prefix))
    kvec.kvec_sync_status(selector(8, 2).handle)
    assert np.all(np.isposinf(out[:3, 4:, 3])) and np.all(np.isneginf(out[:3, 4:, 9])) and np.all(np.isnan(out[:3, 4:, 70]))
    out[:3, 4:, [3, 9, 70]] = 0
    assert np.isfinite(out).all()

def device_time(call):
    """Milliseconds: the least of several."""
    call()
    times = []
    for _ in range(8):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(4):
            call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) / 4)
    return min(times)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_lies_behind_a_prefix_costs_no_time(dtype, bad):
    # The rest of a page may hold anything: the same bits, and no walk for its infinities (which took 60 times the call's time).
    gen = torch.Generator().manual_seed(17)
    cache, prefix = make([500, 140], [4, 3], [1, 17, 40, 23, 5, 6, 7], 8, 256, dtype, gen, weights=False)
    q, sel = queries(7, 32, dtype, gen), selector(32, 8)
    outs, times = [], []
    for fill in (0.0, bad):
        for r, n in enumerate(prefix.lens.tolist()):
            cache.v_pages[int(prefix.page_table[r, (n - 1) // 256]), :, (n - 1) % 256 + 1:] = fill
        outs.append(check(sel, q, cache, prefix))
        times.append(device_time(lambda: sel.shared_decode(q, cache, prefix)))
    assert torch.equal(*outs)
    assert times[1] < 4 * times[0], f"{times[1]:.4f} ms behind infinities, {times[0]:.4f} without"



def test_minus_infinite_logits_have_no_weight():
    gen = torch.Generator().manual_seed(5)
    cache, prefix = make([200, 40], [2, 2], [5, 0, 3, 0], 2, 16, torch.bfloat16, gen)
    for j in range(0, 200, 3):
        cache.k_pages[int(prefix.page_table[0, j // 16]), :, j % 16, 0] = float("-inf")
    for j in range(40):
        cache.k_pages[int(prefix.page_table[1, j // 16]), :, j % 16, 0] = float("-inf")
    q = torch.ones((4, 8, D), dtype=torch.bfloat16, device="cuda")
    out = check(selector(8, 2), q, cache, prefix)
    assert torch.all(out[3] == 0)


def test_logits_far_apart():
    # One part's logits far above the other's, and rows whose maximum moves late.
    gen = torch.Generator().manual_seed(8)
    cache, prefix = make([900], [4], [50] * 4, 2, 16, torch.bfloat16, gen)
    q = queries(4, 8, torch.bfloat16, gen)
    cache.k_pages[int(prefix.page_table[0, 890 // 16]), :, 890 % 16] *= 30
    cache.k_pages[int(cache.page_table[1, 2]), :, 1] *= 60
    check(selector(8, 2), q * 3, cache, prefix)


@pytest.mark.parametrize("dtype,size", [(torch.bfloat16, 2.0 ** 80), (torch.float16, 2.0 ** 10)])
@pytest.mark.parametrize("rise", [20.0, 35.0, 60.0, 200.0])
def test_logits_that_rise_along_the_prefix_and_large_values(dtype, size, rise):
    # Each row's logits grow by `rise` powers of two from the first keys to the last: sums relative to the first maximum, which
    # moves or not, times values that leave little room.
    gen = torch.Generator().manual_seed(int(rise))
    cache, prefix = make([1000], [3], [5, 0, 20], 2, 16, dtype, gen, weights=False)
    for j in range(1000):
        cache.k_pages[int(prefix.page_table[0, j // 16]), :, j % 16, 0] = rise * j / 1000
    cache.v_pages[torch.isfinite(cache.v_pages)] *= size
    q = queries(3, 8, dtype, gen) * 0.25
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    check(selector(8, 2), q, cache, prefix)

@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -100])
@pytest.mark.parametrize("rise", [0.0, 20.0, 35.0, 45.0, 60.0, 200.0])
def test_values_at_the_ends_of_the_range(size, rise):
    # As above, in bf16, with values near the largest and the least that the sums have room for.
    gen = torch.Generator().manual_seed(int(rise) + 1)
    cache, prefix = make([1000], [3], [5, 0, 20], 2, 16, torch.bfloat16, gen, weights=False)
    for j in range(1000):
        cache.k_pages[int(prefix.page_table[0, j // 16]), :, j % 16, 0] = rise * j / 1000
    cache.v_pages[torch.isfinite(cache.v_pages)] *= size / 8     # (below 8 before)
    assert cache.v_pages[torch.isfinite(cache.v_pages)].abs().max() < size
    q = queries(3, 8, torch.bfloat16, gen) * 0.25
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    check(selector(8, 2), q, cache, prefix)


@pytest.mark.parametrize("dtype,size", [(torch.bfloat16, 2.0 ** 100), (torch.bfloat16, 2.0 ** 80), (torch.float16, 60000.0)])
@pytest.mark.parametrize("rise", [6.5, 20.0, 32.5, 33.5, 39.5, 46.5])
def test_long_shares_of_large_values_have_room(dtype, size, rise):
    """Four prefixes of 2^17 slots and eight heads, 221 blocks a CTA: the first block's logits `rise` powers of two below all
    others', so that these meet sums relative to a maximum far below them.  Values are one number, and so are the outputs:
    weights rounded to the type (u), sums and exponentials (4e-5), the type (u)."""
    page, n = 128, 1 << 17
    k = torch.zeros((3, 8, page, D), dtype=dtype, device="cuda")
    v = torch.full_like(k, size)
    k[1:, :, :, 0] = rise
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    table = torch.ones((4, n // page), dtype=torch.int32, device="cuda")
    table[:, 0] = 0                                               # pages are only read: many entries may name one
    prefix = kvec.SharedPrefix(table, ints([n] * 4), ints(range(5)))
    cache = kvec.PagedCache(k, v, torch.full((4, 1), 2, dtype=torch.int32).cuda(), ints([3, 0, 100, 1]))
    q = torch.zeros((4, 32, D), dtype=dtype, device="cuda")
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    sel = selector(32, 8)
    out = f64(sel.shared_decode(q, cache, prefix))
    kvec.kvec_sync_status(sel.handle)
    want, u = float(v[0, 0, 0, 0]), half_step(dtype)
    assert np.all(np.abs(out - want) <= (2 * u + 4e-5) * want)



def test_as_one_cache_of_prefix_and_own_slots():
    # A prefix that fills its pages, read once for all or by every sequence on its own: the same within the roundings.
    gen = torch.Generator().manual_seed(12)
    dtype, lens = torch.float16, [40, 1, 99]
    cache, prefix = make([640], [3], lens, 4, 64, dtype, gen, weights=False)
    q = queries(3, 28, dtype, gen)
    joined = torch.cat([prefix.page_table.expand(3, -1), cache.page_table], 1).contiguous()
    whole = kvec.PagedCache(cache.k_pages, cache.v_pages, joined, cache.lens + 640)
    a, b = f64(selector(28, 4).shared_decode(q, cache, prefix)), f64(selector(28, 4).paged_decode(q, whole))
    vmax = 8.0
    assert np.all(np.abs(a - b) <= 2 * half_step(dtype) * np.abs(b) + (half_step(dtype) + 6e-5 + 2 * 739 * 2.0 ** -25) * vmax)


def test_the_same_bits_every_time():
    gen = torch.Generator().manual_seed(13)
    cache, prefix = make([3000, 700], [40, 20], [(31 * b) % 400 for b in range(60)], 4, 64, torch.bfloat16, gen, weights=False)
    q, sel = queries(60, 28, torch.bfloat16, gen), selector(28, 4)
    first = sel.shared_decode(q, cache, prefix)
    for _ in range(10):
        assert torch.equal(sel.shared_decode(q, cache, prefix), first)


def test_scratch_is_kept_to():
    gen = torch.Generator().manual_seed(14)
    lens = [(13 * b) % 90 for b in range(40)]
    cache, prefix = make([2000, 300, 77], [20, 1, 10], lens, 4, 16, torch.bfloat16, gen)
    q, sel = queries(40, 28, torch.bfloat16, gen), selector(28, 4)
    need = kvec.kvec_shared_decode_bytes(sel.handle, 40, 90, True)
    assert need > 0 and kvec.kvec_shared_decode_bytes(sel.handle, 40, 0, True) == 0
    w0 = cache.weights.clone()
    want = check(sel, q, cache, prefix, max_len=90)
    w1 = cache.weights.clone()
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    cache.weights.copy_(w0)
    out = torch.empty_like(q)
    stream = torch.cuda.current_stream().cuda_stream
    kvec.kvec_shared_decode(sel.handle, 40, q.data_ptr(), cache.c, prefix.c, 90, 2000, out.data_ptr(), room.data_ptr(), need, stream)
    kvec.kvec_sync_status(sel.handle)
    assert torch.equal(out, want) and torch.equal(cache.weights, w1) and torch.all(room[need:] == 0xA5)
    for at, size in ((room.data_ptr(), need - 1), (room.data_ptr() + 16, need)):
        with pytest.raises(kvec.KvecError):
            kvec.kvec_shared_decode(sel.handle, 40, q.data_ptr(), cache.c, prefix.c, 90, 2000, out.data_ptr(), at, size, stream)


def test_page_offsets_past_32_bits():
    Hkv, page, pages = 8, 256, 9000
    k = torch.zeros((pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    assert k.numel() * 2 > 2 ** 32
    v = torch.zeros_like(k)
    gen = torch.Generator().manual_seed(1)
    small, prefix = make([500], [3], [40, 7, 256], Hkv, page, torch.bfloat16, gen, weights=False)
    far = lambda t: torch.where(t < 0, t, pages - 1 - t)
    for p in range(small.k_pages.shape[0]):
        k[pages - 1 - p], v[pages - 1 - p] = small.k_pages[p], small.v_pages[p]
    q = queries(3, 32, torch.bfloat16, gen)
    large = kvec.PagedCache(k, v, far(small.page_table), small.lens)
    sel = selector(32, 8)
    want = check(sel, q, small, prefix)
    assert torch.equal(sel.shared_decode(q, large, kvec.SharedPrefix(far(prefix.page_table), prefix.lens, prefix.cu_seqs)), want)


def test_a_captured_call_takes_groups_and_lengths_of_every_kind():
    gen = torch.Generator().manual_seed(50)
    cache, prefix = make([1000, 700, 90], [25, 10, 5], [300] * 40, 4, 64, torch.bfloat16, gen)
    q, sel, w0 = queries(40, 28, torch.bfloat16, gen), selector(28, 4), cache.weights.clone()
    out = torch.empty_like(q)
    sel.shared_decode(q, cache, prefix, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sel.shared_decode(q, cache, prefix, out=out)
    for plens, cu, lens in (([1000, 700, 90], [0, 25, 35, 40], [300] * 40), ([0, 700, 1], [0, 1, 2, 39], [7 * b for b in range(40)]),
                            ([999, 0, 0], [0, 40, 40, 40], [0] * 40), ([5, 5, 5], [0, 0, 0, 0], [1] * 40)):
        prefix.lens.copy_(torch.tensor(plens, dtype=torch.int32))
        prefix.cu_seqs.copy_(torch.tensor(cu, dtype=torch.int32))
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.weights.copy_(w0)
        graph.replay()
        kvec.kvec_sync_status(sel.handle)
        got, weights = out.clone(), cache.weights.clone()
        cache.weights.copy_(w0)
        want = check(sel, q, cache, prefix)
        assert torch.equal(got, want) and torch.equal(weights, cache.weights)


def test_calls_on_two_streams():
    gen = torch.Generator().manual_seed(21)
    sel, cases, want = selector(28, 4), [], []
    for n in (700, 1300):
        cache, prefix = make([n, 200], [9, 4], [(17 * b) % 99 for b in range(13)], 4, 64, torch.bfloat16, gen, weights=False)
        cases.append((queries(13, 28, torch.bfloat16, gen), cache, prefix))
        want.append(check(sel, *cases[-1]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        outs = [sel.shared_decode(*c, stream=st) for c, st in zip(cases, streams)]
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_steps_of_a_batch_behind_a_prefix():
    """The calls as a program makes them: the prefix stored once, then steps that append each sequence's token and attend,
    and an eviction of what each has of its own; without a gap between the calls."""
    gen = torch.Generator().manual_seed(31)
    dtype, Hq, Hkv, page, batch, P = torch.bfloat16, 28, 4, 32, 5, 150
    sel = selector(Hq, Hkv)
    pages = 5 + 3 * batch + 2 * batch
    k, v = (torch.zeros((pages, Hkv, page, D), dtype=dtype, device="cuda") for _ in range(2))
    w = torch.zeros((pages, Hkv, page), device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    tab = torch.randn((400, 64), generator=gen)
    tab = torch.cat([tab.cos(), tab.sin()], 1).cuda()
    prefix = kvec.SharedPrefix(ints([[4, 2, 0, 1, 3]]), ints([P]), ints([0, batch]))
    x = torch.randn((P, Hq + 2 * Hkv, D), generator=gen).to(dtype).cuda()
    sel.rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], torch.arange(P, dtype=torch.int32).cuda(), tab,
                      kvec.PagedCache(k, v, prefix.page_table, prefix.lens, w), ints([0, P]))
    cache = kvec.PagedCache(k, v, torch.arange(5, 5 + 3 * batch, dtype=torch.int32).view(batch, 3).cuda(), ints([0] * batch), w)
    for step in range(40):
        x = torch.randn((batch, Hq + 2 * Hkv, D), generator=gen).to(dtype).cuda()
        cache.lens += 1
        q = sel.rotate_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], ints([P + step] * batch), tab, cache)
        if step < 38:
            sel.shared_decode(q, cache, prefix)
        else:
            check(sel, q, cache, prefix)
    fresh = torch.arange(5 + 3 * batch, pages, dtype=torch.int32).view(batch, 2).cuda()
    new_lens, kept = sel.paged_evict(cache, fresh, 24, sinks=2, recent=8)
    check(sel, q, kvec.PagedCache(k, v, fresh, new_lens, w), prefix)
    assert new_lens.tolist() == [24] * batch


# ---------------------------------------------------------------- own slots of 8 bits

def make_eight(prefixes, groups, lens, Hkv, page, pool_page, dtype, gen, weights=True):
    """Prefixes in a pool of 16 bits, own slots of 8; NaN numbers and scales past the lengths."""
    pool, prefix = make(prefixes, groups, [0] * len(prefixes), Hkv, pool_page, dtype, gen, weights=False)
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + 1
    perm = torch.randperm(pages, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(1, max(counts))), -1, dtype=torch.int32)
    hole = torch.ones((pages, page), dtype=torch.bool)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = perm[at:at + c]
        at += c
        for j in range(lens[s]):
            hole[table[s, j // page], j % page] = False
    hole = hole[:, None, :].expand(pages, Hkv, page)
    parts = []
    for _ in range(2):
        x = torch.randn((pages, Hkv, page, D), generator=gen)
        scale = x.abs().amax(-1) / 448
        x = (x / scale[..., None]).to(torch.float8_e4m3fn)
        x.view(torch.uint8)[hole] = 0x7f
        scale[hole] = float("nan")
        parts += [x.cuda(), scale.cuda()]
    w = torch.randn((pages, Hkv, page), generator=gen).exp().cuda() if weights else None
    cache = kvec.PagedCache(parts[0], parts[2], table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), w,
                            k_scales=parts[1], v_scales=parts[3], dtype=dtype)
    return cache, kvec.SharedPrefix(prefix.page_table, prefix.lens, prefix.cu_seqs, pool=pool)


def check_eight(sel, q, cache, prefix):
    dtype, u = q.dtype, half_step(q.dtype)
    pool = prefix.pool
    with np.errstate(invalid="ignore"):
        kp, vp = (f64(x) * f64(s)[..., None] for x, s in ((cache.k_pages, cache.k_scales), (cache.v_pages, cache.v_scales)))
    w0 = f64(cache.weights)
    w = None if w0 is None else w0.copy()
    lens, plens, pv = cache.lens.tolist(), prefix.lens.tolist(), f64(pool.v_pages)
    ref = serving.shared_decode(f64(q), kp, vp, w, cache.page_table.cpu().numpy(), lens, cache.capacity,
                                prefix.page_table.cpu().numpy(), plens, prefix.cu_seqs.tolist(),
                                prefix.max_pages * pool.page_size, 1 / np.sqrt(D), pool=(f64(pool.k_pages), pv))
    out = sel.shared_decode(q, cache, prefix)
    kvec.kvec_sync_status(sel.handle)
    vmax = max(np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in (vp, pv))
    n = max(plens) + max(lens)
    tol = u * np.abs(ref) + (u + 4e-5 + (n * 2.0 ** -25 if dtype == torch.float16 else 0.0)) * vmax
    assert np.all(np.abs(f64(out) - ref) <= tol)
    if w is not None:
        assert np.all(np.abs(f64(cache.weights) - w) <= 4e-5 * (w - w0) + 2.0 ** -24 * np.abs(w) + 1e-9)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,page,pool_page,prefixes,groups,lens,weights", [
    (32, 8, 16, 64, [128], [3], [1, 40, 16], True),
    (28, 4, 64, 16, [500, 0], [4, 1], [1, 17, 0, 23, 5], True),
    (16, 2, 128, 256, [700, 33], [20, 30], [(11 * i) % 190 for i in range(55)], False),
    (8, 4, 32, 32, [333], [41], [600 + (37 * b) % 100 for b in range(60)], True),            # a CTA a pair
    (8, 4, 16, 128, [333, 64], [41, 14], [5000] + [0, 30] * 29 + [7], True),                 # shares
    (8, 1, 256, 128, [40], [6], [0] * 6, True),
])
def test_own_slots_of_eight_bits(dtype, Hq, Hkv, page, pool_page, prefixes, groups, lens, weights):
    gen = torch.Generator().manual_seed(sum(lens) + page)
    cache, prefix = make_eight(prefixes, groups, lens, Hkv, page, pool_page, dtype, gen, weights)
    q = queries(len(lens), Hq, dtype, gen)
    check_eight(selector(Hq, Hkv), q, cache, prefix)
    check_eight(selector(Hq, Hkv), q, cache, prefix)

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[40, 0, 700], [9000, 3, 1], [600 + (37 * b) % 100 for b in range(75)]])
def test_a_large_scale_without_weight_costs_the_others_nothing(dtype, lens):
    """Own slots whose values' scales are 2^40 times the others' and whose logits are 104 (base 2) below.  Each output against its
    own size, sum_j p_j |v_j|: u for a prefix's weights, 4e-5 and a rounding as above, and 2^-22 of a product of weight and
    scale or 2^-39 of the largest, n 448 2^-39 of sum_j p_j |s_j| for n slots of numbers up to 448 (a prefix's slots, whose
    values are below 8, count as scales of 8)."""
    gen = torch.Generator().manual_seed(sum(lens))
    cache, prefix = make_eight([300], [len(lens)], lens, 4, 32, 64, dtype, gen, weights=False)
    numbers = torch.zeros(D)
    numbers[0] = 1.0
    numbers = numbers.to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    for s, n in enumerate(lens):
        for j in [*range(min(n // 4, 50)), *range(n - n // 5, n, 7)]:
            at, ofs = int(cache.page_table[s, j // 32]), j % 32
            cache.k_pages.view(torch.uint8)[at, :, ofs] = numbers
            cache.k_scales[at, :, ofs] = -104.0
            cache.v_scales[at, :, ofs] *= 2.0 ** 40
    q = torch.randn((len(lens), 8, D), generator=gen)
    q[:, :, 0] = np.sqrt(D) * np.log(2.0)
    q, pool, sel = q.to(dtype).cuda(), prefix.pool, selector(8, 4)
    with np.errstate(invalid="ignore"):
        kp, vp = (f64(x) * f64(s)[..., None] for x, s in ((cache.k_pages, cache.k_scales), (cache.v_pages, cache.v_scales)))
    scales, pv = np.broadcast_to(np.abs(f64(cache.v_scales))[..., None], vp.shape), f64(pool.v_pages)
    assert np.abs(pv[np.isfinite(pv)]).max() < 8
    ref, size, top = (serving.shared_decode(f64(q), kp, own, None, cache.page_table.cpu().numpy(), lens, cache.capacity,
                                            prefix.page_table.cpu().numpy(), prefix.lens.tolist(), prefix.cu_seqs.tolist(),
                                            300, 1 / np.sqrt(D), pool=(f64(pool.k_pages), x))
                      for own, x in ((vp, pv), (np.abs(vp), np.abs(pv)), (scales, np.full_like(pv, 8.0))))
    out = f64(sel.shared_decode(q, cache, prefix, max_prefix=300))
    kvec.kvec_sync_status(sel.handle)
    u = half_step(dtype)
    tol = u * np.abs(ref) + (u + 4e-5 + 2.0 ** -22) * size + max(lens) * 448 * 2.0 ** -39 * top
    tol += 300 * 2.0 ** -25 * 8 + 2.0 ** -25 if dtype == torch.float16 else 0.0
    assert np.all(np.abs(out - ref) <= tol)



def test_own_slots_of_eight_bits_captured_and_on_another_stream():
    gen = torch.Generator().manual_seed(91)
    cache, prefix = make_eight([700, 100], [9, 4], [(17 * b) % 99 for b in range(15)], 4, 64, 32, torch.bfloat16, gen, weights=False)
    q, sel = queries(15, 28, torch.bfloat16, gen), selector(28, 4)
    want = check_eight(sel, q, cache, prefix)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        other = sel.shared_decode(q, cache, prefix, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(other, want) and torch.equal(sel.shared_decode(q, cache, prefix), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sel.shared_decode(q, cache, prefix)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_wait_that_runs_out_is_reported():
    gen = torch.Generator().manual_seed(2)
    cache, prefix = make([300], [2], [20, 4], 2, 16, torch.bfloat16, gen)
    q, sel = queries(2, 8, torch.bfloat16, gen), selector(8, 2)
    kvec.kvec_set_test_fault(4)
    try:
        sel.shared_decode(q, cache, prefix)
        with pytest.raises(kvec.KvecError) as e:
            kvec.kvec_sync_status(sel.handle)
        assert e.value.status == kvec.KVEC_ERR_DEVICE_TIMEOUT
    finally:
        kvec.kvec_set_test_fault(0)
    cache.weights.zero_()
    check(sel, q, cache, prefix)
