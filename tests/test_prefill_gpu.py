"""GPU parity of prefill attention (kvec_prefill_attention) with its definition in fp64.

Tolerances.  u is half a step of the 16-bit type relative to the value (bf16 2^-8, fp16 2^-11).  The weights are
rounded to the type before they meet the values, which moves the output by at most u sum_t p_t |v_t| (fp16 also by
2^-25 of the largest weight each, n 2^-25 max|v| over n keys); the logits are fp32 sums of exact products and the
exponentials approximate, 2e-5 sum_t p_t |v_t|; the result is rounded once, u |ref|.  The log-sum-exp is fp32: the
logits' 2e-5 and 2^-22 of its value.
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
        _SELECTORS[key] = kvec.KvecSelector(kvec.make_params(Hq, Hkv, num_ext_heads=1, max_batch=64, max_seqlen=64,
                                                             max_layers=1, softmax_scale=scale))
    return _SELECTORS[key]


def cu_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32)


def reference(q, k, v, q_lens, k_lens, window, sinks, scale):
    """out, lse and sum of p |v| in fp64 on the GPU, head by head; masked places count for nothing, whatever they hold."""
    q, k, v = q.double(), k.double(), v.double()
    g = q.shape[1] // k.shape[1]
    out, mass = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -np.inf, dtype=torch.float64, device=q.device)
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        p = torch.arange(nk - nq, nk, device=q.device)[:, None]
        t = torch.arange(nk, device=q.device)[None, :]
        seen = t <= p
        if window:
            seen = seen & ((t > p - window) | (t < sinks))
        for h in range(q.shape[1]):
            if nq == 0 or nk == 0:
                continue
            kk, vv = k[k0:k0 + nk, h // g], v[k0:k0 + nk, h // g]
            x = (q[q0:q0 + nq, h] @ kk.nan_to_num(0, 0, 0).T * scale)
            bad = ~torch.isfinite(kk).all(-1)
            assert not (seen & bad[None, :]).any(), "the reference takes unbounded keys in masked places only"
            x = x.masked_fill(~seen, -np.inf)
            lse[q0:q0 + nq, h] = torch.logsumexp(x, -1)
            w = torch.exp(x - lse[q0:q0 + nq, h, None].clamp(min=-1e300))
            fine = vv.nan_to_num(0, 0, 0)
            o = w @ fine
            # What is infinite or NaN in V reaches the rows that see it.
            for i in torch.nonzero(~torch.isfinite(vv).all(-1)).flatten().tolist():
                part = torch.where(torch.isfinite(vv[i]), torch.zeros_like(vv[i]), vv[i])
                o = torch.where(seen[:, i, None], o + part, o)
            out[q0:q0 + nq, h] = o
            mass[q0:q0 + nq, h] = w @ fine.abs()
        q0, k0 = q0 + nq, k0 + nk
    return out, lse, mass


def check(q, k, v, q_lens, k_lens, window=0, sinks=0, scale=None, **kw):
    dtype, u = q.dtype, torch.finfo(q.dtype).eps / 2
    sel = selector(q.shape[1], k.shape[1], scale or 0.0)
    cu_q, cu_k = cu_of(q_lens), cu_of(k_lens)
    out, lse = sel.prefill_attention(q, k, v, cu_q, cu_q.cuda(), cu_k, cu_k.cuda(), window=window, sinks=sinks, **kw)
    kvec.kvec_sync_status(sel.handle)
    n = sum(q_lens)
    ref, rl, mass = reference(q[:n], k, v, q_lens, k_lens, window, sinks, scale or D ** -0.5)
    got = out[:n].double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[torch.isinf(ref)], ref[torch.isinf(ref)])
    most = max(list(k_lens) + [1])
    tol = u * ref.abs() + (u + 2e-5) * mass + (most * 2.0 ** -25 * 8 if dtype == torch.float16 else 0) + 1e-30
    bad = fine & ~((got - ref).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, by up to {float((got - ref)[fine].abs().max()):.3e}; rows {torch.nonzero(bad.any(-1))[:8].tolist()}"
    gl = lse[:n].double()
    none = torch.isneginf(rl)
    assert torch.equal(torch.isneginf(gl), none) and torch.all(got[none] == 0)
    bad = ~none & ~((gl - rl).abs() <= 2e-5 + 2.0 ** -22 * rl.abs())
    assert not bad.any(), f"lse off by up to {float((gl - rl)[~none].abs().max()):.3e}"
    return out, lse


def tensors(q_lens, k_lens, Hq, Hkv, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    mk = lambda n, h, s=1.0: (torch.randn((n, h, D), generator=gen) * s).to(dtype).cuda()
    return mk(sum(q_lens), Hq, std), mk(sum(k_lens), Hkv), mk(sum(k_lens), Hkv)


SHAPES = [
    (1, 1, [1], [1]), (4, 1, [1], [300]), (8, 8, [5], [5]), (32, 8, [33], [1057]), (28, 4, [33], [200]),
    (8, 2, [128], [128]), (8, 1, [129], [129]), (7, 1, [100], [127]), (12, 4, [300, 1, 64], [300, 500, 64]),
    (16, 8, [257, 0, 3], [700, 12, 2]),                    # no queries; more queries than keys: rows that see nothing
    (6, 2, [10, 4], [0, 4]),                               # no keys
    (4, 4, [1000], [1000]), (5, 1, [700], [1500]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,q_lens,k_lens", SHAPES)
def test_causal(dtype, Hq, Hkv, q_lens, k_lens):
    q, k, v = tensors(q_lens, k_lens, Hq, Hkv, dtype, sum(q_lens) + 7 * sum(k_lens), 2.0)
    check(q, k, v, q_lens, k_lens)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (127, 4), (128, 0), (129, 128), (200, 200), (5, 1000), (4000, 3)])
@pytest.mark.parametrize("Hq,Hkv,q_lens,k_lens", [(8, 2, [700], [700]), (28, 4, [33, 200], [1057, 600]), (4, 4, [1], [513])])
def test_windows_and_first_tokens(Hq, Hkv, q_lens, k_lens, window, sinks):
    q, k, v = tensors(q_lens, k_lens, Hq, Hkv, torch.bfloat16, window + sinks)
    check(q, k, v, q_lens, k_lens, window, sinks)


def test_against_the_plain_definition_row_by_row():
    q_lens, k_lens = [40, 9], [90, 5]
    q, k, v = tensors(q_lens, k_lens, 4, 2, torch.float16, 1)
    f = lambda x: x.double().cpu().numpy()
    for window, sinks in ((0, 0), (20, 3)):
        ref, lse, _ = reference(q, k, v, q_lens, k_lens, window, sinks, D ** -0.5)
        out, z = serving.prefill(f(q), f(k), f(v), cu_of(q_lens).tolist(), cu_of(k_lens).tolist(), window, sinks, D ** -0.5)
        assert np.allclose(ref.cpu().numpy(), out, atol=1e-12) and np.allclose(lse.cpu().numpy(), z, atol=1e-12)
        check(q, k, v, q_lens, k_lens, window, sinks)


def test_the_running_maximum_moves():
    # Logits that grow along the keys by far more than the lazy rescale's threshold, and far down from a first peak.
    q, k, v = tensors([600], [600], 8, 2, torch.bfloat16, 3)
    up = torch.linspace(-30, 30, 600, device="cuda")[:, None]
    q[:, :, 0] = 8.0
    for ramp in (up, -up, up.abs() * (-1) ** (torch.arange(600, device="cuda") // 128)[:, None]):
        k[:, :, 0] = ramp.to(k.dtype)
        check(q, k, v, [600], [600])
        check(q, k, v, [600], [600], 150, 2)


def test_masked_places_hold_anything():
    # Rows behind each sequence and keys that the window has left or a row does not see yet.
    q_lens, k_lens = [30, 200], [300, 200]
    q, k, v = tensors(q_lens, [300, 200, 150], 8, 2, torch.bfloat16, 5)
    k[500:], v[500:] = float("nan"), float("inf")
    k[2:300 - 30 - 63], v[2:300 - 30 - 63] = float("nan"), float("-inf")   # before the window of 64 of every row
    check(q, k, v, q_lens, k_lens, 64, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("where", [0, 60, 150, 255, 299])
def test_unbounded_values_reach_only_the_rows_that_see_them(dtype, where):
    q, k, v = tensors([300], [300], 8, 2, dtype, where)
    v[where, 0, 5], v[where, 1, 100] = float("inf"), float("nan")
    v[min(where + 3, 299), 0, 70] = float("-inf")
    check(q, k, v, [300], [300])
    check(q, k, v, [300], [300], 40, 1)


def test_minus_infinite_logits():
    q, k, v = tensors([200], [200], 4, 4, torch.bfloat16, 8)
    ref = q.clone()
    q[:, :, 0] = 1.0
    k2 = k.clone()
    k2[::2, :, 0] = float("-inf")
    cu = cu_of([200])
    out, lse = selector(4, 4).prefill_attention(q, k2, v, cu, cu.cuda())
    assert torch.all(out[0] == 0) and torch.all(torch.isneginf(lse[0]))     # row 0 sees key 0 alone
    x = torch.einsum("qhd,khd->hqk", q.double(), k.double()) * D ** -0.5
    t = torch.arange(200, device="cuda")
    x = x.masked_fill((t[None, :] > t[:, None]) | (t[None, :] % 2 == 0), -np.inf)
    want = torch.einsum("hqk,khd->qhd", torch.softmax(x, -1).nan_to_num(0), v.double())
    assert torch.isfinite(out).all() and (out.double() - want).abs().max() < 0.05 and ref is not None


def test_a_softmax_scale_of_the_handle():
    q, k, v = tensors([150], [150], 4, 2, torch.float16, 10)
    check(q, k, v, [150], [150], scale=0.5)


def test_rows_behind_the_last_sequence_stay():
    q, k, v = tensors([50], [50], 8, 2, torch.bfloat16, 12)
    out = torch.full_like(q, 9.0)
    lse = torch.full((50, 8), 9.0, device="cuda")
    check(q, k, v, [20, 11], [20, 11], out=out, lse=lse)
    assert torch.all(out[31:] == 9.0) and torch.all(lse[31:] == 9.0) and torch.isfinite(lse).all()


def test_long_rows_and_many_tiles():
    q, k, v = tensors([4096, 1111], [4096, 3333], 8, 2, torch.bfloat16, 14, 2.0)
    check(q, k, v, [4096, 1111], [4096, 3333])
    check(q, k, v, [4096, 1111], [4096, 3333], 512, 4)


def test_captured_and_on_two_streams():
    sel = selector(8, 2)
    cu = cu_of([500, 33])
    dev = cu.cuda()
    sets = [tensors([500, 33], [500, 33], 8, 2, torch.bfloat16, s) for s in (20, 21)]
    want = [sel.prefill_attention(*x, cu, dev) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        got = [sel.prefill_attention(*x, cu, dev, stream=s) for x, s in zip(sets, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    gr = torch.cuda.CUDAGraph()
    x = [t.clone() for t in sets[0]]
    with torch.cuda.graph(gr):
        out, lse = sel.prefill_attention(*x, cu, dev)
    for s, w in zip(sets[::-1], want[::-1]):
        for a, b in zip(x, s):
            a.copy_(b)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w[0]) and torch.equal(lse, w[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,q_lens,k_lens,window,sinks", [
    (28, 4, [1], [20000], 0, 0), (8, 1, [33, 2, 5], [5000, 300, 1], 0, 0), (32, 8, [64], [3001], 0, 0),
    (4, 2, [100], [9000], 4096, 130), (8, 8, [7], [700], 0, 0), (16, 2, [20, 0], [1500, 800], 300, 4),
])
def test_few_rows_on_many_keys(dtype, Hq, Hkv, q_lens, k_lens, window, sinks):
    # The keys of a row are divided over the device; parts of a short sequence see nothing.
    sel = selector(Hq, Hkv)
    cu_q, cu_k = cu_of(q_lens), cu_of(k_lens)
    assert kvec.kvec_prefill_bytes(sel.handle, len(q_lens), cu_q.data_ptr(), cu_k.data_ptr(), window, sinks) > 0
    q, k, v = tensors(q_lens, k_lens, Hq, Hkv, dtype, sum(k_lens), 2.0)
    check(q, k, v, q_lens, k_lens, window, sinks)
    # Logits that jump between the parts, and values without bounds in the blocks of partial sight.
    k[:, :, 0] = torch.where(torch.arange(k.shape[0], device="cuda") % 1000 < 500, 20.0, -20.0)[:, None].to(dtype)
    q[:, :, 0] = 5.0
    check(q, k, v, q_lens, k_lens, window, sinks)
    v[k_lens[0] - 1, 0, 3], v[k_lens[0] - min(k_lens[0], 2), 0, 77] = float("nan"), float("inf")
    check(q, k, v, q_lens, k_lens, window, sinks)


def test_windows_and_first_tokens_of_any_size():
    q, k, v = tensors([90], [700], 8, 2, torch.bfloat16, 40)
    cq, ck = cu_of([90]), cu_of([700])
    run = lambda w, s: selector(8, 2).prefill_attention(q, k, v, cq, cq.cuda(), ck, ck.cuda(), window=w, sinks=s)
    whole, most = run(0, 0), 2 ** 31 - 1
    for window, sinks in ((most, 0), (most, most), (2 ** 20, 7)):
        got = run(window, sinks)
        assert torch.equal(got[0], whole[0]) and torch.equal(got[1], whole[1])
    got = run(1, most)   # every key by the first tokens' rule: other blocks are looked at, the same rows come out
    assert (got[1] - whole[1]).abs().max() <= 4e-5 and torch.all((got[0] - whole[0]).abs().float() <= 0.02)


def test_rows_that_fill_no_tile_do_not_matter():
    # Seven heads leave two of a tile's 128 rows unused; what shared memory holds there is not the call's.
    q, k, v = tensors([200], [600], 7, 1, torch.bfloat16, 41)
    big = [torch.full((400, 8, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    cu8, cu = cu_of([400]), cu_of([200])
    ck = cu_of([600])
    want = selector(7, 1).prefill_attention(q, k, v, cu, cu.cuda(), ck, ck.cuda())
    selector(8, 8).prefill_attention(*big, cu8, cu8.cuda())      # leaves NaN in shared memory
    got = selector(7, 1).prefill_attention(q, k, v, cu, cu.cuda(), ck, ck.cuda())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# Sequences of very different lengths: of the places for the longest one's tiles most are unused.
RAGGED = [
    [1500] + [60] * 3, [1, 0, 700, 0, 0, 130, 2000], [100] * 40 + [1300], [0] * 35 + [900, 5] + [0] * 20,
    list(range(0, 640, 10)),                              # 64 lengths, each with its own number of tiles
]


@pytest.mark.parametrize("lens", RAGGED)
@pytest.mark.parametrize("Hq,Hkv,window,sinks", [(8, 8, 0, 0), (32, 8, 0, 0), (28, 4, 100, 3)])
def test_sequences_of_very_different_lengths(lens, Hq, Hkv, window, sinks):
    q, k, v = tensors(lens, lens, Hq, Hkv, torch.bfloat16, sum(lens), 2.0)
    check(q, k, v, lens, lens, window, sinks)
    keys = [n + 37 * (i % 3) for i, n in enumerate(lens)]
    q, k, v = tensors(lens, keys, Hq, Hkv, torch.float16, sum(lens) + 1, 2.0)
    check(q, k, v, lens, keys, window, sinks)


def test_lengths_on_the_device_below_those_announced():
    # A captured call is replayed with shorter sequences: what the device says counts, rows behind it stay.
    lens, then = [900, 300, 1200, 40], [700, 0, 260, 39]
    q, k, v = tensors(lens, lens, 32, 8, torch.bfloat16, 77)
    sel, cu = selector(32, 8), cu_of(lens)
    dev = cu.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    run = lambda: sel.prefill_attention(q, k, v, cu, dev, cu, dev, out=out, lse=lse)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    dev.copy_(cu_of(then))
    out.fill_(7.0)
    graph.replay()
    kvec.kvec_sync_status(sel.handle)
    n = sum(then)
    ref, rl, mass = reference(q[:n], k[:n], v[:n], then, then, 0, 0, D ** -0.5)
    u = torch.finfo(torch.bfloat16).eps / 2
    assert torch.all((out[:n].double() - ref).abs() <= u * ref.abs() + (u + 2e-5) * mass)
    assert torch.all((lse[:n].double() - rl).abs() <= 2e-5 + 2.0 ** -22 * rl.abs())
    assert torch.all(out[n:] == 7.0)


def test_a_wait_that_runs_out_among_sequences_of_different_lengths():
    lens = [2000, 100, 300, 50]
    q, k, v = tensors(lens, lens, 32, 8, torch.bfloat16, 78)
    sel = kvec.KvecSelector(kvec.make_params(32, 8, num_ext_heads=1, max_batch=64, max_seqlen=64, max_layers=1))
    cu = cu_of(lens)
    run = lambda: sel.prefill_attention(q, k, v, cu, cu.cuda())[0]
    want = run().clone()
    kvec.kvec_sync_status(sel.handle)
    try:
        kvec.kvec_set_test_fault(4)
        run()
        with pytest.raises(kvec.KvecError) as e:
            kvec.kvec_sync_status(sel.handle)
        assert e.value.status == kvec.KVEC_ERR_DEVICE_TIMEOUT
    finally:
        kvec.kvec_set_test_fault(0)
    kvec.kvec_sync_status(sel.handle)
    assert torch.equal(run(), want)
    sel.close()


# Sequences with far more queries than keys: most tiles hold rows before the first key and see nothing, and a CTA meets
# runs of such tiles (of six in the first, of four in the last) between or behind those that do.
MOSTLY_UNSEEING = [
    (32, 8, [8192, 1], [64, 1]), (32, 8, [5000, 3000, 700], [300, 10, 700]), (28, 4, [300, 9000, 20], [300, 100, 20]),
    (32, 8, [6000, 500, 40], [0, 500, 90]), (16, 8, [9000, 4000, 100], [500, 0, 100]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv,q_lens,k_lens", MOSTLY_UNSEEING)
def test_far_more_queries_than_keys(dtype, Hq, Hkv, q_lens, k_lens):
    q, k, v = tensors(q_lens, k_lens, Hq, Hkv, dtype, sum(q_lens), 2.0)
    check(q, k, v, q_lens, k_lens)
    check(q, k, v, q_lens, k_lens, 50, 2)


def test_a_captured_call_meets_far_fewer_keys():
    # The lengths of the keys on the device fall behind those announced, and most rows see nothing any more.
    lens, keys = [4096, 300, 1500], [100, 300, 20]
    q, k, v = tensors(lens, lens, 32, 8, torch.bfloat16, 79)
    sel, cu = selector(32, 8), cu_of(lens)
    dq, dk = cu.cuda(), cu.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    run = lambda: sel.prefill_attention(q, k, v, cu, dq, cu, dk, out=out, lse=lse)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    dk.copy_(cu_of(keys))
    graph.replay()
    kvec.kvec_sync_status(sel.handle)
    ref, rl, mass = reference(q, k, v, lens, keys, 0, 0, D ** -0.5)
    u = torch.finfo(torch.bfloat16).eps / 2
    assert torch.all((out.double() - ref).abs() <= u * ref.abs() + (u + 2e-5) * mass)
    none = torch.isneginf(rl)
    assert torch.equal(torch.isneginf(lse), none) and torch.all(out[none] == 0)
    assert torch.all((lse.double() - rl)[~none].abs() <= 2e-5 + 2.0 ** -22 * rl[~none].abs())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q_lens,k_lens", [([200], [200]), ([20], [3000]), ([700, 20, 40], [700, 300, 40])])
@pytest.mark.parametrize("hit", ["every other", "the first blocks", "all but one"])
def test_minus_infinite_logits_count_for_nothing(dtype, q_lens, k_lens, hit):
    # One tile after another, divided keys, and sequences of different lengths; every row by the tolerances above.
    q, k, v = tensors(q_lens, k_lens, 4, 4, dtype, sum(k_lens) + 1)
    q[:, :, 0] = 1.0
    out_of = torch.zeros(sum(k_lens), dtype=torch.bool, device="cuda")
    at = 0
    for n in k_lens:
        here = out_of[at:at + n]
        if hit == "every other":
            here[::2] = True
        elif hit == "the first blocks":
            here[:n - n // 3] = True
        else:
            here[:] = True
            here[n // 2] = False
        at += n
    k2 = torch.where(out_of[:, None, None] & (torch.arange(D, device="cuda") == 0), torch.full_like(k, -np.inf), k)
    sel, cq, ck = selector(4, 4), cu_of(q_lens), cu_of(k_lens)
    out, lse = sel.prefill_attention(q, k2, v, cq, cq.cuda(), ck, ck.cuda())
    kvec.kvec_sync_status(sel.handle)
    u, q0, k0 = torch.finfo(dtype).eps / 2, 0, 0
    for nq, nk in zip(q_lens, k_lens):
        a, b, c = q[q0:q0 + nq].double(), k[k0:k0 + nk].double(), v[k0:k0 + nk].double()
        x = torch.einsum("qhd,khd->hqk", a, b) * D ** -0.5
        t, p = torch.arange(nk, device="cuda"), torch.arange(nk - nq, nk, device="cuda")
        x = x.masked_fill((t[None, :] > p[:, None]) | out_of[k0:k0 + nk][None, :], -np.inf)
        z = torch.logsumexp(x, -1)
        w = torch.exp(x - z.clamp(min=-1e300)[..., None])
        ref, mass = torch.einsum("hqk,khd->qhd", w, c), torch.einsum("hqk,khd->qhd", w, c.abs())
        got, gl, z = out[q0:q0 + nq].double(), lse[q0:q0 + nq].double(), z.T
        tol = u * ref.abs() + (u + 2e-5) * mass + (nk * 2.0 ** -25 * 8 if dtype == torch.float16 else 0)
        assert torch.all((got - ref).abs() <= tol)
        none = torch.isneginf(z)
        assert torch.equal(torch.isneginf(gl), none) and torch.all(got[none] == 0)
        assert torch.all((gl - z)[~none].abs() <= 2e-5 + 2.0 ** -22 * z[~none].abs())
        q0, k0 = q0 + nq, k0 + nk
