"""The operators of a serving loop run together, as they would be used: a ragged prompt through rotation, prefill
attention and the eviction that takes its log-sum-exp, the kept rows into pages, then decoding steps with
rotation, store, attention and eviction by accumulated weight, on eager calls and from a captured graph.

Every step is compared with its definition in fp64 on the state that the GPU has (keys as stored, weights as
accumulated), with the tolerances of the operators' own tests.
"""
import numpy as np
import pytest
import torch

from oracle import serving
from paper_2606_29563_gb300 import kvec
import test_paged_gpu as paged
import test_prefill_gpu as prefill

pytestmark = pytest.mark.gpu
D, HQ, HKV, PAGE = 128, 16, 4, 32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2606_29563_gb300 import build as kbuild
    kbuild.build()


def selector():
    return kvec.KvecSelector(kvec.make_params(HQ, HKV, num_ext_heads=1, max_batch=4, max_seqlen=1024, max_layers=4))


def test_prompt_eviction_and_decoding():
    dtype, lens, budget, w = torch.bfloat16, [700, 333, 90], 128, 32
    gen = torch.Generator().manual_seed(77)
    sel = selector()
    T, cu = sum(lens), prefill.cu_of(lens)
    cu_host, cu_dev = cu.pin_memory(), cu.cuda()
    tab = paged.rot_table(900, D).cuda()
    norms = [(torch.randn(D, generator=gen) * 0.2 + 1).to(dtype).cuda() for _ in range(2)]
    qkv = torch.randn((T, HQ + 2 * HKV, D), generator=gen).to(dtype).cuda()
    pos = torch.cat([torch.arange(n) for n in lens]).int()
    v = qkv[:, HQ + HKV:].contiguous()
    q, k = sel.rotate_append(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], None, pos.cuda(), tab, cu_tokens=cu_dev, q_norm=norms[0], k_norm=norms[1])
    rows = paged.f64(tab)[pos.numpy()]
    paged.check_rows(q, serving.rotate(paged.f64(qkv[:, :HQ]), paged.f64(norms[0]), 1e-6, rows, False), dtype, "q")
    paged.check_rows(k, serving.rotate(paged.f64(qkv[:, HQ:HQ + HKV]), paged.f64(norms[1]), 1e-6, rows, False), dtype, "k")
    out, lse = sel.prefill_attention(q, k, v, cu_host, cu_dev)
    ref, rl, mass = prefill.reference(q, k, v, lens, lens, 0, 0, D ** -0.5)
    u = 2.0 ** -8
    assert torch.all((out.double() - ref).abs() <= u * ref.abs() + (u + 2e-5) * mass)
    assert torch.all((lse.double() - rl).abs() <= 2e-5 + 2.0 ** -22 * rl.abs())

    # The eviction with the prefill's log-sum-exp scores as the one that forms it itself.
    ends = np.cumsum(lens)
    q_obs = torch.stack([q[e - w:e] for e in ends])
    lse_obs = torch.stack([lse[e - w:e] for e in ends])
    got = []
    for given in (None, lse_obs):
        state = sel.new_state(3)
        idx, kk, vv = sel.select_layer(cu_host, cu_dev, q_obs, k, v, state, budget, lse=given)
        kvec.kvec_sync_status(sel.handle)
        got.append((idx.cpu().numpy(), kk, vv, sel.debug()["P_O"].cpu().numpy()))
    for s, n in enumerate(lens):
        if n > budget:
            a, b = got[0][3][s, :, :n - w], got[1][3][s, :, :n - w]
            assert np.abs(a - b).max() <= 2e-3 * (np.abs(a) + a.mean()).max()
    idx, kept_k, kept_v = got[1][:3]
    held = [min(n, budget) for n in lens]
    for s, n in enumerate(lens):
        base = ends[s] - n
        for h in range(HKV):
            j = torch.from_numpy(idx[s, h, :held[s]]).long().cuda()
            assert torch.equal(kept_k[s, h, :held[s]], k[base + j, h]) and torch.equal(kept_v[s, h, :held[s]], v[base + j, h])

    # Pages for the kept rows and 40 decoded tokens, and as many for the cache after each eviction.
    per = -(-(budget + 40) // PAGE)
    pool = torch.randperm(6 * per, generator=gen).to(torch.int32)
    tables = [pool[:3 * per].view(3, per).contiguous().cuda(), pool[3 * per:].view(3, per).contiguous().cuda()]
    pages = [torch.full((6 * per, HKV, PAGE, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    weights = torch.zeros((6 * per, HKV, PAGE), device="cuda")
    for s in range(3):
        for j in range(held[s]):
            at = int(tables[0][s, j // PAGE])
            pages[0][at, :, j % PAGE], pages[1][at, :, j % PAGE] = kept_k[s, :, j], kept_v[s, :, j]
    seq = torch.tensor(held, dtype=torch.int32).cuda()
    positions = torch.tensor(lens, dtype=torch.int32).cuda()
    one = torch.ones(3, dtype=torch.int32).cuda()
    cache = kvec.PagedCache(pages[0], pages[1], tables[0], seq, weights)
    static = torch.zeros((3, HQ + 2 * HKV, D), dtype=dtype, device="cuda")

    def step():
        seq.add_(one)
        qq = sel.rotate_append(static[:, :HQ], static[:, HQ:HQ + HKV], static[:, HQ + HKV:], positions, tab, cache,
                               q_norm=norms[0], k_norm=norms[1])
        positions.add_(one)
        return qq, sel.paged_decode(qq, cache, window=0)

    graph, which = None, 0
    for i in range(36):
        static.copy_(torch.randn(static.shape, generator=gen).to(dtype))
        before = weights.cpu().double().numpy()
        if i in (5, 21):
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                qq, out = step()
        if graph is None:
            qq, out = step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        n = seq.tolist()
        rows = paged.f64(tab)[positions.cpu().numpy() - 1]
        paged.check_rows(qq, serving.rotate(paged.f64(static[:, :HQ]), paged.f64(norms[0]), 1e-6, rows, False), dtype, "q")
        new_k = serving.rotate(paged.f64(static[:, HQ:HQ + HKV]), paged.f64(norms[1]), 1e-6, rows, False)
        kp, vp = paged.f64(pages[0]), paged.f64(pages[1])
        for s in range(3):
            at = serving.place(tables[which][s].tolist(), n[s] - 1, PAGE, 6 * per)
            paged.check_rows(torch.from_numpy(kp[at[0], :, at[1]]), new_k[s], dtype, "stored key")
            assert np.array_equal(vp[at[0], :, at[1]], paged.f64(static[s, HQ + HKV:]))
            before[at[0], :, at[1]] = 0.0
        grown = before.copy()
        ref = serving.paged_decode(paged.f64(qq), kp, vp, grown, tables[which].cpu().numpy(), n, per * PAGE, 0, 0, D ** -0.5)
        assert np.all(np.abs(paged.f64(out) - ref) <= u * np.abs(ref) + (u * u + 2e-5) * 8.0)
        got_w = weights.cpu().double().numpy()
        assert np.all(np.abs(got_w - grown) <= 2e-5 * (grown - before) + 2.0 ** -24 * np.abs(grown) + 1e-9)
        if i % 16 == 15:   # back to the budget, into the other pages
            kp, vp, wp = paged.f64(pages[0]), paged.f64(pages[1]), got_w.copy()
            rl, rk = serving.evict(kp, vp, wp, tables[which].cpu().numpy(), n, tables[1 - which].cpu().numpy(), per * PAGE, budget, 4, 16)
            nl, kept = sel.paged_evict(cache, tables[1 - which], budget, sinks=4, recent=16)
            torch.cuda.synchronize()
            assert np.array_equal(nl.cpu().numpy(), rl) and np.array_equal(kept.cpu().numpy(), rk)
            assert np.array_equal(paged.f64(pages[0]), kp, equal_nan=True) and np.array_equal(weights.cpu().double().numpy(), wp)
            which = 1 - which
            seq.copy_(nl)
            cache = kvec.PagedCache(pages[0], pages[1], tables[which], seq, weights)
            graph = None
    sel.close()


def test_streaming_with_first_slots_and_a_window():
    # Chunks of a prompt under a window with four first tokens in sight, then steps over the pages that
    # hold the last of them: the same rows by both attentions.
    dtype, n, window, sinks = torch.float16, 300, 100, 4
    gen = torch.Generator().manual_seed(5)
    sel = selector()
    q, k, v = (torch.randn((n, h, D), generator=gen).to(dtype).cuda() for h in (HQ, HKV, HKV))
    cu = prefill.cu_of([n])
    whole, _ = sel.prefill_attention(q, k, v, cu, cu.cuda(), window=window, sinks=sinks)
    for a, b in ((0, 129), (129, 131), (131, 300)):
        cq, ck = prefill.cu_of([b - a]), prefill.cu_of([b])
        part, _ = sel.prefill_attention(q[a:b], k[:b], v[:b], cq, cq.cuda(), ck, ck.cuda(), window=window, sinks=sinks)
        # Each within its tolerance of the same value: twice u |ref| + (u + 2e-5) sum p |v| + n 2^-25 8, with u = 2^-11
        # and sum p |v| below 1.5 for normal values: 2 u |ref| + 1.6e-3.
        assert torch.all((part - whole[a:b]).abs().float() <= 3 * 2.0 ** -11 * whole[a:b].abs().float() + 2e-3)
    per = -(-n // 64)
    pages = [torch.zeros((per, HKV, 64, D), dtype=dtype, device="cuda") for _ in range(2)]
    for x, p in ((k, pages[0]), (v, pages[1])):
        p.copy_(torch.nn.functional.pad(x, (0, 0, 0, 0, 0, per * 64 - n)).view(per, 64, HKV, D).transpose(1, 2))
    table = torch.arange(per, dtype=torch.int32)[None].cuda()
    for m in (300, 150, 101, 100, 5, 1):
        cache = kvec.PagedCache(pages[0], pages[1], table, torch.tensor([m], dtype=torch.int32).cuda())
        row = sel.paged_decode(q[m - 1:m].contiguous(), cache, window=window, sinks=sinks)
        assert torch.all((row - whole[m - 1:m]).abs().float() <= 3 * 2.0 ** -11 * whole[m - 1:m].abs().float() + 2e-3)
    sel.close()


# Kernels are programmatic dependents of what precedes them on the stream; in a caller's captured graph that
# may be a copy, a fill or another stream's kernel, whose results they must still see.
@pytest.mark.parametrize("before", ["copy", "fill", "other stream"])
@pytest.mark.parametrize("call", ["rotate", "decode", "long decode", "evict", "prefill", "divided prefill"])
def test_captured_calls_see_the_work_before_them(before, call):
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda shape, dt=torch.bfloat16: torch.randn(shape, generator=gen, device="cuda").to(dt)
    sel = selector()
    n = {"decode": 300, "long decode": 20000, "evict": 4000}.get(call, 900)
    per = -(-n // 64)
    pool = (2 * per, HKV, 64, D)
    table = torch.arange(per, dtype=torch.int32)[None].cuda()
    lens, lens_src = torch.zeros(1, dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    outs = []
    if call in ("decode", "long decode", "evict"):
        a, b, w = torch.zeros(pool, dtype=torch.bfloat16, device="cuda"), rand(pool), torch.zeros(pool[:3], device="cuda")
        srcs = [rand(pool), rand(pool[:3], torch.float32).abs()]
        fills = [a, w]
        cache = kvec.PagedCache(a, b, table, lens, w)
        q = rand((1, HQ, D))
        if call == "evict":
            fresh = (table + per).contiguous()
            run = lambda: (*sel.paged_evict(cache, fresh, 1000, sinks=2, recent=9), a, b, w)
        else:
            run = lambda: (sel.paged_decode(q, cache), w)
    else:
        few = call == "divided prefill"
        rows = 20 if few else n
        a, k, v = torch.zeros((rows, HQ, D), dtype=torch.bfloat16, device="cuda"), rand((n, HKV, D)), rand((n, HKV, D))
        srcs, fills = [rand((rows, HQ, D))], [a]
        cq, ck = prefill.cu_of([rows]), prefill.cu_of([n])
        dq, dk = cq.cuda(), ck.cuda()
        pos, tab = torch.arange(n, dtype=torch.int32).cuda(), paged.rot_table(n, D).cuda()
        cache = kvec.PagedCache(rand(pool), rand(pool), table, lens)
        if call == "rotate":
            run = lambda: (sel.rotate_append(a, k, v, pos, tab, cache, dq), cache.k_pages[:per - 1], cache.v_pages[:per - 1])
        else:
            run = lambda: sel.prefill_attention(a, k, v, cq, dq, ck, dk)
    side, main = torch.cuda.Stream(), torch.cuda.Stream()

    def work():
        if before == "copy":
            for f, s in zip(fills, srcs):
                f.copy_(s)
            lens.copy_(lens_src)
        elif before == "fill":
            for f, s in zip(fills, srcs):
                f.copy_(s)
            lens.copy_(lens_src)
            fills[0].zero_()
        else:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for f, s in zip(fills, srcs):
                    torch.add(s, 1.0, out=f)
                torch.add(lens_src, 0, out=lens)
            torch.cuda.current_stream().wait_stream(side)
        return run()

    with torch.cuda.stream(main):
        work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            got = work()
        for _ in range(3):
            for s in srcs:
                s.copy_(torch.randn(s.shape, generator=gen, device="cuda").abs().to(s.dtype))
            want = [x.clone() for x in work()]
            torch.cuda.synchronize()
            for f in fills:
                f.fill_(0.5)
            lens.fill_(n // 2)
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(want, got):
                assert torch.equal(x, y)
    sel.close()


@pytest.mark.parametrize("call", ["decode", "long decode", "prefill", "divided prefill"])
def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(call):
    gen = torch.Generator().manual_seed(4)
    sel = selector()
    if "decode" in call:
        lens = [100 if call == "decode" else 20000]
        cache, _ = paged.make_cache(lens, HKV, 64, torch.bfloat16, gen, weights=False)
        q = torch.randn((1, HQ, D), generator=gen).to(torch.bfloat16).cuda()
        run = lambda: sel.paged_decode(q, cache)
    else:
        rows = 700 if call == "prefill" else 5
        q, k, v = prefill.tensors([rows], [700], HQ, HKV, torch.bfloat16, 6)
        cq, ck = prefill.cu_of([rows]), prefill.cu_of([700])
        run = lambda: sel.prefill_attention(q, k, v, cq, cq.cuda(), ck, ck.cuda())[0]
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
    kvec.kvec_sync_status(sel.handle)
    sel.close()


@pytest.mark.parametrize("call", ["rotate", "decode", "evict", "prefill"])
def test_inputs_of_a_call_on_another_stream_may_be_let_go(call):
    # The call waits behind a long one on its stream; its inputs are let go at once, and the next tensors of their sizes
    # are written on the current stream meanwhile.
    gen = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    sel, n = selector(), 700
    per = -(-n // 64)
    pool = (2 * per, HKV, 64, D)
    fixed = [rand(*pool), rand(*pool), torch.arange(per, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32).cuda(),
             torch.rand(pool[:3], generator=gen, device="cuda")]
    if call == "rotate":
        given = [rand(n, HQ, D), rand(n, HKV, D), rand(n, HKV, D), torch.arange(n, dtype=torch.int32).cuda(),
                 paged.rot_table(n, D).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(), rand(D), rand(D)]
        run = lambda c, x, **kw: (*sel.rotate_append(*x[:5], c, x[5], q_norm=x[6], k_norm=x[7], k_out=torch.empty_like(x[1]), **kw),
                                  c.k_pages, c.v_pages)
    elif call == "decode":
        given = [rand(1, HQ, D)]
        run = lambda c, x, **kw: (sel.paged_decode(x[0], c, **kw), c.weights)
    elif call == "evict":
        given = [torch.arange(per, 2 * per, dtype=torch.int32, device="cuda")[None].clone()]
        run = lambda c, x, **kw: (*sel.paged_evict(c, x[0], 300, sinks=2, recent=9, **kw), c.k_pages, c.v_pages, c.weights)
    else:
        cu = prefill.cu_of([n])
        given = [rand(n, HQ, D), rand(n, HKV, D), rand(n, HKV, D), cu.cuda()]
        run = lambda c, x, **kw: sel.prefill_attention(*x[:3], cu, x[3], **kw)
    fresh = lambda: (kvec.PagedCache(*[x.clone() for x in fixed]), [x.clone() for x in given])
    want = [x.clone() for x in run(*fresh())]
    side = torch.cuda.Stream()
    run(*fresh(), stream=side)                          # the side stream's first allocations
    cache, x = fresh()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    got = run(cache, x, stream=side)
    del cache, x
    junk = [torch.full_like(t, 77) for t in given + fixed for _ in range(12)]
    kvec.kvec_sync_status(sel.handle)
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want)) and junk
    sel.close()
